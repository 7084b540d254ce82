"""Operators of a block of experts and of distillation on torch tensors: routing,
products grouped by expert, the combination of a token's rows, and the loss against a
teacher's most likely tokens.  They follow the conventions of ``operators.py``: the
functions named ``isoloco_*`` marshal the C functions of that name, the others check
tensors, allocate what is not given, enqueue on the current torch stream (or ``stream``)
and hand gradients to autograd where an operand requires one.

A block of experts over ``x`` [tokens, dim]:

    r = route_tokens(scores, top_k)                                  # scores [tokens, experts]
    h = expert_matmul(x, w, r.offsets, token=r.token, row=r.row)     # w [experts, hidden, dim], rows by expert
    y = expert_matmul(act(h), w_down, r.offsets)                     # w_down [experts, dim, hidden]
    out = combine_tokens(y, r.row, r.weight)

A student against a teacher:

    with torch.no_grad():
        t = token_logprobs(teacher_logits, scale=scale, top_k=32)
    loss = distill_loss(logits, t.top_logprob, t.top_index, scale=scale).loss
"""
from typing import NamedTuple

import torch
from torch.autograd.function import once_differentiable

from . import (ISOLOCO_EXPERTS_ALIGNED, ISOLOCO_EXPERTS_BACKWARD, ISOLOCO_EXPERTS_GATHERED, ISOLOCO_DISTILL_STATS,
               ISOLOCO_MAX_TOP, ISOLOCO_REST_BUCKET, ISOLOCO_REST_DROP, _check, _lib)
from .operators import (_empty, _F32, _ids, _output, _place, _raw_stream, _recorded, _rows, _same_device, _size_of,
                        _type, _vector, _with_stream, _workspace, _written)

_REST = {"drop": ISOLOCO_REST_DROP, "bucket": ISOLOCO_REST_BUCKET}
_LD = 1 << 22  # rows further apart are copied


# --------------------------------------------------------------------------
# The C functions
# --------------------------------------------------------------------------

def isoloco_route_tokens_workspace_size(tokens, experts):
    return _size_of("isoloco_route_tokens_workspace_size", tokens, experts)


def isoloco_route_tokens(scores, ld_scores, dtype, tokens, experts, top_k, normalize, weight, expert, row, token,
                         offsets, workspace, workspace_bytes, stream=0):
    _check(_lib.isoloco_route_tokens(scores, ld_scores, dtype, tokens, experts, top_k, normalize, weight, expert, row,
                                     token, offsets, workspace, workspace_bytes, stream), "isoloco_route_tokens")


def isoloco_route_tokens_backward(scores, ld_scores, dtype, tokens, experts, top_k, normalize, expert, dweight,
                                  dscores, ld_dscores, stream=0):
    _check(_lib.isoloco_route_tokens_backward(scores, ld_scores, dtype, tokens, experts, top_k, normalize, expert,
                                              dweight, dscores, ld_dscores, stream), "isoloco_route_tokens_backward")


def isoloco_expert_matmul_workspace_size(tokens, rows, experts, dim, cols, ld_x, dtype, flags):
    return _size_of("isoloco_expert_matmul_workspace_size", tokens, rows, experts, dim, cols, ld_x, dtype, flags)


def isoloco_expert_matmul(x, ld_x, tokens, token, w, ld_w, stride_w, dtype, offsets, index_type, experts, rows, dim,
                          cols, out, ld_out, workspace, workspace_bytes, stream=0):
    _check(_lib.isoloco_expert_matmul(x, ld_x, tokens, token, w, ld_w, stride_w, dtype, offsets, index_type, experts,
                                      rows, dim, cols, out, ld_out, workspace, workspace_bytes, stream),
           "isoloco_expert_matmul")


def isoloco_expert_matmul_backward(x, ld_x, tokens, token, w, ld_w, stride_w, dtype, offsets, index_type, experts,
                                   rows, dim, cols, dout, ld_dout, dx, ld_dx, dw, ld_dw, stride_dw, workspace,
                                   workspace_bytes, stream=0):
    _check(_lib.isoloco_expert_matmul_backward(x, ld_x, tokens, token, w, ld_w, stride_w, dtype, offsets, index_type,
                                               experts, rows, dim, cols, dout, ld_dout, dx, ld_dx, dw, ld_dw,
                                               stride_dw, workspace, workspace_bytes, stream),
           "isoloco_expert_matmul_backward")


def isoloco_expert_matmul_backward_tokens(x, ld_x, tokens, token, row, row_type, top_k, w, ld_w, stride_w, dtype, offsets,
                                          index_type, experts, rows, dim, cols, dout, ld_dout, dx, ld_dx, dx_rows, dw,
                                          ld_dw, stride_dw, workspace, workspace_bytes, stream=0):
    _check(_lib.isoloco_expert_matmul_backward_tokens(x, ld_x, tokens, token, row, row_type, top_k, w, ld_w, stride_w,
                                                      dtype, offsets, index_type, experts, rows, dim, cols, dout,
                                                      ld_dout, dx, ld_dx, dx_rows, dw, ld_dw, stride_dw, workspace,
                                                      workspace_bytes, stream), "isoloco_expert_matmul_backward_tokens")


def isoloco_combine_tokens(y, ld_y, dtype, rows, dim, row, index_type, weight, tokens, top_k, out, ld_out, stream=0):
    _check(_lib.isoloco_combine_tokens(y, ld_y, dtype, rows, dim, row, index_type, weight, tokens, top_k, out, ld_out,
                                       stream), "isoloco_combine_tokens")


def isoloco_combine_tokens_backward_workspace_size(tokens, top_k):
    return _size_of("isoloco_combine_tokens_backward_workspace_size", tokens, top_k)


def isoloco_combine_tokens_backward(dout, ld_dout, y, ld_y, dtype, rows, dim, row, index_type, weight, tokens, top_k,
                                    dy, ld_dy, dweight, workspace, workspace_bytes, stream=0):
    _check(_lib.isoloco_combine_tokens_backward(dout, ld_dout, y, ld_y, dtype, rows, dim, row, index_type, weight,
                                                tokens, top_k, dy, ld_dy, dweight, workspace, workspace_bytes, stream),
           "isoloco_combine_tokens_backward")


def isoloco_distill_loss_workspace_size(rows, vocab):
    return _size_of("isoloco_distill_loss_workspace_size", rows, vocab)


def isoloco_distill_loss(logits, ld_logits, dtype, rows, vocab, top_logprob, top_index, index_type, top_k, scale, rest,
                         loss, stats, workspace, workspace_bytes, stream=0):
    _check(_lib.isoloco_distill_loss(logits, ld_logits, dtype, rows, vocab, top_logprob, top_index, index_type, top_k,
                                     scale, rest, loss, stats, workspace, workspace_bytes, stream),
           "isoloco_distill_loss")


def isoloco_distill_loss_backward(logits, ld_logits, dtype, rows, vocab, top_logprob, top_index, index_type, top_k,
                                  scale, rest, stats, dloss, dlogits, ld_dlogits, stream=0):
    _check(_lib.isoloco_distill_loss_backward(logits, ld_logits, dtype, rows, vocab, top_logprob, top_index,
                                              index_type, top_k, scale, rest, stats, dloss, dlogits, ld_dlogits,
                                              stream), "isoloco_distill_loss_backward")


# --------------------------------------------------------------------------
# Routing
# --------------------------------------------------------------------------

class TokenRoutes(NamedTuple):
    """What ``route_tokens`` returns.  ``weight`` (float32) hands a gradient back; the
    others are int32."""
    weight: torch.Tensor   # [tokens, top_k]
    expert: torch.Tensor   # [tokens, top_k], -1: none
    row: torch.Tensor      # [tokens, top_k]: the slot's place in the experts' order
    token: torch.Tensor    # [tokens * top_k]: the place's token
    offsets: torch.Tensor  # [experts + 1]: where each expert's places begin


def _scores(scores):
    index = _place(scores)
    if scores.dim() != 2:
        raise ValueError("scores must be [tokens, experts]")
    dtype = _type("scores", scores)
    return index, dtype, scores.shape[0], scores.shape[1], _rows("scores", scores)[1]


@_with_stream
def route_tokens(scores, top_k, normalize=True, workspace=None):
    """The ``top_k`` experts of each token by its ``scores`` [tokens, experts], their
    weights (the softmax of the chosen scores, or without ``normalize`` the softmax of
    all of them), and the order of the slots by expert.  A score of -infinity is not
    chosen: slots that find no expert have expert -1 and weight 0 and come last."""
    if scores.requires_grad and _recorded(None):
        return TokenRoutes(*_RouteTokens.apply(scores, top_k, normalize, workspace))
    index, dtype, tokens, experts, ld = _scores(scores)
    if not 1 <= top_k <= experts:
        raise ValueError("top_k must be of 1 to %d, not %d" % (experts, top_k))
    device = scores.device
    keep, ws, ws_bytes = _workspace(workspace, isoloco_route_tokens_workspace_size(tokens, experts), device)
    weight = _empty(tokens, top_k, dtype=_F32, device=device)
    expert = _empty(tokens, top_k, dtype=torch.int32, device=device)
    row = _empty(tokens, top_k, dtype=torch.int32, device=device)
    token = _empty(tokens * top_k, dtype=torch.int32, device=device)
    offsets = _empty(experts + 1, dtype=torch.int32, device=device)
    _check(_lib.isoloco_route_tokens(scores.data_ptr(), ld, dtype, tokens, experts, top_k, 1 if normalize else 0,
                                     weight.data_ptr(), expert.data_ptr(), row.data_ptr(), token.data_ptr(),
                                     offsets.data_ptr(), ws, ws_bytes, _raw_stream(index)), "isoloco_route_tokens")
    return TokenRoutes(weight, expert, row, token, offsets)


@_with_stream
def route_tokens_backward(scores, expert, dweight, normalize=True):
    """The gradient in the scores from that of ``route_tokens``' weight, given its expert."""
    index, dtype, tokens, experts, ld = _scores(scores)
    _same_device(index, expert, dweight)
    if expert.dtype != torch.int32 or not expert.is_contiguous() or expert.dim() != 2 or expert.shape[0] != tokens:
        raise ValueError("expert must be contiguous int32 of [tokens, top_k]")
    top_k = expert.shape[1]
    d_at = _vector("dweight", dweight, expert.numel())
    out = _empty(tokens, experts, dtype=scores.dtype, device=scores.device)
    _check(_lib.isoloco_route_tokens_backward(scores.data_ptr(), ld, dtype, tokens, experts, top_k,
                                              1 if normalize else 0, expert.data_ptr(), d_at, out.data_ptr(), experts,
                                              _raw_stream(index)), "isoloco_route_tokens_backward")
    return out


class _RouteTokens(torch.autograd.Function):
    @staticmethod
    def forward(ctx, scores, top_k, normalize, workspace):
        r = route_tokens(scores, top_k, normalize, workspace)
        ctx.save_for_backward(scores, r.expert)
        ctx.normalize = normalize
        ctx.mark_non_differentiable(*r[1:])
        return tuple(r)

    @staticmethod
    @once_differentiable
    def backward(ctx, dweight, *_):
        scores, expert = ctx.saved_tensors
        return route_tokens_backward(scores, expert, dweight.contiguous(), ctx.normalize), None, None, None


# --------------------------------------------------------------------------
# Products grouped by expert
# --------------------------------------------------------------------------

def _expert_operands(x, w, offsets, token):
    index = _place(x)
    _same_device(index, w, offsets, token)
    dtype = _type("x", x)
    if w.dim() != 3 or w.dtype != x.dtype:
        raise ValueError("w must be [experts, cols, dim] of x's type")
    experts, cols, dim = w.shape
    if x.dim() != 2 or x.shape[1] != dim:
        raise ValueError("x must be [rows, %d], not %s" % (dim, tuple(x.shape)))
    tokens, ld_x = _rows("x", x)
    ld_w, stride_w = w.stride(1) if cols > 1 else dim, w.stride(0)
    if dim > 1 and w.stride(2) != 1:
        raise ValueError("w must have unit stride along its last dimension")
    if experts == 1:
        stride_w = cols * ld_w
    if ld_w < dim or stride_w < (cols - 1) * ld_w + dim:
        raise ValueError("w: its rows overlap")
    rows, token_at = tokens, None
    index_type = _ids("offsets", offsets, experts + 1)
    if token is not None:
        rows = token.numel()
        if _ids("token", token, rows) != index_type:
            raise ValueError("offsets and token must be of one type")
        token_at = token.data_ptr()
    at = x.data_ptr(), w.data_ptr()
    aligned = not ((dim | cols | ld_x | ld_w | stride_w) & 7 or (at[0] | at[1]) & 15) and ld_x <= _LD and ld_w <= _LD
    flags = (ISOLOCO_EXPERTS_ALIGNED if aligned else 0) | (ISOLOCO_EXPERTS_GATHERED if token is not None else 0)
    return index, dtype, tokens, rows, experts, dim, cols, ld_x, ld_w, stride_w, index_type, token_at, at, flags


def _row_of(index, row, tokens):
    """Where row [tokens, top_k], the rows of each token, lies, and its type."""
    if row is None:
        raise ValueError("the gradient of x needs row beside token")
    _same_device(index, row)
    if row.dim() != 2 or row.shape[0] != tokens or not 1 <= row.shape[1] <= ISOLOCO_MAX_TOP:
        raise ValueError("row must be [%d, 1 to %d], not %s" % (tokens, ISOLOCO_MAX_TOP, tuple(row.shape)))
    return row.data_ptr(), _ids("row", row, row.numel())


@_with_stream
def expert_matmul(x, w, offsets, token=None, row=None, out=None, workspace=None):
    """``x_r w[e]^T`` for the rows r = offsets[e] .. offsets[e + 1] - 1 of each expert e, w
    [experts, cols, dim]; x_r is ``x[token[r]]`` (x [tokens, dim]), or ``x[r]`` without
    ``token``.  Rows from offsets[-1] on are zeros.  offsets and token are int32 or int64
    and are not read by the host.  ``row`` (``route_tokens``' inverse of token, [tokens,
    top_k]) is needed with ``token`` for the gradient of x."""
    if (x.requires_grad or w.requires_grad) and _recorded(out):
        if token is not None and x.requires_grad:
            _row_of(_place(x), row, x.shape[0])  # (now: it is read by the gradient alone)
        return _ExpertMatmul.apply(x, w, offsets, token, row, workspace)
    index, dtype, tokens, rows, experts, dim, cols, ld_x, ld_w, stride_w, index_type, token_at, at, flags = \
        _expert_operands(x, w, offsets, token)
    if out is None:
        out = _empty(rows, cols, dtype=x.dtype, device=x.device)
        ld_out = cols
    else:
        _same_device(index, out)
        _output("out", out, (rows, cols), x.dtype)
        ld_out = _rows("out", out)[1]
        _written(out)
    keep, ws, ws_bytes = _workspace(workspace, isoloco_expert_matmul_workspace_size(
        tokens, rows, experts, dim, cols, ld_x, dtype, flags), x.device)
    _check(_lib.isoloco_expert_matmul(at[0], ld_x, tokens, token_at, at[1], ld_w, stride_w, dtype, offsets.data_ptr(),
                                      index_type, experts, rows, dim, cols, out.data_ptr(), ld_out, ws, ws_bytes,
                                      _raw_stream(index)), "isoloco_expert_matmul")
    return out


@_with_stream
def expert_matmul_backward(x, w, offsets, dout, token=None, row=None, need_dx=True, need_dw=True, workspace=None):
    """(dx, dw) from ``dout`` [rows, cols]; None for what is not needed.  With ``token``, dx
    is the sum over a token's rows, which ``row`` [tokens, top_k] names, of float32 and
    rounded once."""
    index, dtype, tokens, rows, experts, dim, cols, ld_x, ld_w, stride_w, index_type, token_at, at, flags = \
        _expert_operands(x, w, offsets, token)
    _same_device(index, dout)
    if dout.dtype != x.dtype or tuple(dout.shape) != (rows, cols):
        raise ValueError("dout must be %s of %s" % (x.dtype, (rows, cols)))
    ld_dout, device = _rows("dout", dout)[1], x.device
    d_at = dout.data_ptr()
    if d_at & 15 or ld_dout & 7 or ld_dout > _LD:
        flags &= ~ISOLOCO_EXPERTS_ALIGNED
    dx = dw = dx_at = dw_at = None
    sums = need_dx and token is not None
    if sums:
        row_at, row_type = _row_of(index, row, tokens)
    if need_dx:
        dx = _empty(tokens if sums else rows, dim, dtype=x.dtype, device=device)
        dx_at = dx.data_ptr()
    if need_dw:
        dw = _empty(experts, cols, dim, dtype=x.dtype, device=device)
        dw_at = dw.data_ptr()
    keep, ws, ws_bytes = _workspace(workspace, isoloco_expert_matmul_workspace_size(
        tokens, rows, experts, dim, cols, ld_x, dtype, flags | ISOLOCO_EXPERTS_BACKWARD), device)
    if sums:
        dx_rows = _empty(rows, dim, dtype=_F32, device=device)
        _check(_lib.isoloco_expert_matmul_backward_tokens(
            at[0], ld_x, tokens, token_at, row_at, row_type, row.shape[1], at[1], ld_w,
            stride_w, dtype, offsets.data_ptr(), index_type, experts, rows, dim, cols, d_at, ld_dout, dx_at, dim,
            dx_rows.data_ptr(), dw_at, dim, cols * dim, ws, ws_bytes, _raw_stream(index)),
            "isoloco_expert_matmul_backward_tokens")
        return dx, dw
    _check(_lib.isoloco_expert_matmul_backward(at[0], ld_x, tokens, token_at, at[1], ld_w, stride_w, dtype,
                                               offsets.data_ptr(), index_type, experts, rows, dim, cols, d_at, ld_dout,
                                               dx_at, dim, dw_at, dim, cols * dim, ws, ws_bytes, _raw_stream(index)),
           "isoloco_expert_matmul_backward")
    return dx, dw


class _ExpertMatmul(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, offsets, token, row, workspace):
        ctx.save_for_backward(x, w, offsets, token, row)
        return expert_matmul(x, w, offsets, token, workspace=workspace)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        x, w, offsets, token, row = ctx.saved_tensors
        dx, dw = expert_matmul_backward(x, w, offsets, dout.contiguous(), token, row, *ctx.needs_input_grad[:2])
        return dx, dw, None, None, None, None


# --------------------------------------------------------------------------
# Combination
# --------------------------------------------------------------------------

def _combine_operands(y, row, weight):
    index = _place(y)
    _same_device(index, row, weight)
    dtype = _type("y", y)
    if y.dim() != 2 or row.dim() != 2:
        raise ValueError("y must be [rows, dim] and row [tokens, top_k]")
    rows, ld_y = _rows("y", y)
    tokens, top_k = row.shape
    weight_at = None
    if weight is not None:
        if weight.shape != row.shape:
            raise ValueError("weight must be %s, not %s" % (tuple(row.shape), tuple(weight.shape)))
        weight_at = _vector("weight", weight, row.numel())
    return index, dtype, rows, y.shape[1], ld_y, tokens, top_k, _ids("row", row, row.numel()), weight_at


@_with_stream
def combine_tokens(y, row, weight=None, out=None):
    """``sum_j weight[t, j] * y[row[t, j]]`` for y [rows, dim], row (int32 or int64) and
    weight (float32, or None for ones) [tokens, top_k].  Entries of row outside y add
    nothing.  For the gradient no two entries may be the same."""
    if (y.requires_grad or (weight is not None and weight.requires_grad)) and _recorded(out):
        return _CombineTokens.apply(y, row, weight)
    index, dtype, rows, dim, ld_y, tokens, top_k, index_type, weight_at = _combine_operands(y, row, weight)
    if out is None:
        out = _empty(tokens, dim, dtype=y.dtype, device=y.device)
        ld_out = dim
    else:
        _same_device(index, out)
        _output("out", out, (tokens, dim), y.dtype)
        ld_out = _rows("out", out)[1]
        _written(out)
    _check(_lib.isoloco_combine_tokens(y.data_ptr(), ld_y, dtype, rows, dim, row.data_ptr(), index_type, weight_at,
                                       tokens, top_k, out.data_ptr(), ld_out, _raw_stream(index)),
           "isoloco_combine_tokens")
    return out


@_with_stream
def combine_tokens_backward(dout, y, row, weight=None, need_dy=True, need_dweight=True, workspace=None):
    """(dy, dweight) from ``dout`` [tokens, dim]; None for what is not needed (dweight
    without weight).  No two entries of ``row`` may be the same (the row's gradient is then
    from any of them); rows of y that none names have a zero gradient."""
    index, dtype, rows, dim, ld_y, tokens, top_k, index_type, weight_at = _combine_operands(y, row, weight)
    _same_device(index, dout)
    if dout.dtype != y.dtype or tuple(dout.shape) != (tokens, dim):
        raise ValueError("dout must be %s of %s" % (y.dtype, (tokens, dim)))
    ld_dout, device = _rows("dout", dout)[1], y.device
    dy = dweight = dy_at = dweight_at = keep = ws = None
    ws_bytes = 0
    if need_dy:
        dy = _empty(rows, dim, dtype=y.dtype, device=device)
        dy_at = dy.data_ptr()
        keep, ws, ws_bytes = _workspace(workspace, isoloco_combine_tokens_backward_workspace_size(tokens, top_k), device)
    if need_dweight and weight is not None:
        dweight = _empty(tokens, top_k, dtype=_F32, device=device)
        dweight_at = dweight.data_ptr()
    _check(_lib.isoloco_combine_tokens_backward(dout.data_ptr(), ld_dout, y.data_ptr(), ld_y, dtype, rows, dim,
                                                row.data_ptr(), index_type, weight_at, tokens, top_k, dy_at, dim,
                                                dweight_at, ws, ws_bytes, _raw_stream(index)),
           "isoloco_combine_tokens_backward")
    return dy, dweight


class _CombineTokens(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, row, weight):
        ctx.save_for_backward(y, row, weight)
        return combine_tokens(y, row, weight)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        y, row, weight = ctx.saved_tensors
        dy, dweight = combine_tokens_backward(dout.contiguous(), y, row, weight, ctx.needs_input_grad[0],
                                              ctx.needs_input_grad[2])
        return dy, None, dweight


# --------------------------------------------------------------------------
# Distillation
# --------------------------------------------------------------------------

class DistillLoss(NamedTuple):
    """What ``distill_loss`` returns: ``loss`` (float32, the logits' leading shape) hands a
    gradient back; ``stats`` is what ``distill_loss_backward`` takes."""
    loss: torch.Tensor
    stats: torch.Tensor


def _distill_operands(logits, top_logprob, top_index, rest):
    index = _place(logits)
    _same_device(index, top_logprob, top_index)
    dtype = _type("logits", logits)
    rows, ld = _rows("logits", logits)
    if top_index.shape != top_logprob.shape or top_index.shape[:-1] != logits.shape[:-1]:
        raise ValueError("top_logprob and top_index must have the logits' leading shape and one more dimension")
    if top_logprob.requires_grad and torch.is_grad_enabled():
        raise ValueError("the teacher's log probabilities carry no gradient: detach them")
    mode = _REST.get(rest)
    if mode is None:
        raise ValueError("rest must be one of %s" % ", ".join(sorted(_REST)))
    return (index, dtype, rows, ld, logits.shape[-1], top_index.shape[-1], _vector("top_logprob", top_logprob,
            top_logprob.numel()), _ids("top_index", top_index, top_index.numel()), mode)


@_with_stream
def distill_loss(logits, top_logprob, top_index, scale=1.0, rest="drop", workspace=None):
    """The divergence of softmax(scale * logits) from a teacher of which each row has its
    most likely tokens, ``top_index`` (int32 or int64; entries outside the vocabulary
    are none) with ``top_logprob`` (float32), [..., top_k] each, as ``token_logprobs``
    gives them.  ``rest``: "drop" compares the listed tokens alone, the teacher's
    probabilities over their sum; "bucket" compares all others' sum as one more.  Mask
    logits with -infinity: where every other column has a large finite one, the bucket is
    as far from the teacher's as that says."""
    if logits.requires_grad and _recorded(None):
        if top_logprob.requires_grad:
            raise ValueError("the teacher's log probabilities carry no gradient: detach them")
        return DistillLoss(*_DistillLoss.apply(logits, top_logprob, top_index, scale, rest, workspace))
    index, dtype, rows, ld, vocab, top_k, top_at, index_type, mode = _distill_operands(logits, top_logprob, top_index,
                                                                                       rest)
    device = logits.device
    keep, ws, ws_bytes = _workspace(workspace, isoloco_distill_loss_workspace_size(rows, vocab), device)
    loss = _empty(*logits.shape[:-1], dtype=_F32, device=device)
    stats = _empty(*logits.shape[:-1], ISOLOCO_DISTILL_STATS, dtype=_F32, device=device)
    _check(_lib.isoloco_distill_loss(logits.data_ptr(), ld, dtype, rows, vocab, top_at, top_index.data_ptr(),
                                     index_type, top_k, scale, mode, loss.data_ptr(), stats.data_ptr(), ws, ws_bytes,
                                     _raw_stream(index)), "isoloco_distill_loss")
    return DistillLoss(loss, stats)


@_with_stream
def distill_loss_backward(logits, top_logprob, top_index, stats, dloss, scale=1.0, rest="drop", out=None):
    """The gradient in the logits from that of ``distill_loss``' loss, given its stats;
    ``out`` may be ``logits`` itself."""
    index, dtype, rows, ld, vocab, top_k, top_at, index_type, mode = _distill_operands(logits, top_logprob, top_index,
                                                                                       rest)
    _same_device(index, stats, dloss, out)
    stats_at, dloss_at = _vector("stats", stats, rows * ISOLOCO_DISTILL_STATS), _vector("dloss", dloss, rows)
    if out is None:
        out = _empty(*logits.shape, dtype=logits.dtype, device=logits.device)
        ld_out = vocab
    else:
        _output("out", out, logits.shape, logits.dtype)
        ld_out = _rows("out", out)[1]
        _written(out)
    _check(_lib.isoloco_distill_loss_backward(logits.data_ptr(), ld, dtype, rows, vocab, top_at, top_index.data_ptr(),
                                              index_type, top_k, scale, mode, stats_at, dloss_at, out.data_ptr(),
                                              ld_out, _raw_stream(index)), "isoloco_distill_loss_backward")
    return out


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, top_logprob, top_index, scale, rest, workspace):
        r = distill_loss(logits, top_logprob, top_index, scale, rest, workspace)
        ctx.save_for_backward(logits, top_logprob, top_index, r.stats)
        ctx.scale, ctx.rest = scale, rest
        ctx.mark_non_differentiable(r.stats)
        return tuple(r)

    @staticmethod
    @once_differentiable
    def backward(ctx, dloss, _):
        logits, top_logprob, top_index, stats = ctx.saved_tensors
        d = distill_loss_backward(logits, top_logprob, top_index, stats, dloss.contiguous(), ctx.scale, ctx.rest)
        return d, None, None, None, None, None

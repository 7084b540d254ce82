"""Operators of the workers' inner training step on torch tensors.

The functions named ``isoloco_*`` have the name and the argument order of the C
functions they marshal (``include/isoloco.h``) and take addresses.  The others
take tensors: they check shapes, types and strides (``ValueError``), allocate
what is not given with torch's allocator, and enqueue on the current torch
stream (or ``stream``, a raw stream handle) of the current device, where the tensors
have to be.  Matrices
need unit stride along a row; a further leading dimension is allowed where the
rows stay evenly spaced.  Arguments that the library itself refuses raise
``IsoLoCoError``.

``embedding``, ``token_logprobs`` and ``gated_ffn`` are differentiable: where an
operand requires a gradient, the result carries the function that forms it (once:
there is no second derivative).  ``out`` is refused then, as torch's functions do.
"""
import array
import ctypes
import functools
from typing import NamedTuple, Optional

import torch
from torch.autograd.function import once_differentiable

from . import (ISOLOCO_ACT_GELU, ISOLOCO_ACT_SILU, ISOLOCO_BF16, ISOLOCO_F32, ISOLOCO_FFN_ALIGNED,
               ISOLOCO_FFN_BACKWARD, ISOLOCO_I32, ISOLOCO_I64, IsoLoCoError, _check, _lib)

_DTYPE = {torch.float32: ISOLOCO_F32, torch.bfloat16: ISOLOCO_BF16}
_INDEX = {torch.int32: ISOLOCO_I32, torch.int64: ISOLOCO_I64}
_FFN_LD = 1 << 22  # rows further apart are copied
_ACT = {"silu": ISOLOCO_ACT_SILU, "gelu": ISOLOCO_ACT_GELU}


# --------------------------------------------------------------------------
# The C functions
# --------------------------------------------------------------------------

@functools.lru_cache(maxsize=1024)
def _size_of(name, *args):
    # (a size is a function of its arguments alone)
    n = ctypes.c_size_t()
    status = getattr(_lib, name)(*args, ctypes.byref(n))
    if status:
        raise IsoLoCoError(status, name)
    return n.value


def isoloco_clip_workspace_size(n_tensors):
    return _size_of("isoloco_clip_workspace_size", n_tensors)


def isoloco_clip_grads(src, dst, counts, dtypes, max_norm, norm, workspace, workspace_bytes, stream=0):
    """src, dst (or None), counts, dtypes: sequences of one entry per tensor."""
    n = len(src)
    if len(counts) != n or len(dtypes) != n or (dst is not None and len(dst) != n):
        raise ValueError("src, dst, counts and dtypes must have one entry per tensor")
    s, c, t = array.array("Q", src), array.array("q", counts), array.array("i", dtypes)
    d = array.array("Q", dst) if dst is not None else None
    _check(_lib.isoloco_clip_grads(s.buffer_info()[0], d.buffer_info()[0] if d is not None else None,
                                   c.buffer_info()[0], t.buffer_info()[0], n, max_norm, norm, workspace,
                                   workspace_bytes, stream), "isoloco_clip_grads")


def isoloco_embedding(table, ld_table, dtype, vocab, dim, ids, id_type, n, scale, out, ld_out, out_dtype, stream=0):
    _check(_lib.isoloco_embedding(table, ld_table, dtype, vocab, dim, ids, id_type, n, scale, out, ld_out, out_dtype,
                                  stream), "isoloco_embedding")


def isoloco_embedding_backward_workspace_size(n, vocab, dim):
    return _size_of("isoloco_embedding_backward_workspace_size", n, vocab, dim)


def isoloco_embedding_backward(ids, id_type, n, dout, ld_dout, dtype, vocab, dim, scale, accumulate, dtable,
                               ld_dtable, dtable_dtype, workspace, workspace_bytes, stream=0):
    _check(_lib.isoloco_embedding_backward(ids, id_type, n, dout, ld_dout, dtype, vocab, dim, scale, accumulate,
                                           dtable, ld_dtable, dtable_dtype, workspace, workspace_bytes, stream),
           "isoloco_embedding_backward")


def isoloco_token_logprobs_workspace_size(rows, vocab, top_k):
    return _size_of("isoloco_token_logprobs_workspace_size", rows, vocab, top_k)


def isoloco_token_logprobs(logits, ld_logits, dtype, rows, vocab, targets, target_type, scale, top_k, logprob,
                           entropy, lse, top_logprob, top_index, workspace, workspace_bytes, stream=0):
    _check(_lib.isoloco_token_logprobs(logits, ld_logits, dtype, rows, vocab, targets, target_type, scale, top_k,
                                       logprob, entropy, lse, top_logprob, top_index, workspace, workspace_bytes,
                                       stream), "isoloco_token_logprobs")


def isoloco_token_logprobs_backward(logits, ld_logits, dtype, rows, vocab, targets, target_type, scale, lse, entropy,
                                    dlogprob, dentropy, dlogits, ld_dlogits, stream=0):
    _check(_lib.isoloco_token_logprobs_backward(logits, ld_logits, dtype, rows, vocab, targets, target_type, scale,
                                                lse, entropy, dlogprob, dentropy, dlogits, ld_dlogits, stream),
           "isoloco_token_logprobs_backward")


def isoloco_gated_ffn_workspace_size(tokens, dim, hidden, dtype, flags):
    return _size_of("isoloco_gated_ffn_workspace_size", tokens, dim, hidden, dtype, flags)


def isoloco_gated_ffn(x, ld_x, w_gate, w_up, ld_w, dtype, tokens, dim, hidden, act, out, ld_out, workspace,
                      workspace_bytes, stream=0):
    _check(_lib.isoloco_gated_ffn(x, ld_x, w_gate, w_up, ld_w, dtype, tokens, dim, hidden, act, out, ld_out,
                                  workspace, workspace_bytes, stream), "isoloco_gated_ffn")


def isoloco_gated_ffn_backward(x, ld_x, w_gate, w_up, ld_w, dtype, tokens, dim, hidden, act, dout, ld_dout, dx, ld_dx,
                               dw_gate, dw_up, ld_dw, workspace, workspace_bytes, stream=0):
    _check(_lib.isoloco_gated_ffn_backward(x, ld_x, w_gate, w_up, ld_w, dtype, tokens, dim, hidden, act, dout,
                                           ld_dout, dx, ld_dx, dw_gate, dw_up, ld_dw, workspace, workspace_bytes,
                                           stream), "isoloco_gated_ffn_backward")


# --------------------------------------------------------------------------
# Tensors
# --------------------------------------------------------------------------

# (the public functions make a Stream object per call, 2 us of a small operator's 10)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)
_empty = torch.empty  # (its sizes one by one: 0.3 us less than as a tuple)
_F32 = torch.float32


def _with_stream(f):
    """Adds ``stream`` (a raw handle): the call runs, and allocates, with it as the
    current stream."""
    @functools.wraps(f)
    def call(*args, stream=None, **kwargs):
        if stream is None:
            return f(*args, **kwargs)
        with torch.cuda.stream(torch.cuda.ExternalStream(stream)):
            return f(*args, **kwargs)
    return call


def _place(t):
    """The index of the device that t and the call are on."""
    index = t.get_device()
    if index < 0:
        raise ValueError("tensors must be on the GPU")
    if index != torch.cuda.current_device():
        raise ValueError("the tensors are on device %d, the current device is %d" %
                         (index, torch.cuda.current_device()))
    return index


def _same_device(index, *tensors):
    for t in tensors:
        if t is not None and t.get_device() != index:
            raise ValueError("the tensors are on different devices")


def _workspace(given, need, device):
    """(tensor, address, bytes) of ``given`` (uint8) or of a new one, 256-byte aligned."""
    if need == 0:
        return None, None, 0
    if given is None:
        given = _empty(need + 255, dtype=torch.uint8, device=device)
    elif given.dtype != torch.uint8 or not given.is_contiguous() or given.device != device:
        raise ValueError("workspace must be a contiguous uint8 tensor on the operands' device")
    base = given.data_ptr()
    at = (base + 255) // 256 * 256
    return given, at, max(0, base + given.numel() - at)


def _type(name, t):
    d = _DTYPE.get(t.dtype)
    if d is None:
        raise ValueError("%s must be float32 or bfloat16, not %s" % (name, t.dtype))
    return d


def _rows(name, t):
    """(rows, ld) of a tensor seen as a matrix of its last dimension's rows."""
    if t.is_contiguous():
        if not t.dim():
            raise ValueError("%s must have a dimension" % name)
        c = t.shape[-1]
        return (t.numel() // c if c else 0), c
    c = t.shape[-1]
    n = t.numel() // c if c else 0
    if c > 1 and t.stride(-1) != 1:
        raise ValueError("%s must have unit stride along its last dimension" % name)
    if t.dim() == 2:
        ld = t.stride(0) if t.shape[0] > 1 else c
    else:
        try:
            flat = t.view(-1, c)
        except RuntimeError:
            raise ValueError("%s: its rows are not evenly spaced" % name) from None
        ld = flat.stride(0) if n > 1 else c
    if ld < c:
        raise ValueError("%s: its rows overlap" % name)
    return n, ld


def _ids(name, t, n):
    i = _INDEX.get(t.dtype)
    if i is None:
        raise ValueError("%s must be int32 or int64, not %s" % (name, t.dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if t.numel() != n:
        raise ValueError("%s must have %d elements, not %d" % (name, n, t.numel()))
    return i


def _vector(name, t, n):
    if t.dtype != _F32 or not t.is_contiguous() or t.numel() != n:
        raise ValueError("%s must be contiguous float32 of %d elements" % (name, n))
    return t.data_ptr()


def _output(name, t, shape, dtype):
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype:
        raise ValueError("%s must be %s of %s" % (name, dtype, tuple(shape)))
    return t


# raises tensors' version counters, by which autograd finds that one it kept has changed
_written = torch.autograd.graph.increment_version


def _recorded(out):
    """Whether a call with an operand that requires a gradient is recorded for one."""
    if not torch.is_grad_enabled():
        return False
    if out is not None:
        raise ValueError("a result written to out carries no gradient, and an operand requires one")
    return True


@_with_stream
def clip_grads(grads, max_norm, out=None, workspace=None):
    """Scale the tensors of ``grads`` (contiguous, float32 or bfloat16 each) so that
    the norm over all of them is at most ``max_norm``: in place, or into the
    tensors of ``out``.  Returns a float32 tensor [norm before, coefficient] on the
    device.  An infinite or NaN norm leaves them as they are.  No tensor may be given
    twice (a tied gradient counts once) or overlap another one's result."""
    grads = list(grads)
    if not grads:
        raise ValueError("no gradients")
    index = _place(grads[0])
    types = [_DTYPE.get(g.dtype, -1) for g in grads]
    if -1 in types:
        raise ValueError("gradients must be float32 or bfloat16")
    if not all([g.is_contiguous() and g.get_device() == index for g in grads]):
        raise ValueError("gradients must be contiguous and on one device")
    src = [g.data_ptr() for g in grads]
    dst, results = src, grads
    if out is not None:
        results = out = list(out)
        if len(out) != len(grads):
            raise ValueError("out must have one tensor per gradient")
        if not all([o.shape == g.shape and o.dtype == g.dtype and o.is_contiguous() and o.get_device() == index
                    for g, o in zip(grads, out)]):
            raise ValueError("out must match the gradients and be contiguous")
        dst = [o.data_ptr() for o in out]
    device = grads[0].device
    keep, ws, ws_bytes = _workspace(workspace, isoloco_clip_workspace_size(len(grads)), device)
    norm = _empty(2, dtype=_F32, device=device)
    isoloco_clip_grads(src, dst, [g.numel() for g in grads], types, max_norm, norm.data_ptr(), ws, ws_bytes,
                       _raw_stream(index))
    _written(results)
    return norm


@_with_stream
def embedding(table, ids, scale=1.0, out=None, out_dtype=None):
    """``scale * table[ids]`` in ``out_dtype`` (default: the table's); ids outside the
    table give rows of zeros."""
    if table.requires_grad and _recorded(out):
        return _Embedding.apply(table, ids, scale, out_dtype)
    if table.dim() != 2:
        raise ValueError("table must be a matrix")
    index = _place(table)
    _same_device(index, ids, out)
    vocab, dim = table.shape
    n = ids.numel()
    dtype, id_type, ld = _type("table", table), _ids("ids", ids, n), _rows("table", table)[1]
    if out is None:
        out = _empty(*ids.shape, dim, dtype=out_dtype or table.dtype, device=table.device)
        ld_out = dim
    else:
        _output("out", out, (*ids.shape, dim), out_dtype or out.dtype)
        ld_out = _rows("out", out)[1]
        _written(out)
    _check(_lib.isoloco_embedding(table.data_ptr(), ld, dtype, vocab, dim, ids.data_ptr(), id_type, n, scale,
                                  out.data_ptr(), ld_out, _type("out", out), _raw_stream(index)),
           "isoloco_embedding")
    return out


@_with_stream
def embedding_backward(ids, dout, vocab, scale=1.0, out=None, accumulate=False, out_dtype=None, workspace=None):
    """The table's gradient [vocab, dim] from ``dout`` (ids' shape + [dim]), in
    ``out_dtype`` (default float32).  ``accumulate`` adds it to ``out``."""
    if accumulate and out is None:
        raise ValueError("accumulate needs out")
    if dout.shape[:-1] != ids.shape:
        raise ValueError("dout must have the shape of ids and one more dimension")
    index = _place(dout)
    _same_device(index, ids, out)
    dim = dout.shape[-1]
    n, ld = _rows("dout", dout)
    dtype, id_type = _type("dout", dout), _ids("ids", ids, n)
    if out is None:
        out = _empty(vocab, dim, dtype=out_dtype or _F32, device=dout.device)
        ld_out = dim
    else:
        _output("out", out, (vocab, dim), out_dtype or out.dtype)
        ld_out = _rows("out", out)[1]
        _written(out)
    keep, ws, ws_bytes = _workspace(workspace, isoloco_embedding_backward_workspace_size(n, vocab, dim), dout.device)
    _check(_lib.isoloco_embedding_backward(ids.data_ptr(), id_type, n, dout.data_ptr(), ld, dtype, vocab, dim, scale, 1
                                           if accumulate else 0, out.data_ptr(), ld_out, _type("out", out), ws,
                                           ws_bytes, _raw_stream(index)),
           "isoloco_embedding_backward")
    return out


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, ids, scale, out_dtype):
        ctx.save_for_backward(ids)
        ctx.vocab, ctx.scale, ctx.dtype = table.shape[0], scale, table.dtype
        return embedding(table, ids, scale, out_dtype=out_dtype)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        ids, = ctx.saved_tensors
        return embedding_backward(ids, dout.contiguous(), ctx.vocab, ctx.scale, out_dtype=ctx.dtype), None, None, None


class TokenLogProbs(NamedTuple):
    """What ``token_logprobs`` returns, with the logits' leading shape; the last two
    have one more dimension of ``top_k`` and are None without it.  ``logprob`` and
    ``entropy`` hand gradients back."""
    logprob: Optional[torch.Tensor]
    entropy: torch.Tensor
    lse: torch.Tensor
    top_logprob: Optional[torch.Tensor]
    top_index: Optional[torch.Tensor]


@_with_stream
def token_logprobs(logits, targets=None, scale=1.0, top_k=0, workspace=None):
    """Log probabilities of ``targets`` under softmax(scale * logits) over the last
    dimension, with the rows' entropy and log-sum-exp and the ``top_k`` most likely
    tokens (int64, of equal ones the lower index first).  Targets outside the
    vocabulary are ignored (0)."""
    if logits.requires_grad and _recorded(None):
        return TokenLogProbs(*_TokenLogProbs.apply(logits, targets, scale, top_k, workspace))
    index = _place(logits)
    dtype = _type("logits", logits)
    rows, ld = _rows("logits", logits)
    shape, vocab, device = logits.shape[:-1], logits.shape[-1], logits.device
    logprob = target_at = logprob_at = top = top_index = top_at = index_at = None
    t_type = 0
    if targets is not None:
        _same_device(index, targets)
        t_type = _ids("targets", targets, rows)
        entropy, lse, logprob = _empty(3, *shape, dtype=_F32, device=device).unbind()
        target_at, logprob_at = targets.data_ptr(), logprob.data_ptr()
    else:
        entropy, lse = _empty(2, *shape, dtype=_F32, device=device).unbind()
    ws_need = isoloco_token_logprobs_workspace_size(rows, vocab, top_k)
    if top_k:
        top = _empty(*shape, top_k, dtype=_F32, device=device)
        top_index = _empty(*shape, top_k, dtype=torch.int64, device=device)
        top_at, index_at = top.data_ptr(), top_index.data_ptr()
    keep, ws, ws_bytes = _workspace(workspace, ws_need, device)
    _check(_lib.isoloco_token_logprobs(logits.data_ptr(), ld, dtype, rows, vocab, target_at, t_type, scale, top_k,
                                       logprob_at, entropy.data_ptr(), lse.data_ptr(), top_at, index_at, ws, ws_bytes,
                                       _raw_stream(index)),
           "isoloco_token_logprobs")
    return TokenLogProbs(logprob, entropy, lse, top, top_index)


@_with_stream
def token_logprobs_backward(logits, targets, lse, dlogprob, entropy=None, dentropy=None, scale=1.0, out=None):
    """The gradient in the logits from that of ``token_logprobs``' logprob (and
    entropy), given its lse (and entropy).  ``targets`` and ``dlogprob`` may both be
    None; ``out`` may be ``logits`` itself."""
    if (targets is None) != (dlogprob is None):
        raise ValueError("targets and dlogprob go together")
    if dentropy is not None and entropy is None:
        raise ValueError("dentropy needs entropy")
    index = _place(logits)
    _same_device(index, targets, lse, dlogprob, entropy, dentropy, out)
    dtype = _type("logits", logits)
    rows, ld = _rows("logits", logits)
    vocab = logits.shape[-1]
    target_at = dlogprob_at = entropy_at = dentropy_at = None
    t_type = 0
    if targets is not None:
        t_type = _ids("targets", targets, rows)
        target_at, dlogprob_at = targets.data_ptr(), _vector("dlogprob", dlogprob, rows)
    if dentropy is not None:
        entropy_at, dentropy_at = _vector("entropy", entropy, rows), _vector("dentropy", dentropy, rows)
    if out is None:
        out = _empty(*logits.shape, dtype=logits.dtype, device=logits.device)
        ld_out = vocab
    else:
        _output("out", out, logits.shape, logits.dtype)
        ld_out = _rows("out", out)[1]
        _written(out)
    _check(_lib.isoloco_token_logprobs_backward(logits.data_ptr(), ld, dtype, rows, vocab, target_at, t_type, scale,
                                                _vector("lse", lse, rows), entropy_at, dlogprob_at, dentropy_at,
                                                out.data_ptr(), ld_out, _raw_stream(index)),
           "isoloco_token_logprobs_backward")
    return out


class _TokenLogProbs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, scale, top_k, workspace):
        # (the vectors are views of one allocation, which autograd lets nobody write: .data are none)
        logprob, entropy, lse, top, top_index = (
            None if t is None else t.data for t in token_logprobs(logits, targets, scale, top_k, workspace))
        ctx.save_for_backward(logits, targets, lse, entropy)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        if top_k:
            ctx.mark_non_differentiable(top_index)
        return logprob, entropy, lse, top, top_index

    @staticmethod
    @once_differentiable
    def backward(ctx, dlogprob, dentropy, dlse, dtop, _):
        if dlse is not None or dtop is not None:
            raise NotImplementedError("lse and top_logprob have no gradient: detach them")
        logits, targets, lse, entropy = ctx.saved_tensors
        if dlogprob is None:
            targets = None
        else:
            dlogprob = dlogprob.contiguous()
        if dentropy is not None:
            dentropy = dentropy.contiguous()
        d = token_logprobs_backward(logits, targets, lse, dlogprob, entropy, dentropy, ctx.scale)
        return d, None, None, None, None


def _ffn_operands(x, w_gate, w_up, act):
    index = _place(x)
    _same_device(index, w_gate, w_up)
    dtype = _type("x", x)
    if w_gate.dim() != 2 or w_gate.shape != w_up.shape or w_gate.dtype != x.dtype or w_up.dtype != x.dtype:
        raise ValueError("w_gate and w_up must be [hidden, dim] matrices of x's type")
    hidden, dim = w_gate.shape
    if not x.dim() or x.shape[-1] != dim:
        raise ValueError("x must end in a dimension of %d, not %s" % (dim, tuple(x.shape)))
    tokens, ld_x = _rows("x", x)
    ld_w = _rows("w_gate", w_gate)[1]
    if ld_w != _rows("w_up", w_up)[1]:
        raise ValueError("w_gate and w_up must have the same row stride")
    a = _ACT.get(act)
    if a is None:
        raise ValueError("act must be one of %s" % ", ".join(sorted(_ACT)))
    at = x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr()
    aligned = not ((ld_x | ld_w) & 7 or (at[0] | at[1] | at[2]) & 15) and ld_x <= _FFN_LD and ld_w <= _FFN_LD
    return index, dtype, tokens, dim, hidden, ld_x, ld_w, a, at, ISOLOCO_FFN_ALIGNED if aligned else 0


@_with_stream
def gated_ffn(x, w_gate, w_up, act="silu", out=None, workspace=None):
    """``act(x w_gate^T) * (x w_up^T)`` for x [..., dim] and weights [hidden, dim]; act
    is "silu" or "gelu"."""
    if (x.requires_grad or w_gate.requires_grad or w_up.requires_grad) and _recorded(out):
        return _GatedFfn.apply(x, w_gate, w_up, act, workspace)
    index, dtype, tokens, dim, hidden, ld_x, ld_w, a, at, flags = _ffn_operands(x, w_gate, w_up, act)
    if out is None:
        out = _empty(*x.shape[:-1], hidden, dtype=x.dtype, device=x.device)
        ld_out = hidden
    else:
        _same_device(index, out)
        _output("out", out, (*x.shape[:-1], hidden), x.dtype)
        ld_out = _rows("out", out)[1]
        _written(out)
    keep, ws, ws_bytes = _workspace(workspace, isoloco_gated_ffn_workspace_size(tokens, dim, hidden, dtype, flags),
                                    x.device)
    _check(_lib.isoloco_gated_ffn(at[0], ld_x, at[1], at[2], ld_w, dtype, tokens, dim, hidden, a, out.data_ptr(),
                                  ld_out, ws, ws_bytes, _raw_stream(index)),
           "isoloco_gated_ffn")
    return out


@_with_stream
def gated_ffn_backward(x, w_gate, w_up, dout, act="silu", need_dx=True, need_dw=True, workspace=None):
    """(dx, dw_gate, dw_up) from ``dout`` [..., hidden]; None for what is not needed."""
    index, dtype, tokens, dim, hidden, ld_x, ld_w, a, at, flags = _ffn_operands(x, w_gate, w_up, act)
    _same_device(index, dout)
    if dout.dtype != x.dtype or tuple(dout.shape) != (*x.shape[:-1], hidden):
        raise ValueError("dout must be %s of %s" % (x.dtype, (*x.shape[:-1], hidden)))
    ld_dout, device = _rows("dout", dout)[1], x.device
    dx = dwg = dwu = dx_at = dwg_at = dwu_at = None
    if need_dx:
        dx = _empty(*x.shape, dtype=x.dtype, device=device)
        dx_at = dx.data_ptr()
    if need_dw:
        dwg = _empty(hidden, dim, dtype=x.dtype, device=device)
        dwu = _empty(hidden, dim, dtype=x.dtype, device=device)
        dwg_at, dwu_at = dwg.data_ptr(), dwu.data_ptr()
    keep, ws, ws_bytes = _workspace(workspace, isoloco_gated_ffn_workspace_size(
        tokens, dim, hidden, dtype, flags | ISOLOCO_FFN_BACKWARD), device)
    _check(_lib.isoloco_gated_ffn_backward(at[0], ld_x, at[1], at[2], ld_w, dtype, tokens, dim, hidden, a,
                                           dout.data_ptr(), ld_dout, dx_at, dim, dwg_at, dwu_at, dim, ws, ws_bytes,
                                           _raw_stream(index)),
           "isoloco_gated_ffn_backward")
    return dx, dwg, dwu


class _GatedFfn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_gate, w_up, act, workspace):
        ctx.save_for_backward(x, w_gate, w_up)
        ctx.act = act
        return gated_ffn(x, w_gate, w_up, act, workspace=workspace)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        need_x, need_gate, need_up = ctx.needs_input_grad[:3]
        dx, dwg, dwu = gated_ffn_backward(*ctx.saved_tensors, dout.contiguous(), ctx.act, need_x, need_gate or need_up)
        return dx, dwg if need_gate else None, dwu if need_up else None, None, None

"""Operators of the workers' inner training step on torch tensors.

The functions named ``isoloco_*`` have the name and the argument order of the C
functions they marshal (``include/isoloco.h``) and take addresses.  The others
take tensors: they check shapes, types and strides (``ValueError``), allocate
what is not given with torch's allocator, and enqueue on the current torch
stream of the tensors' device (or ``stream``, a raw stream handle).  Matrices
need unit stride along a row; a further leading dimension is allowed where the
rows stay evenly spaced.  Arguments that the library itself refuses raise
``IsoLoCoError``.
"""
import array
import ctypes
from typing import NamedTuple, Optional

import torch

from . import (ISOLOCO_ACT_GELU, ISOLOCO_ACT_SILU, ISOLOCO_BF16, ISOLOCO_F32, ISOLOCO_FFN_ALIGNED,
               ISOLOCO_FFN_BACKWARD, ISOLOCO_I32, ISOLOCO_I64, _check, _lib)

_DTYPE = {torch.float32: ISOLOCO_F32, torch.bfloat16: ISOLOCO_BF16}
_INDEX = {torch.int32: ISOLOCO_I32, torch.int64: ISOLOCO_I64}
_ACT = {"silu": ISOLOCO_ACT_SILU, "gelu": ISOLOCO_ACT_GELU}


# --------------------------------------------------------------------------
# The C functions
# --------------------------------------------------------------------------

def _size_of(name, *args):
    n = ctypes.c_size_t()
    _check(getattr(_lib, name)(*args, ctypes.byref(n)), name)
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

class _On:
    """The device and stream of a call: memory allocated inside belongs to that stream."""

    def __init__(self, t, stream):
        if not t.is_cuda:
            raise ValueError("tensors must be on the GPU")
        self.device = t.device
        self.handle = stream
        self.contexts = []

    def __enter__(self):
        if self.device.index != torch.cuda.current_device():
            self.contexts.append(torch.cuda.device(self.device))
            self.contexts[-1].__enter__()
        if self.handle is None:
            self.handle = torch.cuda.current_stream(self.device).cuda_stream
        else:
            self.contexts.append(torch.cuda.stream(torch.cuda.ExternalStream(self.handle, self.device)))
            self.contexts[-1].__enter__()
        return self

    def __exit__(self, *exc):
        while self.contexts:
            self.contexts.pop().__exit__(*exc)

    def empty(self, shape, dtype):
        return torch.empty(shape, dtype=dtype, device=self.device)

    def workspace(self, given, need):
        """(address, bytes) of `given` (a uint8 tensor) or of a new one, aligned to 256 bytes."""
        if need == 0:
            return None, 0, None
        t = torch.empty(need + 255, dtype=torch.uint8, device=self.device) if given is None else given
        if t.dtype != torch.uint8 or not t.is_contiguous() or t.device != self.device:
            raise ValueError("workspace must be a contiguous uint8 tensor on the operands' device")
        base = t.data_ptr()
        at = (base + 255) // 256 * 256
        return at, max(0, base + t.numel() - at), t


def _type(name, t):
    d = _DTYPE.get(t.dtype)
    if d is None:
        raise ValueError("%s must be float32 or bfloat16, not %s" % (name, t.dtype))
    return d


def _rows(name, t, cols=None):
    """(rows, ld) of a tensor seen as a matrix of its last dimension's rows."""
    if t.dim() == 0 or (cols is not None and t.shape[-1] != cols):
        raise ValueError("%s must end in a dimension of %s, not %s" % (name, cols, tuple(t.shape)))
    c = t.shape[-1]
    n = t.numel() // c if c else 0
    if t.is_contiguous():
        return n, c
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


def _same_device(on, **tensors):
    for name, t in tensors.items():
        if t is not None and t.device != on.device:
            raise ValueError("%s is on %s, not on %s" % (name, t.device, on.device))


def _ids(name, t, n=None):
    i = _INDEX.get(t.dtype)
    if i is None:
        raise ValueError("%s must be int32 or int64, not %s" % (name, t.dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if n is not None and t.numel() != n:
        raise ValueError("%s must have %d elements, not %d" % (name, n, t.numel()))
    return i


def _vector(name, t, n):
    if t.dtype != torch.float32 or not t.is_contiguous() or t.numel() != n:
        raise ValueError("%s must be contiguous float32 of %d elements" % (name, n))
    return t.data_ptr()


def _output(on, name, t, shape, dtype):
    """A new tensor, or the given one if it has the shape and type."""
    if t is None:
        return on.empty(shape, dtype)
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype:
        raise ValueError("%s must be %s of %s" % (name, dtype, tuple(shape)))
    return t


def clip_grads(grads, max_norm, out=None, workspace=None, stream=None):
    """Scale the tensors of ``grads`` (contiguous, float32 or bfloat16 each) so that
    the norm over all of them is at most ``max_norm``: in place, or into the
    tensors of ``out``.  Returns a float32 tensor [norm before, coefficient] on the
    device.  An infinite or NaN norm leaves them as they are."""
    grads = list(grads)
    if not grads:
        raise ValueError("no gradients")
    if out is not None:
        out = list(out)
        if len(out) != len(grads):
            raise ValueError("out must have one tensor per gradient")
    with _On(grads[0], stream) as on:
        device = on.device
        for g in grads:
            if not g.is_contiguous() or g.device != device:
                raise ValueError("gradients must be contiguous and on one device")
        if out is not None:
            for g, o in zip(grads, out):
                if o.shape != g.shape or o.dtype != g.dtype or not o.is_contiguous() or o.device != device:
                    raise ValueError("out must match the gradients and be contiguous")
        types = [_type("a gradient", g) for g in grads]
        src = [g.data_ptr() for g in grads]
        ws, ws_bytes, keep = on.workspace(workspace, isoloco_clip_workspace_size(len(grads)))
        norm = on.empty(2, torch.float32)
        isoloco_clip_grads(src, src if out is None else [o.data_ptr() for o in out], [g.numel() for g in grads], types,
                           max_norm, norm.data_ptr(), ws, ws_bytes, on.handle)
        return norm


def embedding(table, ids, scale=1.0, out=None, out_dtype=None, stream=None):
    """``scale * table[ids]`` in ``out_dtype`` (default: the table's); ids outside the
    table give rows of zeros."""
    if table.dim() != 2:
        raise ValueError("table must be a matrix")
    with _On(table, stream) as on:
        _same_device(on, ids=ids, out=out)
        vocab, dim = table.shape
        dtype, id_type = _type("table", table), _ids("ids", ids)
        _, ld = _rows("table", table)
        out = _output(on, "out", out, (*ids.shape, dim), out_dtype or (table.dtype if out is None else out.dtype))
        n, ld_out = _rows("out", out)
        isoloco_embedding(table.data_ptr(), ld, dtype, vocab, dim, ids.data_ptr(), id_type, ids.numel(), scale,
                          out.data_ptr(), ld_out, _type("out", out), on.handle)
        return out


def embedding_backward(ids, dout, vocab, scale=1.0, out=None, accumulate=False, out_dtype=None, workspace=None,
                       stream=None):
    """The table's gradient [vocab, dim] from ``dout`` (ids' shape + [dim]), in
    ``out_dtype`` (default float32).  ``accumulate`` adds it to ``out``."""
    if accumulate and out is None:
        raise ValueError("accumulate needs out")
    if tuple(dout.shape[:-1]) != tuple(ids.shape):
        raise ValueError("dout must have the shape of ids and one more dimension")
    with _On(dout, stream) as on:
        _same_device(on, ids=ids, out=out)
        dtype, id_type = _type("dout", dout), _ids("ids", ids)
        dim = dout.shape[-1]
        n, ld = _rows("dout", dout)
        out = _output(on, "out", out, (vocab, dim), out_dtype or (torch.float32 if out is None else out.dtype))
        _, ld_out = _rows("out", out)
        ws, ws_bytes, keep = on.workspace(workspace, isoloco_embedding_backward_workspace_size(n, vocab, dim))
        isoloco_embedding_backward(ids.data_ptr(), id_type, n, dout.data_ptr(), ld, dtype, vocab, dim, scale,
                                   1 if accumulate else 0, out.data_ptr(), ld_out, _type("out", out), ws, ws_bytes,
                                   on.handle)
        return out


class TokenLogProbs(NamedTuple):
    """What ``token_logprobs`` returns, with the logits' leading shape; the last two
    have one more dimension of ``top_k`` and are None without it."""
    logprob: Optional[torch.Tensor]
    entropy: torch.Tensor
    lse: torch.Tensor
    top_logprob: Optional[torch.Tensor]
    top_index: Optional[torch.Tensor]


def token_logprobs(logits, targets=None, scale=1.0, top_k=0, workspace=None, stream=None):
    """Log probabilities of ``targets`` under softmax(scale * logits) over the last
    dimension, with the rows' entropy and log-sum-exp and the ``top_k`` most likely
    tokens (int64, of equal ones the lower index first).  Targets outside the
    vocabulary are ignored (0)."""
    with _On(logits, stream) as on:
        _same_device(on, targets=targets)
        dtype = _type("logits", logits)
        vocab = logits.shape[-1] if logits.dim() else 0
        rows, ld = _rows("logits", logits)
        shape = tuple(logits.shape[:-1])
        t_type = _ids("targets", targets, rows) if targets is not None else 0
        logprob = on.empty(shape, torch.float32) if targets is not None else None
        entropy, lse = on.empty(shape, torch.float32), on.empty(shape, torch.float32)
        top = on.empty((*shape, top_k), torch.float32) if top_k else None
        index = on.empty((*shape, top_k), torch.int64) if top_k else None
        ws, ws_bytes, keep = on.workspace(workspace, isoloco_token_logprobs_workspace_size(rows, vocab, top_k))
        isoloco_token_logprobs(logits.data_ptr(), ld, dtype, rows, vocab,
                               targets.data_ptr() if targets is not None else None, t_type, scale, top_k,
                               logprob.data_ptr() if targets is not None else None, entropy.data_ptr(),
                               lse.data_ptr(), top.data_ptr() if top_k else None, index.data_ptr() if top_k else None,
                               ws, ws_bytes, on.handle)
        return TokenLogProbs(logprob, entropy, lse, top, index)


def token_logprobs_backward(logits, targets, lse, dlogprob, entropy=None, dentropy=None, scale=1.0, out=None,
                            stream=None):
    """The gradient in the logits from that of ``token_logprobs``' logprob (and
    entropy), given its lse (and entropy).  ``targets`` and ``dlogprob`` may both be
    None; ``out`` may be ``logits`` itself."""
    if (targets is None) != (dlogprob is None):
        raise ValueError("targets and dlogprob go together")
    if dentropy is not None and entropy is None:
        raise ValueError("dentropy needs entropy")
    with _On(logits, stream) as on:
        _same_device(on, targets=targets, lse=lse, dlogprob=dlogprob, entropy=entropy, dentropy=dentropy, out=out)
        dtype = _type("logits", logits)
        vocab = logits.shape[-1] if logits.dim() else 0
        rows, ld = _rows("logits", logits)
        t_type = _ids("targets", targets, rows) if targets is not None else 0
        out = _output(on, "out", out, tuple(logits.shape), logits.dtype)
        _, ld_out = _rows("out", out)
        isoloco_token_logprobs_backward(
            logits.data_ptr(), ld, dtype, rows, vocab, targets.data_ptr() if targets is not None else None, t_type,
            scale, _vector("lse", lse, rows), _vector("entropy", entropy, rows) if dentropy is not None else None,
            _vector("dlogprob", dlogprob, rows) if dlogprob is not None else None,
            _vector("dentropy", dentropy, rows) if dentropy is not None else None, out.data_ptr(), ld_out, on.handle)
        return out


def _ffn_operands(on, x, w_gate, w_up, act):
    dtype = _type("x", x)
    if w_gate.dim() != 2 or w_gate.shape != w_up.shape or w_gate.dtype != x.dtype or w_up.dtype != x.dtype:
        raise ValueError("w_gate and w_up must be [hidden, dim] matrices of x's type")
    _same_device(on, w_gate=w_gate, w_up=w_up)
    hidden, dim = w_gate.shape
    tokens, ld_x = _rows("x", x, dim)
    ld_w, ld_u = _rows("w_gate", w_gate)[1], _rows("w_up", w_up)[1]
    if ld_w != ld_u:
        raise ValueError("w_gate and w_up must have the same row stride")
    if act not in _ACT:
        raise ValueError("act must be one of %s" % ", ".join(sorted(_ACT)))
    aligned = (ld_x | ld_w) % 8 == 0 and (x.data_ptr() | w_gate.data_ptr() | w_up.data_ptr()) % 16 == 0
    return dtype, tokens, dim, hidden, ld_x, ld_w, _ACT[act], ISOLOCO_FFN_ALIGNED if aligned else 0


def gated_ffn(x, w_gate, w_up, act="silu", out=None, workspace=None, stream=None):
    """``act(x w_gate^T) * (x w_up^T)`` for x [..., dim] and weights [hidden, dim]; act
    is "silu" or "gelu"."""
    with _On(x, stream) as on:
        dtype, tokens, dim, hidden, ld_x, ld_w, a, flags = _ffn_operands(on, x, w_gate, w_up, act)
        _same_device(on, out=out)
        out = _output(on, "out", out, (*x.shape[:-1], hidden), x.dtype)
        _, ld_out = _rows("out", out)
        ws, ws_bytes, keep = on.workspace(workspace, isoloco_gated_ffn_workspace_size(tokens, dim, hidden, dtype,
                                                                                               flags))
        isoloco_gated_ffn(x.data_ptr(), ld_x, w_gate.data_ptr(), w_up.data_ptr(), ld_w, dtype, tokens, dim, hidden, a,
                          out.data_ptr(), ld_out, ws, ws_bytes, on.handle)
        return out


def gated_ffn_backward(x, w_gate, w_up, dout, act="silu", need_dx=True, need_dw=True, workspace=None, stream=None):
    """(dx, dw_gate, dw_up) from ``dout`` [..., hidden]; None for what is not needed."""
    with _On(x, stream) as on:
        dtype, tokens, dim, hidden, ld_x, ld_w, a, flags = _ffn_operands(on, x, w_gate, w_up, act)
        _same_device(on, dout=dout)
        if dout.dtype != x.dtype or tuple(dout.shape) != (*x.shape[:-1], hidden):
            raise ValueError("dout must be %s of %s" % (x.dtype, (*x.shape[:-1], hidden)))
        _, ld_dout = _rows("dout", dout, hidden)
        dx = on.empty(x.shape, x.dtype) if need_dx else None
        dwg = on.empty((hidden, dim), x.dtype) if need_dw else None
        dwu = on.empty((hidden, dim), x.dtype) if need_dw else None
        ws, ws_bytes, keep = on.workspace(workspace, isoloco_gated_ffn_workspace_size(
            tokens, dim, hidden, dtype, flags | ISOLOCO_FFN_BACKWARD))
        isoloco_gated_ffn_backward(x.data_ptr(), ld_x, w_gate.data_ptr(), w_up.data_ptr(), ld_w, dtype, tokens, dim,
                                   hidden, a, dout.data_ptr(), ld_dout, dx.data_ptr() if need_dx else None, dim,
                                   dwg.data_ptr() if need_dw else None, dwu.data_ptr() if need_dw else None, dim, ws,
                                   ws_bytes, on.handle)
        return dx, dwg, dwu

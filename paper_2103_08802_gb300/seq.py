"""Token-sequence operators of libpnn.so on torch CUDA tensors.

embed, embed_grad        embedding lookup with scaling, its gradient by sorted tokens
recur, recur_grad        gated linear recurrence along time and its backward pass
recur_step               one token of it on a pool of states
distill                  loss and gradient of learning from a teacher's top logits

The formulas and the rules for empty and masked rows stand in include/pnn.h.
As in `pnn`, every step runs in the library's kernels; this module checks and
marshals arguments, and takes outputs and workspaces from torch.  Calls return
at once.  They run on `stream` (a torch.cuda.Stream) or, without one, on
torch's current stream; tensors made or last used on another stream are the
caller's to order (Stream.wait_stream), outputs belong to the stream of the
call.  Wrong arguments raise TypeError (types, shapes, devices) or PnnError.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import pnn
from .pnn import DistillArgs, EmbedArgs, RecurArgs, RecurStepArgs, _global_check, load

__all__ = ["sync", "embed", "embed_grad", "recur", "recur_grad", "recur_step", "distill"]

_DT = {torch.float32: pnn.DTYPE["f32"], torch.bfloat16: pnn.DTYPE["bf16"]}
_IDS = {torch.int32: 32, torch.int64: 64}


def _value(t, name, dims, dev, shape=None):
    """Checks for a float32 / bfloat16 tensor of CUDA device dev whose last axis is contiguous."""
    if (isinstance(t, torch.Tensor) and t.get_device() == dev and t.dtype in _DT and t.dim() == dims
            and (t.stride(-1) == 1 or t.shape[-1] <= 1 or t.numel() == 0) and (shape is None or t.shape == shape)):
        return
    raise TypeError(f"{name} must be a float32 or bfloat16 tensor of the current CUDA device, {dims}-dimensional with a "
                    f"contiguous last axis" + (f", of shape {tuple(shape)}" if shape is not None else ""))


def _flat(t, name, dtype, dev, shape):
    """The address of a contiguous tensor of one type and shape on CUDA device dev; None for None."""
    if t is None:
        return None
    if isinstance(t, torch.Tensor) and t.get_device() == dev and t.dtype == dtype and t.is_contiguous() and t.shape == shape:
        return t.data_ptr()
    raise TypeError(f"{name} must be a contiguous {dtype} tensor of the current CUDA device, of shape {tuple(shape)}")


def _ids(ids, dev):
    if isinstance(ids, torch.Tensor) and ids.get_device() == dev and ids.dtype in _IDS and ids.is_contiguous():
        return ids.data_ptr(), _IDS[ids.dtype]
    raise TypeError("ids must be a contiguous int32 or int64 tensor of the current CUDA device")


def _here(stream):
    """The current device, and the handle of the call's stream."""
    dev = torch.cuda.current_device()
    return dev, torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


def _new(shape, dtype, device, stream):
    """An output or workspace from the pool of the call's stream."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _matrix(t, n, stream):
    """t as n rows: a view, or a copy that the call's stream makes and owns."""
    if stream is None:
        return t.reshape(n, t.shape[-1])
    with torch.cuda.stream(stream):
        return t.reshape(n, t.shape[-1])


def _row_stride(t):
    """The row stride of a matrix (of one row: any that does not overlap)."""
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def sync(stream=None):
    """Waits for the stream; raises PnnError if a bounded device-side wait gave up, on any stream of the device, since
    this stream's last call."""
    lib = load()
    _global_check(lib, lib.pnn_seq_sync(_here(stream)[1]))


def embed(ids, table, scale=1.0, out=None, dtype=None, stream=None):
    """scale * table[ids]: ids of any shape, table vocab x width; a zero row
    where an id lies outside the table.  dtype: of the result (the table's)."""
    dev, st = _here(stream)
    p, bits = _ids(ids, dev)
    _value(table, "table", 2, dev)
    lib = load()
    n, (v, d) = ids.numel(), table.shape
    if out is None:
        out = _new((*ids.shape, d), dtype or table.dtype, table.device, stream)
        stride = d
    else:
        _value(out, "out", 2, dev, (n, d))
        stride = _row_stride(out)
    a = EmbedArgs(n, v, d, p, bits, scale, table.data_ptr(), _DT[table.dtype], table.stride(0),
                  out.data_ptr(), _DT.get(out.dtype, -1), stride)
    rc = lib.pnn_embed_forward(C.byref(a), st)
    if rc:
        _global_check(lib, rc)
    return out


def embed_grad(ids, dout, vocab=None, scale=1.0, dtable=None, accumulate=False, dtype=torch.float32, stream=None):
    """Gradient of embed with respect to its table.  dout: ids.shape x width.
    Without dtable a new vocab x width tensor of `dtype` is written whole; with
    dtable, that tensor is (accumulate: added to, only rows that occur)."""
    dev, st = _here(stream)
    p, bits = _ids(ids, dev)
    n = ids.numel()
    if not isinstance(dout, torch.Tensor) or dout.dim() < 1 or (dout.dim() != 2 and dout.shape[:-1] != ids.shape):
        raise TypeError("dout must have shape ids.shape x width")
    if dout.dim() != 2:
        dout = _matrix(dout, n, stream)
    d = dout.shape[-1]
    _value(dout, "dout", 2, dev, (n, d))
    if dtable is None:
        if vocab is None or accumulate:
            raise TypeError("embed_grad needs vocab, or dtable to add to")
        dtable = _new((vocab, d), dtype, dout.device, stream)
    else:
        _value(dtable, "dtable", 2, dev, (dtable.shape[0] if vocab is None else vocab, d))
    lib = load()
    a = EmbedArgs(n, dtable.shape[0], d, p, bits, scale, None, 0, 0, None, 0, 0, dout.data_ptr(), _DT[dout.dtype], _row_stride(dout),
                  dtable.data_ptr(), _DT.get(dtable.dtype, -1), _row_stride(dtable), int(accumulate))
    nb = C.c_size_t()
    rc = lib.pnn_embed_workspace_bytes(C.byref(a), C.byref(nb))
    if rc:
        _global_check(lib, rc)
    ws = _new((max(256, nb.value),), torch.uint8, dout.device, stream)
    rc = lib.pnn_embed_backward(C.byref(a), ws.data_ptr(), nb.value, st)
    if rc:
        _global_check(lib, rc)
    return dtable


def _recur_args(z, x, lengths, h0, dev):
    _value(z, "z", 3, dev)
    _value(x, "x", 3, dev)
    (b, t, h), d = z.shape, x.shape[-1]
    if x.shape[:2] != z.shape[:2] or x.dtype != z.dtype or h <= 0 or d % h:
        raise TypeError("x must be batch x time x channels of z's type, its channels a multiple of z's heads")
    return RecurArgs(b, t, h, d // h, _DT[z.dtype], z.data_ptr(), z.stride(0), z.stride(1),
                     x.data_ptr(), x.stride(0), x.stride(1), _flat(lengths, "lengths", torch.int32, dev, (b,)),
                     _flat(h0, "h0", torch.float32, dev, (b, d)))


def _recur_workspace(lib, a, backward, device, stream):
    n = C.c_size_t()
    rc = lib.pnn_recur_workspace_bytes(C.byref(a), backward, C.byref(n))
    if rc:
        _global_check(lib, rc)
    return (_new((n.value,), torch.uint8, device, stream) if n.value else None), n.value


def _saved_size(lib, a):
    n = C.c_size_t()
    rc = lib.pnn_recur_saved_size(C.byref(a), C.byref(n))
    if rc:
        _global_check(lib, rc)
    return n.value


def recur(z, x, h0=None, lengths=None, save=False, h=None, stream=None):
    """h_t = f_t h_{t-1} + (1 - f_t) x_t with f = sigmoid(z).  z: batch x time
    x heads, x: batch x time x channels (strided rows are fine), h0: fp32
    batch x channels, lengths: int32.  Returns (h, h_last), with save=True also
    what recur_grad needs."""
    dev, st = _here(stream)
    a = _recur_args(z, x, lengths, h0, dev)
    lib = load()
    b, t, d = x.shape
    if h is None:
        h = _new((b, t, d), x.dtype, x.device, stream)
        a.h, a.h_stride_b, a.h_stride_t = h.data_ptr(), t * d, d
    else:
        _value(h, "h", 3, dev, x.shape)
        if h.dtype != x.dtype:
            raise TypeError("h must have x's type")
        a.h, a.h_stride_b, a.h_stride_t = h.data_ptr(), h.stride(0), h.stride(1)
    last = _new((b, d), torch.float32, x.device, stream)
    a.h_last = last.data_ptr()
    if save:
        saved = _new((_saved_size(lib, a),), torch.float32, x.device, stream)
        a.saved = saved.data_ptr()
    ws, n = _recur_workspace(lib, a, 0, x.device, stream)
    rc = lib.pnn_recur_forward(C.byref(a), None if ws is None else ws.data_ptr(), n, st)
    if rc:
        _global_check(lib, rc)
    return (h, last, saved) if save else (h, last)


def recur_grad(z, x, saved, dh, dh_last=None, lengths=None, stream=None):
    """Backward of recur: (dz, dx, dh0) from dh (batch x time x channels, x's
    type) and dh_last (fp32 batch x channels or None).  z, x and lengths as in
    the forward that returned `saved`."""
    dev, st = _here(stream)
    a = _recur_args(z, x, lengths, None, dev)
    lib = load()
    b, t, d = x.shape
    _value(dh, "dh", 3, dev, x.shape)
    if dh.dtype != x.dtype:
        raise TypeError("dh must have x's type")
    a.dh, a.dh_stride_b, a.dh_stride_t = dh.data_ptr(), dh.stride(0), dh.stride(1)
    a.dh_last = _flat(dh_last, "dh_last", torch.float32, dev, (b, d))
    a.saved = _flat(saved, "saved", torch.float32, dev, (_saved_size(lib, a),))
    h = z.shape[2]
    dz = _new((b, t, h), x.dtype, x.device, stream)
    dx = _new((b, t, d), x.dtype, x.device, stream)
    dh0 = _new((b, d), torch.float32, x.device, stream)
    a.dz, a.dz_stride_b, a.dz_stride_t = dz.data_ptr(), t * h, h
    a.dx, a.dx_stride_b, a.dx_stride_t = dx.data_ptr(), t * d, d
    a.dh0 = dh0.data_ptr()
    ws, n = _recur_workspace(lib, a, 1, x.device, stream)
    rc = lib.pnn_recur_backward(C.byref(a), None if ws is None else ws.data_ptr(), n, st)
    if rc:
        _global_check(lib, rc)
    return dz, dx, dh0


def recur_step(z, x, state, slots=None, out=None, stream=None):
    """One token for each sequence of the batch: row i advances state[slots[i]]
    (fp32, slots x channels) in place and the result, rounded, is returned
    (batch x channels).  A slot outside the pool marks an empty place."""
    dev, st = _here(stream)
    _value(z, "z", 2, dev)
    _value(x, "x", 2, dev)
    _value(state, "state", 2, dev)
    (b, h), (n, d) = z.shape, state.shape
    if x.shape != (b, d) or x.dtype != z.dtype or h <= 0 or d % h or state.dtype != torch.float32:
        raise TypeError("x must be batch x channels of z's type, its channels a multiple of z's heads; state fp32 slots x channels")
    lib = load()
    if out is None:
        out = _new((b, d), x.dtype, x.device, stream)
        stride = d
    else:
        _value(out, "out", 2, dev, (b, d))
        if out.dtype != x.dtype:
            raise TypeError("out must have x's type")
        stride = out.stride(0)
    a = RecurStepArgs(b, h, d // h, n, _DT[x.dtype], z.data_ptr(), z.stride(0), x.data_ptr(), x.stride(0),
                      _flat(slots, "slots", torch.int32, dev, (b,)), state.data_ptr(), _row_stride(state), out.data_ptr(), stride)
    rc = lib.pnn_recur_step(C.byref(a), st)
    if rc:
        _global_check(lib, rc)
    return out


def distill(logits, ids, teacher, labels=None, weight=None, tau=1.0, alpha=1.0, grad=True, out=None, stream=None):
    """Per-row loss (fp32) and gradient of the logits (None with grad=False).
    logits: rows x vocab; ids (int32) and teacher: rows x k; labels (int32) and
    weight (fp32): rows.  out: the gradient's buffer, may be the logits."""
    dev, st = _here(stream)
    _value(logits, "logits", 2, dev)
    r, v = logits.shape
    lib = load()
    k, pi, pt, tt = 0, None, None, 0
    if ids is None and teacher is not None:
        raise TypeError("teacher needs ids")
    if ids is not None:
        if not isinstance(ids, torch.Tensor) or ids.dim() != 2:
            raise TypeError("ids must be a matrix, rows x k")
        k = ids.shape[-1]
        pi = _flat(ids, "ids", torch.int32, dev, (r, k))
        _value(teacher, "teacher", 2, dev, (r, k))
        pt, tt = _flat(teacher, "teacher", teacher.dtype, dev, (r, k)), _DT[teacher.dtype]
    loss = _new((r,), torch.float32, logits.device, stream)
    stride = 0
    if not grad:
        out = None
    elif out is None:
        out = _new((r, v), logits.dtype, logits.device, stream)
        stride = v
    else:
        _value(out, "out", 2, dev, (r, v))
        if out.dtype != logits.dtype:
            raise TypeError("out must have the logits' type")
        stride = out.stride(0)
    a = DistillArgs(r, v, k, _DT[logits.dtype], logits.data_ptr(), logits.stride(0), pi, pt, tt,
                    _flat(labels, "labels", torch.int32, dev, (r,)), _flat(weight, "weight", torch.float32, dev, (r,)), tau, alpha,
                    loss.data_ptr(), None if out is None else out.data_ptr(), stride)
    rc = lib.pnn_distill(C.byref(a), st)
    if rc:
        _global_check(lib, rc)
    return loss, out

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


def _need(ok, what):
    if not ok:
        raise TypeError(what)


def _value(t, name, dims, shape=None):
    """A float32 / bfloat16 CUDA tensor on the current device whose last axis is contiguous."""
    _need(isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in _DT and t.dim() == dims
          and t.get_device() == torch.cuda.current_device()
          and (t.stride(-1) == 1 or t.shape[-1] <= 1 or t.numel() == 0)
          and (shape is None or t.shape == shape),
          f"{name} must be a float32 or bfloat16 tensor of the current CUDA device, {dims}-dimensional with a "
          f"contiguous last axis" + (f", of shape {tuple(shape)}" if shape is not None else ""))
    return t


def _flat(t, name, dtype, shape):
    """A contiguous CUDA tensor of one type and shape on the current device, or None."""
    if t is None:
        return None
    _need(isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.is_contiguous() and t.shape == shape
          and t.get_device() == torch.cuda.current_device(),
          f"{name} must be a contiguous {dtype} tensor of the current CUDA device, of shape {tuple(shape)}")
    return t.data_ptr()


def _ids(ids):
    _need(isinstance(ids, torch.Tensor) and ids.is_cuda and ids.dtype in _IDS and ids.is_contiguous()
          and ids.get_device() == torch.cuda.current_device(),
          "ids must be a contiguous int32 or int64 tensor of the current CUDA device")
    return ids.data_ptr(), _IDS[ids.dtype]


class _On:
    """Within it, outputs and workspaces come from the pool of the call's
    stream, whose handle it gives."""

    def __init__(self, stream):
        self.ctx = torch.cuda.stream(stream)

    def __enter__(self):
        self.ctx.__enter__()
        return torch.cuda.current_stream().cuda_stream

    def __exit__(self, *e):
        self.ctx.__exit__(*e)


class _Here:
    """The same for torch's current stream: nothing to enter."""

    def __enter__(self):
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())

    def __exit__(self, *e):
        pass


_HERE = _Here()


def _on(stream):
    return _HERE if stream is None else _On(stream)


def sync(stream=None):
    """Waits for the stream; raises PnnError if a bounded device-side wait gave up since the last call."""
    lib = load()
    with _on(stream) as st:
        _global_check(lib, lib.pnn_seq_sync(st))


def embed(ids, table, scale=1.0, out=None, dtype=None, stream=None):
    """scale * table[ids]: ids of any shape, table vocab x width; a zero row
    where an id lies outside the table.  dtype: of the result (the table's)."""
    p, bits = _ids(ids)
    _value(table, "table", 2)
    lib = load()
    n, (v, d) = ids.numel(), table.shape
    with _on(stream) as st:
        if out is None:
            res = torch.empty((*ids.shape, d), dtype=dtype or table.dtype, device=table.device)
            out = res.view(n, d)
        else:
            res = _value(out, "out", 2, (n, d))
        a = EmbedArgs(n, v, d, p, bits, scale, table.data_ptr(), _DT[table.dtype], table.stride(0),
                      out.data_ptr(), _DT.get(out.dtype, -1), max(out.stride(0), d) if n <= 1 else out.stride(0))
        _global_check(lib, lib.pnn_embed_forward(C.byref(a), st))
    return res


def embed_grad(ids, dout, vocab=None, scale=1.0, dtable=None, accumulate=False, dtype=torch.float32, stream=None):
    """Gradient of embed with respect to its table.  dout: ids.shape x width.
    Without dtable a new vocab x width tensor of `dtype` is written whole; with
    dtable, that tensor is (accumulate: added to, only rows that occur)."""
    p, bits = _ids(ids)
    n = ids.numel()
    _need(isinstance(dout, torch.Tensor) and dout.dim() >= 1, "dout must be a tensor of shape ids.shape x width")
    if dout.dim() != 2:
        _need(dout.shape[:-1] == ids.shape, "dout must have shape ids.shape x width")
        dout = dout.reshape(n, dout.shape[-1])
    d = dout.shape[-1]
    _value(dout, "dout", 2, (n, d))
    _need(dtable is not None or (vocab is not None and not accumulate), "embed_grad needs vocab, or dtable to add to")
    lib = load()
    with _on(stream) as st:
        if dtable is None:
            dtable = torch.empty((vocab, d), dtype=dtype, device=dout.device)
        else:
            _value(dtable, "dtable", 2, (dtable.shape[0] if vocab is None else vocab, d))
        a = EmbedArgs(n, dtable.shape[0], d, p, bits, scale)
        a.dout, a.dout_dtype = dout.data_ptr(), _DT[dout.dtype]
        a.dout_stride = max(dout.stride(0), d) if n <= 1 else dout.stride(0)
        a.dtable, a.dtable_dtype, a.dtable_stride = dtable.data_ptr(), _DT.get(dtable.dtype, -1), dtable.stride(0)
        a.accumulate = int(accumulate)
        nb = C.c_size_t()
        _global_check(lib, lib.pnn_embed_workspace_bytes(C.byref(a), C.byref(nb)))
        ws = torch.empty(max(256, nb.value), dtype=torch.uint8, device=dout.device)
        _global_check(lib, lib.pnn_embed_backward(C.byref(a), ws.data_ptr(), nb.value, st))
    return dtable


def _recur_args(z, x, lengths, h0=None):
    _value(z, "z", 3)
    _value(x, "x", 3)
    (b, t, h), d = z.shape, x.shape[-1]
    _need(x.shape[:2] == (b, t) and x.dtype == z.dtype and h > 0 and d % h == 0,
          "x must be batch x time x channels of z's type, its channels a multiple of z's heads")
    return RecurArgs(b, t, h, d // h, _DT[z.dtype], z.data_ptr(), z.stride(0), z.stride(1),
                     x.data_ptr(), x.stride(0), x.stride(1), _flat(lengths, "lengths", torch.int32, (b,)),
                     _flat(h0, "h0", torch.float32, (b, d)))


def recur(z, x, h0=None, lengths=None, save=False, h=None, stream=None):
    """h_t = f_t h_{t-1} + (1 - f_t) x_t with f = sigmoid(z).  z: batch x time
    x heads, x: batch x time x channels (strided rows are fine), h0: fp32
    batch x channels, lengths: int32.  Returns (h, h_last), with save=True also
    what recur_grad needs."""
    a = _recur_args(z, x, lengths, h0)
    lib = load()
    b, t, d = x.shape
    with _on(stream) as st:
        if h is None:
            h = torch.empty((b, t, d), dtype=x.dtype, device=x.device)
        else:
            _value(h, "h", 3, x.shape)
            _need(h.dtype == x.dtype, "h must have x's type")
        a.h, a.h_stride_b, a.h_stride_t = h.data_ptr(), h.stride(0), h.stride(1)
        last = torch.empty((b, d), dtype=torch.float32, device=x.device)
        a.h_last = last.data_ptr()
        n = C.c_size_t()
        if save:
            _global_check(lib, lib.pnn_recur_saved_size(C.byref(a), C.byref(n)))
            saved = torch.empty(n.value, dtype=torch.float32, device=x.device)
            a.saved = saved.data_ptr()
        _global_check(lib, lib.pnn_recur_workspace_bytes(C.byref(a), 0, C.byref(n)))
        ws = torch.empty(n.value, dtype=torch.uint8, device=x.device) if n.value else None
        _global_check(lib, lib.pnn_recur_forward(C.byref(a), None if ws is None else ws.data_ptr(), n.value, st))
    return (h, last, saved) if save else (h, last)


def recur_grad(z, x, saved, dh, dh_last=None, lengths=None, stream=None):
    """Backward of recur: (dz, dx, dh0) from dh (batch x time x channels, x's
    type) and dh_last (fp32 batch x channels or None).  z, x and lengths as in
    the forward that returned `saved`."""
    a = _recur_args(z, x, lengths)
    lib = load()
    b, t, d = x.shape
    _value(dh, "dh", 3, x.shape)
    _need(dh.dtype == x.dtype, "dh must have x's type")
    a.dh, a.dh_stride_b, a.dh_stride_t = dh.data_ptr(), dh.stride(0), dh.stride(1)
    a.dh_last = _flat(dh_last, "dh_last", torch.float32, (b, d))
    n = C.c_size_t()
    _global_check(lib, lib.pnn_recur_saved_size(C.byref(a), C.byref(n)))
    a.saved = _flat(saved, "saved", torch.float32, (n.value,))
    _global_check(lib, lib.pnn_recur_workspace_bytes(C.byref(a), 1, C.byref(n)))
    with _on(stream) as st:
        dz = torch.empty(z.shape, dtype=x.dtype, device=x.device)
        dx = torch.empty((b, t, d), dtype=x.dtype, device=x.device)
        dh0 = torch.empty((b, d), dtype=torch.float32, device=x.device)
        a.dz, a.dz_stride_b, a.dz_stride_t = dz.data_ptr(), dz.stride(0), dz.stride(1)
        a.dx, a.dx_stride_b, a.dx_stride_t = dx.data_ptr(), dx.stride(0), dx.stride(1)
        a.dh0 = dh0.data_ptr()
        ws = torch.empty(n.value, dtype=torch.uint8, device=x.device) if n.value else None
        _global_check(lib, lib.pnn_recur_backward(C.byref(a), None if ws is None else ws.data_ptr(), n.value, st))
    return dz, dx, dh0


def recur_step(z, x, state, slots=None, out=None, stream=None):
    """One token for each sequence of the batch: row i advances state[slots[i]]
    (fp32, slots x channels) in place and the result, rounded, is returned
    (batch x channels).  A slot outside the pool marks an empty place."""
    _value(z, "z", 2)
    _value(x, "x", 2)
    _value(state, "state", 2, (state.shape[0], x.shape[1]))
    (b, h), d = z.shape, x.shape[1]
    _need(x.shape[0] == b and x.dtype == z.dtype and h > 0 and d % h == 0 and state.dtype == torch.float32,
          "x must be batch x channels of z's type, its channels a multiple of z's heads; state fp32 slots x channels")
    lib = load()
    with _on(stream) as st:
        if out is None:
            out = torch.empty((b, d), dtype=x.dtype, device=x.device)
        else:
            _value(out, "out", 2, (b, d))
            _need(out.dtype == x.dtype, "out must have x's type")
        a = RecurStepArgs(b, h, d // h, state.shape[0], _DT[x.dtype], z.data_ptr(), z.stride(0),
                          x.data_ptr(), x.stride(0), _flat(slots, "slots", torch.int32, (b,)),
                          state.data_ptr(), max(state.stride(0), d) if state.shape[0] <= 1 else state.stride(0),
                          out.data_ptr(), out.stride(0))
        _global_check(lib, lib.pnn_recur_step(C.byref(a), st))
    return out


def distill(logits, ids, teacher, labels=None, weight=None, tau=1.0, alpha=1.0, grad=True, out=None, stream=None):
    """Per-row loss (fp32) and gradient of the logits (None with grad=False).
    logits: rows x vocab; ids (int32) and teacher: rows x k; labels (int32) and
    weight (fp32): rows.  out: the gradient's buffer, may be the logits."""
    _value(logits, "logits", 2)
    r, v = logits.shape
    k = 0 if ids is None else ids.shape[-1]
    lib = load()
    a = DistillArgs(r, v, k, _DT[logits.dtype], logits.data_ptr(), logits.stride(0))
    if k:
        a.ids = _flat(ids, "ids", torch.int32, (r, k))
        _value(teacher, "teacher", 2, (r, k))
        a.teacher, a.teacher_dtype = _flat(teacher, "teacher", teacher.dtype, (r, k)), _DT[teacher.dtype]
    a.labels, a.weight = _flat(labels, "labels", torch.int32, (r,)), _flat(weight, "weight", torch.float32, (r,))
    a.tau, a.alpha = tau, alpha
    with _on(stream) as st:
        loss = torch.empty(r, dtype=torch.float32, device=logits.device)
        a.loss = loss.data_ptr()
        if grad:
            if out is None:
                out = torch.empty((r, v), dtype=logits.dtype, device=logits.device)
            else:
                _value(out, "out", 2, (r, v))
                _need(out.dtype == logits.dtype, "out must have the logits' type")
            a.dlogits, a.dlogits_stride = out.data_ptr(), out.stride(0)
        _global_check(lib, lib.pnn_distill(C.byref(a), st))
    return loss, (out if grad else None)

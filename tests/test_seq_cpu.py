"""Host-side checks of the token-sequence calls (no GPU): the argument rules of
include/pnn.h, answered before any device work, and the fp64 references of
the GPU tests against torch autograd and closed forms."""
import ctypes as C
import math

import pytest
import torch

import seq_ref as R

FAKE = 4096  # an address that is never used: every call below is refused (or has nothing to do) on the host


@pytest.fixture(scope="module")
def pnn():
    from paper_2103_08802_gb300 import build, pnn as P
    build.build()
    P.load()
    return P


def embed_args(P, **kw):
    a = P.EmbedArgs(5, 9, 16, FAKE, 32, 1.0, FAKE, 0, 16, FAKE, 0, 16, FAKE, 0, 16, FAKE, 0, 16, 0)
    for k, v in kw.items():
        setattr(a, k, v)
    return C.byref(a)


def recur_args(P, **kw):
    a = P.RecurArgs(2, 7, 4, 3, 0)
    for n, d in (("z", 4), ("x", 12), ("h", 12), ("dh", 12), ("dz", 4), ("dx", 12)):
        setattr(a, n, FAKE)
        setattr(a, n + "_stride_b", 7 * d)
        setattr(a, n + "_stride_t", d)
    a.saved = FAKE
    for k, v in kw.items():
        setattr(a, k, v)
    return C.byref(a)


def step_args(P, **kw):
    a = P.RecurStepArgs(2, 4, 3, 5, 0, FAKE, 4, FAKE, 12, FAKE, FAKE, 12, FAKE, 12)
    for k, v in kw.items():
        setattr(a, k, v)
    return C.byref(a)


def distill_args(P, **kw):
    a = P.DistillArgs(3, 10, 2, 0, FAKE, 10, FAKE, FAKE, 0, FAKE, FAKE, 1.0, 0.5, FAKE, FAKE + 4096, 10)
    for k, v in kw.items():
        setattr(a, k, v)
    return C.byref(a)


BAD = [
    ("pnn_embed_forward", embed_args, dict(tokens=-1)), ("pnn_embed_forward", embed_args, dict(tokens=2 ** 31)),
    ("pnn_embed_forward", embed_args, dict(vocab=0)), ("pnn_embed_forward", embed_args, dict(width=0)),
    ("pnn_embed_forward", embed_args, dict(ids=None)), ("pnn_embed_forward", embed_args, dict(ids_bits=16)),
    ("pnn_embed_forward", embed_args, dict(ids=FAKE + 4, ids_bits=64)), ("pnn_embed_forward", embed_args, dict(table=None)),
    ("pnn_embed_forward", embed_args, dict(table=FAKE + 2)), ("pnn_embed_forward", embed_args, dict(table_dtype=2)),
    ("pnn_embed_forward", embed_args, dict(out_stride=15)), ("pnn_embed_forward", embed_args, dict(table_stride=-16)),
    ("pnn_recur_forward", recur_args, dict(batch=0)), ("pnn_recur_forward", recur_args, dict(batch=65536)),
    ("pnn_recur_forward", recur_args, dict(time=0)), ("pnn_recur_forward", recur_args, dict(heads=2 ** 30)),
    ("pnn_recur_forward", recur_args, dict(width=0)), ("pnn_recur_forward", recur_args, dict(dtype=7)),
    ("pnn_recur_forward", recur_args, dict(z=None)), ("pnn_recur_forward", recur_args, dict(x=FAKE + 1)),
    ("pnn_recur_forward", recur_args, dict(h=None)), ("pnn_recur_forward", recur_args, dict(h_stride_t=11)),
    ("pnn_recur_forward", recur_args, dict(h_stride_b=12)), ("pnn_recur_forward", recur_args, dict(x_stride_t=-12)),
    ("pnn_recur_forward", recur_args, dict(h0=FAKE + 2)), ("pnn_recur_forward", recur_args, dict(saved=FAKE + 2)),
    ("pnn_recur_step", step_args, dict(batch=-1)), ("pnn_recur_step", step_args, dict(slot=None, slots=1)),
    ("pnn_recur_step", step_args, dict(state=None)), ("pnn_recur_step", step_args, dict(state_stride=11)),
    ("pnn_recur_step", step_args, dict(h_stride=3)), ("pnn_recur_step", step_args, dict(x=None)),
    ("pnn_recur_step", step_args, dict(dtype=-1)), ("pnn_recur_step", step_args, dict(slots=-1)),
    ("pnn_distill", distill_args, dict(rows=-1)), ("pnn_distill", distill_args, dict(vocab=0)),
    ("pnn_distill", distill_args, dict(k=1025)), ("pnn_distill", distill_args, dict(k=-1)),
    ("pnn_distill", distill_args, dict(tau=0.0)), ("pnn_distill", distill_args, dict(tau=math.nan)),
    ("pnn_distill", distill_args, dict(tau=math.inf)), ("pnn_distill", distill_args, dict(alpha=1.01)),
    ("pnn_distill", distill_args, dict(alpha=-0.1)), ("pnn_distill", distill_args, dict(alpha=math.nan)),
    ("pnn_distill", distill_args, dict(logits=None)), ("pnn_distill", distill_args, dict(ids=None)),
    ("pnn_distill", distill_args, dict(teacher=None)), ("pnn_distill", distill_args, dict(teacher_dtype=3)),
    ("pnn_distill", distill_args, dict(loss=None)), ("pnn_distill", distill_args, dict(dlogits_stride=9)),
    ("pnn_distill", distill_args, dict(dlogits=FAKE, dlogits_stride=12)), ("pnn_distill", distill_args, dict(labels=FAKE + 1)),
    ("pnn_distill", distill_args, dict(dtype=5)),
]


@pytest.mark.parametrize("call,make,kw", BAD, ids=lambda v: str(v) if isinstance(v, (str, dict)) else "")
def test_bad_arguments_are_refused(pnn, call, make, kw):
    lib = pnn.load()
    more = (None, 0) if call == "pnn_recur_forward" else ()
    assert getattr(lib, call)(make(pnn, **kw), *more, None) == 1
    assert lib.pnn_last_error(None).startswith(b"pnn_")


def test_null_arguments_and_outputs(pnn):
    lib, nb = pnn.load(), C.c_size_t()
    for call in ("pnn_embed_forward", "pnn_recur_step", "pnn_distill"):
        assert getattr(lib, call)(None, None) == 1
    for call in ("pnn_embed_backward", "pnn_recur_forward", "pnn_recur_backward"):
        assert getattr(lib, call)(None, None, 0, None) == 1
    for call, make, more in (("pnn_embed_workspace_bytes", embed_args, ()), ("pnn_recur_workspace_bytes", recur_args, (1,)),
                             ("pnn_recur_saved_size", recur_args, ())):
        assert getattr(lib, call)(make(pnn), *more, None) == 1
        assert getattr(lib, call)(None, *more, C.byref(nb)) == 1
        assert getattr(lib, call)(make(pnn), *more, C.byref(nb)) == 0 and nb.value > 0


def test_workspaces_are_checked(pnn):
    lib, nb = pnn.load(), C.c_size_t()
    assert lib.pnn_embed_workspace_bytes(embed_args(pnn), C.byref(nb)) == 0
    assert lib.pnn_embed_backward(embed_args(pnn), FAKE, nb.value - 1, None) == 2
    assert lib.pnn_embed_backward(embed_args(pnn), FAKE + 16, nb.value, None) == 1
    assert lib.pnn_embed_backward(embed_args(pnn, dtable=None), FAKE, nb.value, None) == 1
    assert lib.pnn_embed_backward(embed_args(pnn, dout=None), FAKE, nb.value, None) == 1
    assert lib.pnn_embed_backward(embed_args(pnn, dout_stride=8), FAKE, nb.value, None) == 1
    assert lib.pnn_recur_workspace_bytes(recur_args(pnn), 1, C.byref(nb)) == 0
    assert lib.pnn_recur_backward(recur_args(pnn), FAKE, nb.value - 1, None) == 2
    assert lib.pnn_recur_backward(recur_args(pnn), None, nb.value, None) == 1
    assert lib.pnn_recur_backward(recur_args(pnn, saved=None), FAKE, nb.value, None) == 1
    assert lib.pnn_recur_backward(recur_args(pnn, dz_stride_t=3), FAKE, nb.value, None) == 1
    assert lib.pnn_recur_backward(recur_args(pnn, dh=None), FAKE, nb.value, None) == 1


def test_nothing_to_do_is_no_error(pnn):
    lib = pnn.load()
    assert lib.pnn_embed_forward(embed_args(pnn, tokens=0, ids=None, table=None), None) == 0
    assert lib.pnn_embed_backward(embed_args(pnn, tokens=0, accumulate=1), None, 0, None) == 0
    assert lib.pnn_recur_step(step_args(pnn, batch=0), None) == 0
    assert lib.pnn_distill(distill_args(pnn, rows=0, logits=None), None) == 0


def test_reference_gradients_against_autograd():
    """The references' hand-written gradients equal torch autograd of their own forward to fp64 rounding."""
    g = torch.Generator().manual_seed(1)
    z = torch.randn(2, 6, 3, generator=g, dtype=torch.float64, requires_grad=True)
    x = torch.randn(2, 6, 6, generator=g, dtype=torch.float64, requires_grad=True)
    h0 = torch.randn(2, 6, generator=g, dtype=torch.float64, requires_grad=True)
    n = torch.tensor([6, 4])
    dh, dl = torch.randn(2, 6, 6, generator=g, dtype=torch.float64), torch.randn(2, 6, generator=g, dtype=torch.float64)
    s, loss = h0, 0.0
    f = torch.sigmoid(z).repeat_interleave(2, -1)
    for t in range(6):
        on = (t < n)[:, None]
        s = torch.where(on, f[:, t] * s + (1 - f[:, t]) * x[:, t], s)
        loss = loss + torch.where(on, s * dh[:, t], 0.0).sum()
    (loss + (s * dl).sum()).backward()
    got = R.recur_grad(z.detach(), x.detach(), 2, dh, dl, h0.detach(), n)
    for a, e in zip(got, (z.grad, x.grad, h0.grad)):
        assert float((a - e).abs().max()) <= 1e-13
    s = torch.randn(3, 8, generator=g, dtype=torch.float64, requires_grad=True)
    ids, t = torch.tensor([[1, 2, 2], [0, 5, -1], [-1, 9, -1]]), torch.randn(3, 3, generator=g, dtype=torch.float64)
    labels, w = torch.tensor([2, -1, 7]), torch.tensor([0.5, 2.0, 1.0])
    loss, dl, _, _ = R.distill(s.detach(), ids, t, labels, w, 2.0, 0.6)
    total = []
    for i in range(3):
        ok = (ids[i] >= 0) & (ids[i] < 8)
        row = torch.zeros((), dtype=torch.float64)
        if ok.any():
            p = torch.softmax(t[i][ok] / 2.0, 0)
            row = 0.6 * 4.0 * (p * (p.log() - torch.log_softmax(s[i] / 2.0, 0)[ids[i][ok]])).sum()
        if labels[i] >= 0:
            row = row - 0.4 * torch.log_softmax(s[i], 0)[labels[i]]
        total.append(row)
    total = torch.stack(total)
    assert float((total.detach() - loss).abs().max()) <= 1e-12
    (total * w.double()).sum().backward()
    assert float((s.grad - dl).abs().max()) <= 1e-12

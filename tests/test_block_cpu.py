"""Linear attention, norms and policy loss without a GPU: arguments refused on the
host, and the fp64 references of the GPU tests against autograd and closed forms."""
import ctypes as C
import math

import pytest
import torch

import block_ref as B
from test_seq_args_cpu import host  # noqa: F401

FAKE = 4096  # an address that is never used: every call below is refused on the host


@pytest.fixture(scope="module")
def pnn():
    from paper_2103_08802_gb300 import build, pnn as P
    build.build()
    P.load()
    return P


def attend_args(P, **kw):
    row = lambda d: (FAKE, 7 * 3 * d, 3 * d, d)  # noqa: E731
    a = P.AttendArgs(2, 7, 3, 8, 16, 0, 1.0, *row(8), *row(8), *row(16), FAKE, FAKE, FAKE, *row(16), FAKE, *row(16), FAKE, *row(8), *row(8), *row(16), FAKE)
    for k, v in kw.items():
        setattr(a, k, v)
    return C.byref(a)


def step_args(P, **kw):
    a = P.AttendStepArgs(2, 3, 8, 16, 5, 0, 1.0, FAKE, 24, 8, FAKE, 24, 8, FAKE, 48, 16, FAKE, FAKE, FAKE, 384, FAKE, 48, 16)
    for k, v in kw.items():
        setattr(a, k, v)
    return C.byref(a)


def norm_args(P, **kw):
    a = P.NormArgs(5, 16, 0, 1, 1.0, 1e-6, *(FAKE, 16) * 3, FAKE, FAKE, FAKE, *(FAKE, 16) * 7, FAKE, FAKE, FAKE)
    for k, v in kw.items():
        setattr(a, k, v)
    return C.byref(a)


def policy_args(P, **kw):
    a = P.PolicyArgs(3, 10, 0, FAKE, 10, FAKE, FAKE, FAKE, FAKE, FAKE, 0.2, 0.2, 0.1, 1.0, FAKE, FAKE, FAKE + 4096, 10)
    for k, v in kw.items():
        setattr(a, k, v)
    return C.byref(a)


FORWARD, BACKWARD = "pnn_attend_forward", "pnn_attend_backward"
BAD = [
    *((FORWARD, attend_args, kw) for kw in (
        dict(batch=0), dict(heads=0), dict(batch=2 ** 16, heads=2 ** 15), dict(time=0), dict(time=2 ** 31 - 100), dict(time=2 ** 30 + 1), dict(batch=2 ** 15, heads=2 ** 14 + 1), dict(dk=0), dict(dk=257), dict(dv=257),
        dict(dtype=2), dict(scale=math.nan), dict(scale=math.inf), dict(q=None), dict(k=FAKE + 2), dict(v_stride_t=-16), dict(o=None),
        dict(o_stride_h=15), dict(o_stride_t=47), dict(o_stride_b=330), dict(decay=None), dict(decay=FAKE + 2), dict(lengths=FAKE + 1),
        dict(s0=FAKE + 2), dict(s_last=FAKE + 1))),
    *((BACKWARD, attend_args, kw) for kw in (
        dict(dout=None), dict(dq=None), dict(dk_out_stride_t=23), dict(dv_out_stride_h=8), dict(ds_last=FAKE + 2), dict(ds0=FAKE + 2), dict(dq_stride_b=0))),
    *(("pnn_attend_step", step_args, kw) for kw in (
        dict(batch=-1), dict(batch=65536), dict(heads=0), dict(heads=32768), dict(dk=257), dict(dv=0), dict(slots=-1), dict(slot=None, slots=1), dict(state=None),
        dict(state=FAKE + 2), dict(state_stride=383), dict(decay=None), dict(o_stride_h=15), dict(o_stride_b=47), dict(q=None), dict(v=FAKE + 1), dict(scale=math.nan))),
    *(("pnn_norm_forward", norm_args, kw) for kw in (
        dict(rows=-1), dict(rows=2 ** 31), dict(width=0), dict(width=16385), dict(dtype=3), dict(res_dtype=-1), dict(eps=0.0), dict(eps=math.inf), dict(eps=math.nan),
        dict(scale=math.nan), dict(weight=FAKE + 2), dict(x=None), dict(gate=FAKE + 2), dict(res=FAKE + 1), dict(h=None), dict(h_stride=15), dict(n=None),
        dict(n_stride=0), dict(x_stride=-16))),
    *(("pnn_norm_backward", norm_args, kw) for kw in (
        dict(weight=None), dict(scales=None), dict(next_weight=None), dict(gate=None), dict(dn=None), dict(dx=None), dict(dgate_stride=15),
        dict(dres=FAKE + 1), dict(dweight=FAKE + 2), dict(dh=FAKE + 1))),
    *(("pnn_policy", policy_args, kw) for kw in (
        dict(rows=-1), dict(rows=2 ** 31), dict(vocab=0), dict(dtype=4), dict(logits=None), dict(logits_stride=-1), dict(labels=None), dict(advantage=None), dict(loss=None),
        dict(old=FAKE + 1), dict(ref=FAKE + 2), dict(weight=FAKE + 3), dict(logp=FAKE + 1), dict(tau=0.0), dict(tau=math.inf), dict(tau=math.nan), dict(tau=4e-39),
        dict(clip_low=-0.1), dict(clip_low=1.1), dict(clip_low=math.nan), dict(clip_high=-0.1), dict(clip_high=math.nan), dict(beta=-1.0), dict(beta=math.inf),
        dict(dlogits_stride=9), dict(dlogits=FAKE, dlogits_stride=12), dict(dlogits=FAKE + 4097))),
]


@pytest.mark.parametrize("call,make,kw", BAD, ids=lambda v: str(v) if isinstance(v, (str, dict)) else "")
def test_bad_arguments_are_refused(pnn, call, make, kw):
    lib = pnn.load()
    more = (FAKE, 2 ** 40) if call in (FORWARD, BACKWARD, "pnn_norm_backward") else ()
    assert getattr(lib, call)(make(pnn, **kw), *more, None) == 1
    assert lib.pnn_last_error(None).startswith(b"pnn_")


def test_workspaces_and_nothing(pnn):
    lib, nb = pnn.load(), C.c_size_t()
    for call, more in ((FORWARD, (None, 0)), (BACKWARD, (None, 0)), ("pnn_attend_step", ()), ("pnn_norm_forward", ()), ("pnn_norm_backward", (None, 0)), ("pnn_policy", ())):
        assert getattr(lib, call)(None, *more, None) == 1
    long = attend_args(pnn, batch=1, heads=1, time=100000)
    assert lib.pnn_attend_workspace_bytes(long, 0, C.byref(nb)) == 0 and nb.value > 0
    assert lib.pnn_attend_workspace_bytes(long, 1, None) == 1
    assert lib.pnn_norm_workspace_bytes(norm_args(pnn), C.byref(nb)) == 0 and nb.value > 0
    assert lib.pnn_norm_backward(norm_args(pnn), FAKE, nb.value - 1, None) == 2
    assert lib.pnn_norm_backward(norm_args(pnn), FAKE + 16, nb.value, None) == 1
    assert lib.pnn_norm_backward(norm_args(pnn), None, nb.value, None) == 1
    assert lib.pnn_policy(policy_args(pnn, rows=0), None) == 0 and lib.pnn_norm_forward(norm_args(pnn, rows=0), None) == 0
    assert lib.pnn_attend_step(step_args(pnn, batch=0), None) == 0


def test_the_bindings_refuse(host):  # noqa: F811
    """Types, shapes and missing partners are answered before the library is reached."""
    from paper_2103_08802_gb300 import seq
    q, v, a = torch.zeros(2, 5, 3, 8), torch.zeros(2, 5, 3, 16), torch.ones(3)
    bad = [lambda: seq.attend(q, q[:, :4], v, a), lambda: seq.attend(q, q, v[:1], a), lambda: seq.attend(q, q, v.bfloat16(), a),
           lambda: seq.attend(q, q.half(), v, a), lambda: seq.attend(q, q, v, a[:2]), lambda: seq.attend(q, q, v, a.double()),
           lambda: seq.attend(q[0], q[0], v[0], a), lambda: seq.attend(q.transpose(2, 3), q, v, a), lambda: seq.attend(q, q, v, a, s0=torch.zeros(2, 3, 16, 8)),
           lambda: seq.attend(q, q, v, a, lengths=torch.zeros(2)), lambda: seq.attend(q, q, v, a, o=v.bfloat16()), lambda: seq.attend_grad(q, q, v, a, q),
           lambda: seq.attend_grad(q, q, v, a, v.bfloat16()), lambda: seq.attend_grad(q, q, v, a, v, ds_last=torch.zeros(2, 3, 8)),
           lambda: seq.attend_step(q[:, 0], q[:, 0], v[:, 0], a, torch.zeros(4, 3, 16, 8)), lambda: seq.attend_step(q[:, 0], q[:, 0], v[:, 0], a, torch.zeros(4, 3, 8, 16).bfloat16()),
           lambda: seq.attend_step(q[:, 0], q[:, 0], v[:, 0], a, torch.zeros(4, 8, 3, 16).transpose(1, 2)),
           lambda: seq.attend_step(q[:, 0], q[:, 0], v[:, 0], a, torch.zeros(4, 3, 8, 16), slots=torch.zeros(2))]
    x, w = torch.zeros(4, 8), torch.ones(8)
    bad += [lambda: seq.norm(x, weight=w[:7]), lambda: seq.norm(x, weight=w.bfloat16()), lambda: seq.norm(x, gate=x.bfloat16()), lambda: seq.norm(x, gate=x[:3]),
            lambda: seq.norm(x, res=x.half()), lambda: seq.norm(x, res=x[:, :4]), lambda: seq.norm(x, scale=w[:3]), lambda: seq.norm(x.half(), weight=w),
            lambda: seq.norm_grad(x, x, dn=x, weight=w), lambda: seq.norm_grad(x, x, weight=w, next_weight=w), lambda: seq.norm_grad(x, x.bfloat16(), weight=w),
            lambda: seq.norm_grad(x, x, weight=w, res=x.bfloat16()), lambda: seq.norm(torch.tensor(1.0), weight=w)]
    s, n, f = torch.zeros(4, 9), torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    bad += [lambda: seq.policy(s, None, f), lambda: seq.policy(s, n, None), lambda: seq.policy(s, n.long(), f), lambda: seq.policy(s, n, f.double()),
            lambda: seq.policy(s, n, f[:3]), lambda: seq.policy(s, n, f, old=f[:1]), lambda: seq.policy(s, n, f, out=s.bfloat16()), lambda: seq.policy(s.half(), n, f)]
    for i, call in enumerate(bad):
        with pytest.raises(TypeError):
            call()
            pytest.fail(str(i))


def test_attend_reference_against_autograd():
    g = torch.Generator().manual_seed(1)
    f = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    q, k, v, do, s0, ds = f(2, 6, 2, 3), f(2, 6, 2, 3), f(2, 6, 2, 4), f(2, 6, 2, 4), f(2, 2, 3, 4), f(2, 2, 3, 4)
    a, ln = torch.tensor([0.9, 0.0], dtype=torch.float64), torch.tensor([6, 3])
    xs = [x.clone().requires_grad_() for x in (q, k, v, s0)]
    o, s = B.attend(*xs[:3], a, xs[3], ln, 0.7)
    grads = torch.autograd.grad((o * do).sum() + (s * ds).sum(), xs)
    for x, y in zip(B.attend_grad(q, k, v, a, do, s0, ds, ln, 0.7), grads):
        assert torch.allclose(x, y, atol=1e-12)
    # the sum written out
    i = torch.arange(6)
    m = torch.where(i[:, None] >= i, 0.9 ** (i[:, None] - i).clamp(min=0), 0.0)
    want = 0.7 * ((q[0, :, 0] @ k[0, :, 0].t()) * m) @ v[0, :, 0] + 0.7 * 0.9 ** (i[:, None] + 1.0) * (q[0, :, 0] @ s0[0, 0])
    assert torch.allclose(o[0, :, 0], want, atol=1e-12)


def test_policy_reference_against_autograd():
    g = torch.Generator().manual_seed(2)
    s = torch.randn(8, 11, generator=g, dtype=torch.float64).requires_grad_()
    labels, A = torch.randint(0, 11, (8,), generator=g), torch.randn(8, generator=g, dtype=torch.float64)
    lp = torch.log_softmax(s / 1.3, 1).gather(1, labels[:, None])[:, 0]
    old, ref = lp.detach() - 0.4 * torch.randn(8, generator=g, dtype=torch.float64), lp.detach() + torch.randn(8, generator=g, dtype=torch.float64)
    w = torch.rand(8, generator=g, dtype=torch.float64)
    r = torch.exp(lp - old)
    loss = -torch.minimum(r * A, r.clamp(0.8, 1.3) * A) + 0.2 * (torch.exp(ref - lp) - (ref - lp) - 1)
    want, = torch.autograd.grad((loss * w).sum(), s)
    got, _ = B.policy(s.detach(), labels, A, old, ref, w, (0.2, 0.3), 0.2, 1.3)
    assert torch.allclose(got[0], loss.detach(), atol=1e-12) and torch.allclose(got[1], lp.detach(), atol=1e-12)
    assert torch.allclose(got[2], want, atol=1e-12)


def test_norm_reference_by_hand():
    x, w = torch.tensor([[3.0, 4.0]], dtype=torch.float64), torch.tensor([2.0, 1.0], dtype=torch.float64)
    r = 1 / math.sqrt(12.5 + 1e-6)
    h, n = B.norm(x, weight=w, scale=0.5, res=x, next_weight=w)
    assert torch.allclose(h, torch.tensor([[3 + 3 * r, 4 + 2 * r]], dtype=torch.float64))
    assert torch.allclose(n, h * w / math.sqrt(h.square().mean() + 1e-6))
    # (a closed form: the gradient of x / rms along x itself is that of eps alone)
    d = B.norm_grad(x, x * 0 + torch.tensor([1.0, 0.0]), weight=torch.ones(2).double())["x"]
    assert abs(float((d * x).sum())) < 1e-6

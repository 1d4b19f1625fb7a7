"""Token-sequence operators on the GPU at the edges of what they accept: offsets
beyond 32 bits, limits of shared memory, streams, status, forms that few calls
take.  Exact values where the arithmetic gives them, else the fp64
implementations and bounds of seq_ref."""
import math
import os
import subprocess
import sys

import pytest
import torch

import seq_ref as R
from test_gpu_seq import dev, held, randn

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
INF = math.inf


@pytest.fixture(scope="module")
def seq():
    from paper_2103_08802_gb300 import build
    build.build()
    from paper_2103_08802_gb300 import seq as S
    return S


def test_states_beyond_32_bits(seq):
    """batch x channels above 2^31: every sequence reads its own h0 and dh_last and writes its own h_last and dh0.  One
    step from z = +inf keeps a state to the bit and from z = -inf replaces it, so that sums of 0 and 1 are exact."""
    b, d = 65535, 32832
    assert (b - 1) * d > 2 ** 31
    z = torch.zeros(b, 1, 1, dtype=BF, device="cuda")
    z[::2], z[1::2] = INF, -INF
    x = torch.full((b, 1, d), 2.0, dtype=BF, device="cuda")
    row = (torch.arange(b, device="cuda") % 127).float()[:, None]  # a value of each sequence's own, exact in bf16
    col = torch.arange(d, device="cuda").float() % 2 - 0.5
    h0 = row * col
    h, last, saved = seq.recur(z, x, h0=h0, save=True)
    assert torch.equal(last[::2], h0[::2]) and bool((last[1::2] == 2).all())
    assert torch.equal(saved.view(b, d), h0)
    assert torch.equal(h[-3:, 0].float(), last[-3:])
    del last, saved, h
    saved = h0.clone().view(-1)
    dz, dx, dh0 = seq.recur_grad(z, x, saved, x, dh_last=h0)
    want = h0[::2] + 2  # G = dh + dh_last, kept by f = 1
    assert torch.equal(dh0[::2], want) and bool((dh0[1::2] == 0).all())
    del want, dh0
    assert bool((dx[::2] == 0).all()) and bool((dz == 0).all())
    assert torch.equal(dx[-4::2, 0], (h0[-4::2] + 2).to(BF))


def test_distill_near_the_default_shared_memory(seq):
    """Lists of pairs that bring a CTA's shared memory just below 48 KB without the kernel's own, each the first call of
    its kernel in a fresh process: a larger list before it would have raised the limit for all."""
    code = """
import torch
import test_gpu_seq as T
from paper_2103_08802_gb300 import seq
BF, F32 = torch.bfloat16, torch.float32
for v, ks, dt in ((10000, (160, 159, 169), BF), (6000, (165, 159, 169), F32), (4000, (935, 932, 937), BF), (4000, (935, 932, 937), F32)):
    for k in ks:
        T.check_distill(seq, *T.dist_case((2, v, k, dt, F32, 1.0, 1.0, False)))
"""
    here = os.path.dirname(os.path.abspath(__file__))
    env = dict(os.environ, PYTHONPATH=os.pathsep.join([os.path.dirname(here), here, os.environ.get("PYTHONPATH", "")]))
    out = subprocess.run([sys.executable, "-c", code], env=env, capture_output=True, text=True)
    assert out.returncode == 0, out.stderr[-2000:]


def test_embed_grad_copies_rows_on_its_stream(seq):
    """A dout whose rows cannot be viewed as a matrix, made late on the call's stream: the copy follows it there, and its
    memory is not handed to the current stream while the call still reads it."""
    s = torch.cuda.Stream()
    g = torch.Generator().manual_seed(21)
    ids, base = torch.randint(0, 50, (16, 128), generator=g).cuda(), torch.randint(-8, 9, (128, 16, 64), generator=g).float().cuda()
    want = torch.zeros(50, 64, device="cuda").index_add_(0, ids.view(-1), (base * 2).transpose(0, 1).reshape(-1, 64))  # whole numbers
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        dout = (base * 2).transpose(0, 1)
    got = seq.embed_grad(ids, dout, vocab=50, stream=s)
    junk = [torch.full((16 * 128, 64), 1e9, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert torch.equal(got, want) and len(junk) == 4


def test_distill_entries_are_written_last(seq):
    """Rows of a warp whose pairs and labels lie among other lanes' vectors: every named place holds its own gradient, not
    the softmax that another lane wrote there, in all of many rows and calls."""
    g = torch.Generator().manual_seed(22)
    for v, k, dt in ((2000, 32, BF), (1000, 31, F32), (300, 7, F32)):
        s = (randn(g, 8, v) * 2).to(dt)
        ids = torch.stack([torch.randperm(v, generator=g)[:k] for _ in range(8)]).int()
        t, labels = randn(g, 8, k), torch.randint(0, v, (8,), generator=g).int()
        loss, dl, bl, bd = R.distill(s, ids, t, labels, None, 2.0, 0.5)
        sc, ic, tc, lc = (w.repeat(500, *[1] * (w.dim() - 1)) for w in dev(s, ids, t, labels))
        first = seq.distill(sc, ic, tc, labels=lc, tau=2.0, alpha=0.5)
        held("loss", first[0][:8], loss, bl)
        held("grad", first[1][:8], dl, bd)
        for _ in range(5):
            grad = seq.distill(sc, ic, tc, labels=lc, tau=2.0, alpha=0.5)[1]
            assert torch.equal(grad.view(500, 8, v), first[1][:8].expand(500, 8, v))


def test_embed_grad_of_a_broadcast_row(seq):
    """One row for all tokens (the gradient of a sum over them), as expand gives it: whole numbers, exact."""
    g = torch.Generator().manual_seed(23)
    ids = torch.randint(-1, 40, (3, 700), generator=g).cuda()
    count = torch.bincount(ids[ids >= 0], minlength=40).float()[:, None]
    for d, dt in ((72, BF), (333, F32)):
        row = torch.randint(-8, 9, (d,), generator=g).to(dt).cuda()
        for dout in (row.expand(2100, d), row.expand(3, 700, d)):
            assert torch.equal(seq.embed_grad(ids if dout.dim() == 3 else ids.view(-1), dout, vocab=40), count * row.float())


def test_distill_smallest_tau(seq):
    """At the smallest tau each softmax is its maximum alone: a student that agrees has no loss, and no NaN."""
    s, ids = torch.tensor([[0.0, 3.0, 1.0]], device="cuda"), torch.tensor([[1, 2]], dtype=torch.int32, device="cuda")
    loss, grad = seq.distill(s, ids, torch.tensor([[5.0, 4.0]], device="cuda"), tau=4.5e-39)
    assert loss.item() == 0 and bool((grad == 0).all())


def test_gates_accuracy(seq):
    """f and 1 - f as a step shows them (from state 1 and x = 0, and the other way round): relatively accurate from z = -70
    and up to z = 87, off by 2^-126 beyond."""
    from test_seq_bounds_cpu import GATE, LEAST
    z = torch.linspace(-100, 100, 40001, dtype=torch.float64).float()
    zd, one, none = z.double(), torch.ones(1, 40001, device="cuda"), torch.zeros(1, 40001, device="cuda")
    zc = z.cuda().view(1, 1, -1)
    f, g = (seq.recur(zc, x[:, None], h0=h0)[1][0].cpu().double() for x, h0 in ((none, one), (one, none)))
    for got, exact, accurate in ((f, 1 / (1 + torch.exp(-zd)), zd >= -70), (g, 1 / (1 + torch.exp(zd)), zd <= 87)):
        lim = GATE(zd) * exact + torch.where(accurate, 0.0, LEAST)
        assert bool(((got - exact).abs() <= lim).all()), float(((got - exact).abs() / lim).max())

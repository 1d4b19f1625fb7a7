"""The plans by which the recurrence and the distillation lay a call out over
the GPU, each against the fp64 implementations within the bounds of seq_ref:
heads of widths that are no multiple of 8 on rows that TMA can swizzle, few
long sequences cut into segments for every kind of gate and row, and logits
longer than the registers of a CTA."""
import math

import pytest
import torch

import seq_ref as R
from test_gpu_seq import dev, dist_case, held, randn

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
INF = math.inf


@pytest.fixture(scope="module")
def seq():
    from paper_2103_08802_gb300 import build
    build.build()
    from paper_2103_08802_gb300 import seq as S
    return S


def rows(g, b, t, d, dt, layout):
    """aligned: rows follow one another (16-byte multiples where d is one); odd: rows of a wider buffer, an odd place in it."""
    if layout == "aligned":
        return randn(g, b, t, d, dtype=dt).cuda()
    wide = randn(g, b, t, d + 3 - d % 2, dtype=dt).cuda()
    return wide[:, :, 1:d + 1]


def check_recur(seq, b, t, heads, width, dt, layout, lengths=None, seed=31):
    g = torch.Generator().manual_seed(seed)
    d = heads * width
    z, x, dh = rows(g, b, t, heads, dt, "aligned"), rows(g, b, t, d, dt, layout), rows(g, b, t, d, dt, layout)
    z.mul_(2).add_(1.5)
    u = torch.rand(b, t, heads, generator=g).cuda()
    z[u < 0.01], z[u > 0.995] = INF, -INF
    h0, dl = randn(g, b, d), randn(g, b, d)
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)
    zc, xc, dhc = (v.cpu().contiguous() for v in (z, x, dh))
    want = R.recur(zc, xc, width, h0, n)[:2] + R.recur_grad(zc, xc, width, dhc, dl, h0, n)
    bounds = R.recur_bounds(zc, xc, width, h0, n, dhc, dl)
    nc, h0c, dlc = dev(n, h0, dl)
    if n is not None:  # what lies behind a sequence's end is not looked at
        for i, m in enumerate(n.clamp(0, t).tolist()):
            z[i, m:], x[i, m:], dh[i, m:] = float("nan"), INF, float("nan")
    got = seq.recur(z, x, h0=h0c, lengths=nc, save=True)
    grads = seq.recur_grad(z, x, got[2], dh, dh_last=dlc, lengths=nc)
    for name, a, e, lim in zip(("h", "h_last", "dz", "dx", "dh0"), (*got[:2], *grads), want, bounds):
        held(name, a, e, lim)


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("heads,width", [(80, 5), (128, 3), (64, 2), (24, 17), (8, 130), (2, 100), (1, 204), (16, 31)])
def test_other_heads_on_aligned_rows(seq, heads, width, dt):
    """Several tiles, heads that cross them, pieces that end inside a sequence; chunks of a row beyond the first."""
    check_recur(seq, 3, 155, heads, width, dt, "aligned", [155, 73, 1])


SEGMENTS = [  # batch, time, heads, width: two launches in both directions
    (1, 1100, 16, 5), (1, 1100, 40, 3), (2, 900, 8, 16), (1, 1100, 3, 64), (1, 1100, 2, 72), (1, 1000, 1, 201), (1, 1915, 80, 16),
    (1, 1915, 260, 5), (2, 901, 64, 1),
]


@pytest.mark.parametrize("layout", ["aligned", "odd"])
@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("case", SEGMENTS, ids=str)
def test_segments(seq, case, dt, layout):
    """Few chains of many pieces; sequences that end in a segment's middle, in its first step, or before it begins."""
    b, t = case[:2]
    check_recur(seq, *case, dt, layout, None if b == 1 else [t, t // 2])


def test_a_sequence_that_ends_early_in_segments(seq):
    for n in (0, 1, 72, 73, 700):
        check_recur(seq, 1, 1100, 16, 5, BF, "aligned", [n])
        check_recur(seq, 1, 1100, 4, 16, BF, "odd", [n])


TWO_WALKS = [  # rows, vocab, k, dtype, teacher, tau, alpha, labels: 160 rows or more, longer than a CTA's registers
    (160, 40001, 9, F32, F32, 2.0, 0.5, True), (160, 40001, 200, BF, BF, 3.0, 0.5, True), (330, 36000, 33, BF, F32, 1.0, 1.0, False),
    (160, 33792, 40, F32, BF, 4.0, 0.7, True), (170, 67592, 16, BF, BF, 2.0, 0.5, True), (160, 17001, 5, F32, F32, 1.0, 0.0, True),
]


@pytest.mark.parametrize("case", TWO_WALKS, ids=str)
def test_distill_long_rows(seq, case):
    """Many rows walked twice by one CTA each, with its gradient, in place and the loss alone; repeated ids, labels that the
    teacher names, masked logits, rows without a teacher or a label."""
    s, ids, t, labels, weight, tau, alpha = dist_case(case)
    n, v, k = case[:3]
    r = torch.arange(n)
    ids[r % 5 == 1, k - 1] = ids[r % 5 == 1, 0]
    ids[r % 7 == 3, 2:1 + k // 2] = -1
    ids[r % 13 == 6] = -1
    t[r % 11 == 2, 1] = -INF
    s[r % 3 == 1, v - v // 50:] = -INF
    s[r % 17 == 5, :v // 2] = torch.finfo(s.dtype).min
    s[9] = -INF
    ids[r % 3 == 1] = torch.where(ids[r % 3 == 1] >= v - v // 50, 7, ids[r % 3 == 1])  # a teacher of masked places: infinite loss
    if labels is not None:
        labels[r % 3 == 0] = ids[r % 3 == 0, 1]
        labels[r % 3 == 1] = labels[r % 3 == 1].clamp(max=v - v // 50 - 1)
    loss, dl, bl, bd = R.distill(s, ids, t, labels, weight, tau, alpha)
    loss[loss > torch.finfo(F32).max] = INF  # beyond the output's range (a teacher that names a logit at the lowest value)
    sc, ic, tc, lc, wc = dev(s, ids, t, labels, weight)
    got, grad = seq.distill(sc, ic, tc, labels=lc, weight=wc, tau=tau, alpha=alpha)
    held("loss", got, loss, bl)
    held("grad", grad, dl, bd)
    held("loss alone", seq.distill(sc, ic, tc, labels=lc, tau=tau, alpha=alpha, grad=False)[0], loss, bl)
    in_place = seq.distill(sc, ic, tc, labels=lc, weight=wc, tau=tau, alpha=alpha, out=sc)
    assert torch.equal(sc, grad) and torch.equal(in_place[0], got)


def test_distill_long_rows_at_odd_places(seq):
    """The same rows out of a wider buffer, and a gradient that starts elsewhere in 16 bytes."""
    g = torch.Generator().manual_seed(32)
    r, v, k = 160, 36003, 6
    for dt, off, to in ((BF, 1, 1), (BF, 3, 6), (F32, 2, 1)):
        wide = (randn(g, r, v + 11) * 2).to(dt)
        s = wide[:, off:off + v]
        ids, t = torch.randint(0, v, (r, k), generator=g).int(), randn(g, r, k)
        loss, dl, bl, bd = R.distill(s, ids, t, tau=2.0)
        buf = torch.full((r, v + 13), 6.0, dtype=dt, device="cuda")
        got, grad = seq.distill(wide.cuda()[:, off:off + v], ids.cuda(), t.cuda(), tau=2.0, out=buf[:, to:to + v])
        held("loss", got, loss, bl)
        held("grad", grad, dl, bd)
        assert bool((buf[:, :to] == 6).all()) and bool((buf[:, to + v:] == 6).all())

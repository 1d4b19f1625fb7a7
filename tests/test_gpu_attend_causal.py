"""Linear attention of rows that are not finite: what depends on them is not
finite, and what does not is as accurate as without them."""
import math

import pytest
import torch

import block_ref as B
import seq_ref as R
from test_gpu_block import BF, F32, attend_case, cuda, seq  # noqa: F401
from test_gpu_seq import held

pytestmark = pytest.mark.gpu

CASES = [  # batch, time, heads, dk, dv, type, lengths: either kernel, chunks whole and partial, one segment and several
    (2, 300, 2, 64, 64, BF, None), (1, 290, 4, 128, 64, BF, [257]), (1, 260, 2, 64, 128, BF, None), (1, 1600, 1, 128, 128, BF, None),
    (2, 200, 1, 72, 24, BF, [200, 131]), (1, 20, 4, 64, 64, BF, None), (2, 90, 3, 33, 65, BF, [90, 40]), (1, 200, 1, 200, 256, BF, None),
    (1, 70, 4, 40, 72, F32, None), (1, 700, 2, 24, 40, F32, [650]), (1, 100, 1, 256, 40, F32, None), (2, 33, 2, 16, 16, F32, [33, 2]),
]


@pytest.mark.parametrize("what", ["v", "k", "q", "do"])
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_rows_that_are_not_finite(seq, case, value, what):  # noqa: F811
    """One entry near a third and the whole row near four fifths of every sequence.  The rows that a chunk's product spoils are
    formed again token by token, two roundings of 2^-24 each."""
    q, k, v, do, a, s0, ds, ln = attend_case(case)
    x = {"q": q, "k": k, "v": v, "do": do}
    n = [case[1]] * case[0] if case[6] is None else case[6]
    for b, t in enumerate(n):
        x[what][b, t // 3, 0, 1] = value
        x[what][b, 4 * t // 5] = -value
    scale = case[3] ** -0.5
    f64 = B.attend(q, k, v, a, s0, ln, scale) + B.attend_grad(q, k, v, a, do, s0, ds, ln, scale)
    bounds = B.attend_bounds(q, k, v, a, do, s0, ds, ln, scale)
    m = lambda t: t.abs()  # noqa: E731
    size = B.attend(m(q), m(k), m(v), a, m(s0), ln, scale) + B.attend_grad(m(q), m(k), m(v), a, m(do), m(s0), m(ds), ln, scale)
    Q, K, V, D, A, S0, DS, LN = cuda(q, k, v, do, a, s0, ds, ln)
    got = seq.attend(Q, K, V, A, s0=S0, lengths=LN, scale=scale) + seq.attend_grad(Q, K, V, A, D, s0=S0, ds_last=DS, lengths=LN, scale=scale)
    seq.sync()
    for name, x, want, bound, s in zip(("o", "s_last", "dq", "dk", "dv", "ds0"), got, f64, bounds, size):
        fine = torch.isfinite(want)
        assert torch.equal(torch.isfinite(x).cpu(), fine), name
        keep = lambda t: torch.where(fine, t, 0.0)  # noqa: E731
        held(name, keep(x.cpu().double()).to(x.dtype).cuda(), keep(want), keep(bound + 2 * case[1] * R.U * s) + R.TINY)

"""Linear attention of short bf16 sequences whose heads need the tensor-core kernel:
how many bits its outputs have there."""
import pytest

import block_ref as B
import seq_ref as R
from test_gpu_block import BF, attend_case, cuda, near, seq  # noqa: F401
from test_gpu_seq import held

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", [(20, 32, 16, 128, 128), (20, 32, 16, 128, 64), (20, 9, 16, 72, 128), (64, 32, 16, 64, 64)], ids=str)
def test_many_short_sequences(seq, case):  # noqa: F811
    """More heads than multiprocessors: wider than 64 their scores and states have 8 bits on their way into an output, one
    rounding of 2^-8 / sqrt(3) of it in the mean beside its own; up to 64 16 bits, the output's own alone."""
    q, k, v, do, a, s0, ds, _ = attend_case((*case, BF, None))
    exact = B.attend(q, k, v, a, s0) + B.attend_grad(q, k, v, a, do, s0, ds)
    bounds = B.attend_bounds(q, k, v, a, do, s0, ds)
    Q, K, V, D, A, S0, DS = cuda(q, k, v, do, a, s0, ds)
    got = seq.attend(Q, K, V, A, s0=S0) + seq.attend_grad(Q, K, V, A, D, s0=S0, ds_last=DS)
    wide = max(case[3:]) > 64
    for name, x, want, bound in zip(("o", "s_last", "dq", "dk", "dv", "ds0"), got, exact, bounds):
        held(name, x, want, bound)
        near(name, x, want, R.U * 32 if name in ("s_last", "ds0") else 2 ** -8 if wide else 2 ** -8 / 3 ** 0.5)

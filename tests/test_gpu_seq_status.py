"""What pnn_seq_sync reports of device-side waits that gave up: a wait made to
run out after a short limit (nothing faults, hangs or traps), on one stream and
seen from others."""
import pytest
import torch

pytestmark = pytest.mark.gpu
ETIMEOUT = 5


def status(seq, stream=None):
    from paper_2103_08802_gb300.pnn import PnnError
    try:
        seq.sync(stream)
    except PnnError as e:
        return e.status
    return 0


def test_every_stream_learns_of_a_wait_that_gave_up():
    from paper_2103_08802_gb300 import build, pnn
    build.build()
    from paper_2103_08802_gb300 import seq
    lib = pnn.load()
    assert lib.pnn_selftest_seq_timeout(0, None) == 1 and lib.pnn_selftest_seq_timeout(10 ** 11, None) == 1
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for s in (None, a, b):
        status(seq, s)
    assert [status(seq, s) for s in (None, a, b)] == [0, 0, 0]
    for _ in range(2):
        assert lib.pnn_selftest_seq_timeout(1_000_000, a.cuda_stream) == 0
        a.synchronize()
        assert status(seq, b) == ETIMEOUT  # it may have been this stream's
        assert status(seq, a) == ETIMEOUT  # and was this one's, whoever asked first
        assert status(seq) == ETIMEOUT
        assert [status(seq, s) for s in (a, None, b)] == [0, 0, 0]
    # the operators go on
    table = torch.randn(9, 16, device="cuda")
    ids = torch.arange(9, device="cuda")
    assert torch.equal(seq.embed(ids, table), table) and status(seq) == 0

"""Arguments of the token-sequence calls that are answered on the host, without a GPU."""
import ctypes as C

import pytest
import torch

from paper_2103_08802_gb300 import seq


@pytest.fixture
def host(monkeypatch):
    """Host tensors stand for device tensors; the library is not reached by a call that is refused."""
    class Lib:
        def __getattr__(self, name):
            def call(*args):
                raise AssertionError(name + " was reached")
            return call
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 1, raising=False)
    monkeypatch.setattr(seq, "load", Lib)


def test_a_teacher_comes_with_its_ids(host):
    """Logits of a teacher without the places that they belong to were dropped, and the labels' term alone computed."""
    logits, ids, teacher = torch.zeros(2, 9), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3)
    for a, t in ((None, teacher), (ids, None), (ids[0], teacher), ([[1, 2, 3], [4, 5, 6]], teacher), (torch.tensor(3, dtype=torch.int32), teacher)):
        with pytest.raises(TypeError):
            seq.distill(logits, a, t, labels=ids[:, 0].contiguous())


def test_tau_whose_exponents_overflow_is_refused():
    """log2(e) / tau is a factor of every exponent; where it is infinite a row's own maximum gave 0 * inf."""
    from paper_2103_08802_gb300 import build, pnn
    build.build()
    lib = pnn.load()
    at = 4096  # never used: rows = 0 where the call is accepted
    for tau, ok in ((3.5e-39, False), (4.2e-39, False), (4.5e-39, True), (1e-30, True)):
        a = pnn.DistillArgs(0, 10, 2, 0, at, 10, at, at, 0, at, at, tau, 0.5, at, at + 4096, 10)
        assert (lib.pnn_distill(C.byref(a), None) == 0) == ok

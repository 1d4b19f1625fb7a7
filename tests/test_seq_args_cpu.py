"""Arguments of the token-sequence calls that are answered on the host, without a GPU."""
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

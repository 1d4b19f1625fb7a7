"""The token network's command and its defaults."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def seqnet():
    from paper_2103_08802_gb300 import build
    build.build()
    from paper_2103_08802_gb300 import seqnet
    return seqnet


def test_the_command_runs_to_its_end(seqnet, capsys):
    """All of its parts, a few steps each: teacher, student, linear attention, its policy, and the continuation."""
    seqnet.main(steps=4, vocab=64, k=4)
    said = capsys.readouterr().out
    for part in ("teacher:", "student: step 3", "linear attention:", "policy: step 0", "continued: ["):
        assert part in said, said

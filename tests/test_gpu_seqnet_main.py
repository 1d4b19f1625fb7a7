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


@pytest.mark.parametrize("width,heads", [(8, 1), (64, 1), (96, 1), (200, 4), (256, 4), (328, 8), (1000, 20)])
def test_default_heads_divide_the_width(seqnet, width, heads):
    """Every multiple of 8 is a width: of width // 64 heads where they divide it, else of the fewest more that do."""
    net = seqnet.SeqNet(16, width, 1, mixer="attend")
    assert (net.heads, net.head) == (heads, width // heads)
    tokens = torch.arange(10, dtype=torch.int32, device="cuda").view(2, 5)
    loss, grads = net.loss_and_grads(tokens, None, None, labels=tokens, alpha=0.0)
    assert bool(torch.isfinite(loss).all()) and grads.keys() == net.params.keys()


@pytest.mark.parametrize("mixer", ["recur", "attend"])
def test_prompts_that_are_slices(seqnet, mixer):
    """The first tokens of longer rows, and columns: as a copy of them, by either mixer."""
    net = seqnet.SeqNet(64, 64, 2, heads=8, seed=4, mixer=mixer)
    tokens = torch.randint(0, 64, (4, 12), generator=torch.Generator().manual_seed(2)).int().cuda()
    for prompt in (tokens[:, :7], tokens.t()[:5], tokens[:, ::3]):
        assert not prompt.is_contiguous()
        assert torch.equal(net.generate(prompt, 3), net.generate(prompt.contiguous(), 3))

"""The token network on a stream of its own, and its calls at their edges."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def net():
    from paper_2103_08802_gb300 import build
    build.build()
    from paper_2103_08802_gb300.seqnet import SeqNet
    return SeqNet(72, 64, 2, heads=16, seed=3)


def test_a_stream_of_its_own(net):
    """Tokens, parameters and states that are made late on a stream: forward, gradients and a step there follow them and
    give the bits of the default stream."""
    g = torch.Generator().manual_seed(4)
    x = torch.randint(0, 72, (3, 37), generator=g).int().cuda()
    ids = torch.stack([torch.randperm(72, generator=g)[:5] for _ in range(111)]).view(3, 37, 5).int().cuda()
    teacher = torch.randn(3, 37, 5, generator=g).cuda()

    def work(x, states):
        logits = net.forward(x)
        loss, grads = net.loss_and_grads(x, ids, teacher, labels=x, tau=2.0, alpha=0.5)
        return [logits, loss, net.step(x[:, 0].contiguous(), states), *states, *(grads[k] for k in sorted(grads))]

    start = [torch.randn(3, 64, generator=g).cuda() for _ in range(2)]
    want = work(x, [v.clone() for v in start])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        late, states = x + 0, [v.clone() for v in start]
        got = work(late, states)
    s.synchronize()
    assert all(torch.equal(a, e) for a, e in zip(got, want)) and len(got) == len(want)


def test_weights_of_tokens(net):
    """Weights in the tokens' shape weigh as their flat form does."""
    g = torch.Generator().manual_seed(5)
    x = torch.randint(0, 72, (2, 9), generator=g).int().cuda()
    w = torch.rand(2, 9, generator=g).cuda()
    a, b = (net.loss_and_grads(x, None, None, labels=x, weight=v, alpha=0.0) for v in (w, w.view(-1)))
    assert torch.equal(a[0], b[0]) and all(torch.equal(a[1][k], b[1][k]) for k in a[1])


def test_generation_of_nothing(net):
    """No steps give no tokens, an empty prompt is refused."""
    x = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    none = net.generate(x, 0)
    assert none.shape == (2, 0) and none.dtype == torch.int32
    with pytest.raises(ValueError):
        net.generate(x[:, :0], 3)

"""The token network that runs the sequence operators together: its gradients
against torch autograd of the same network, training, and generation token by
token against the scan."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def net_of():
    from paper_2103_08802_gb300 import build
    build.build()
    from paper_2103_08802_gb300.seqnet import SeqNet
    return SeqNet


def case(seed, b, t, vocab, k):
    g = torch.Generator().manual_seed(seed)
    x = torch.randint(0, vocab, (b, t), generator=g).int()
    x[0, 3] = -1
    ids = torch.stack([torch.randperm(vocab, generator=g)[:k] for _ in range(b * t)]).view(b, t, k).int()
    teacher, labels = torch.randn(b, t, k, generator=g) * 2, torch.randint(0, vocab, (b, t), generator=g).int()
    return [v.cuda() for v in (x, ids, teacher, labels)]


def autograd(net, x, ids, teacher, labels, lengths, tau, alpha):
    """The same network in torch, fp64 on values rounded to bf16 where the convolutions round theirs."""
    P = {k: v.double().requires_grad_() for k, v in net.params.items()}

    class Round(torch.autograd.Function):  # operands to bf16, forwards and backwards
        @staticmethod
        def forward(ctx, v):
            return v.bfloat16().double()

        @staticmethod
        def backward(ctx, g):
            return g

    def lin(h, name):
        return Round.apply(h) @ Round.apply(P[name]).t()

    b, t = x.shape
    live = (torch.arange(t, device="cuda") < lengths[:, None])[..., None]
    h = torch.where((x >= 0)[..., None], P["embed"][x.clamp(min=0).long()] * net.scale, 0.0)
    for i in range(net.layers):
        f = torch.sigmoid(lin(h, f"z{i}")).repeat_interleave(net.width // net.heads, -1)
        v, s, out = lin(h, f"x{i}"), torch.zeros(b, net.width, dtype=torch.float64, device="cuda"), []
        for j in range(t):
            s = torch.where(live[:, j], f[:, j] * s + (1 - f[:, j]) * v[:, j], s)
            out.append(torch.where(live[:, j], s, 0.0))
        h = h + lin(torch.stack(out, 1), f"o{i}")
    logits = lin(h, "out")
    p = torch.softmax(teacher.double() / tau, -1)
    lq = torch.log_softmax(logits / tau, -1).gather(-1, ids.long())
    loss = alpha * tau ** 2 * (p * (p.log() - lq)).sum(-1) - (1 - alpha) * torch.log_softmax(logits, -1).gather(-1, labels.long()[..., None])[..., 0]
    loss.mean().backward()
    return loss.detach().reshape(-1), {k: v.grad for k, v in P.items()}


@pytest.mark.parametrize("heads", [64, 8], ids=["own_gates", "shared_gates"])
def test_gradients_against_autograd(net_of, heads):
    """Both sides round the same operands to bf16 in the forward pass; the
    library's backward also rounds the gradients that its convolutions read (2^-9
    of each, at most five of them in a chain here), and values that land on the
    other side of a rounding boundary move by 2^-8: 2 % of the norm bounds both."""
    net = net_of(72, 64, 2, heads=heads, seed=3)
    x, ids, teacher, labels = case(4, 3, 37, 72, 5)
    lengths = torch.tensor([37, 20, 0], dtype=torch.int32, device="cuda")
    loss, grads = net.loss_and_grads(x, ids, teacher, labels=labels, tau=2.0, alpha=0.6, lengths=lengths)
    want, wg = autograd(net, x, ids, teacher, labels, lengths, 2.0, 0.6)
    assert ((loss.double() - want).norm() / want.norm()).item() <= 5e-3
    for k, g in grads.items():
        err = ((g.double() - wg[k]).norm() / wg[k].norm()).item()
        assert err <= 2e-2, (k, err)


def test_training_lowers_the_loss(net_of):
    """A student learns a fixed teacher's pairs: 200 steps on one batch at least halve the loss."""
    net = net_of(64, 64, 1, seed=5)
    x, ids, teacher, _ = case(6, 4, 32, 64, 4)
    losses = [net.train_step(0.2, x, ids, teacher, tau=1.0).mean().item() for _ in range(200)]
    assert losses[-1] <= 0.5 * losses[0], losses[::40]


def test_generation_follows_the_scan(net_of):
    """Logits token by token equal those of the whole sequence up to fp32
    reordering in the recurrence, and what it can move across bf16 rounding (1 %)."""
    net = net_of(80, 64, 2, heads=16, seed=7)
    x = case(8, 5, 19, 80, 2)[0].clamp(min=0)
    whole, states = net.forward(x), net.new_states(5)
    for t in range(19):
        one = net.step(x[:, t].contiguous(), states)
        assert ((one - whole[:, t]).norm() / whole[:, t].norm()).item() <= 1e-2
    assert net.generate(x, 3).shape == (5, 3)

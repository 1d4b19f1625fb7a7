"""The token network with linear attention, which runs attention, norms and the
policy loss together: its gradients against torch autograd of the same network,
training, and generation token by token against the prompt at once."""
import pytest
import torch

from test_gpu_seqnet import case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def net_of():
    from paper_2103_08802_gb300 import build
    build.build()
    from paper_2103_08802_gb300.seqnet import SeqNet
    return lambda *a, **kw: SeqNet(*a, mixer="attend", **kw)


class Round(torch.autograd.Function):
    """Operands to bf16, forwards; the gradient passes."""

    @staticmethod
    def forward(ctx, v):
        return v.bfloat16().double()

    @staticmethod
    def backward(ctx, g):
        return g


def unit(x):
    return x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt()


def logits_of(net, P, x, lengths):
    """The same network in torch, fp64 on values rounded to bf16 where the convolutions round theirs."""
    def lin(h, name):
        return Round.apply(h) @ Round.apply(P[name]).t()

    b, t = x.shape
    H, d = net.heads, net.head
    live = (torch.arange(t, device="cuda") < lengths[:, None])[..., None, None]
    h = torch.where((x >= 0)[..., None], P["embed"][x.clamp(min=0).long()] * net.scale, 0.0)
    n = unit(h) * P["pre0"]
    for i in range(net.layers):
        q, k, v, g = (lin(n, f"{m}{i}").view(b, t, H, d) for m in "qkvg")
        s, out = torch.zeros(b, H, d, d, dtype=torch.float64, device="cuda"), []
        for j in range(t):
            s = torch.where(live[:, j, :, :, None], net.decay.double()[:, None, None] * s + k[:, j, :, :, None] * v[:, j, :, None], s)
            out.append(torch.where(live[:, j], d ** -0.5 * torch.einsum("bhk,bhkv->bhv", q[:, j], s), 0.0))
        y = unit(torch.stack(out, 1)) * P[f"head{i}"] * torch.nn.functional.silu(g)
        h = h + P[f"res{i}"] * unit(lin(y.reshape(b, t, -1), f"o{i}")) * P[f"post{i}"]
        n = unit(h) * P[f"pre{i + 1}"]
    return lin(n, "out")


@pytest.mark.parametrize("heads", [1, 4], ids=["one_head", "heads"])
@pytest.mark.parametrize("loss", ["distill", "policy"])
def test_gradients_against_autograd(net_of, heads, loss):
    """The library's backward rounds the gradients that its convolutions read
    (2^-9 of each, at most five of them in a chain here), and values that land on
    the other side of a rounding boundary move by 2^-8: 2 % of the norm bounds both."""
    net = net_of(72, 64, 2, heads=heads, seed=3)
    x, ids, teacher, labels = case(4, 3, 37, 72, 5)
    lengths = torch.tensor([37, 20, 1], dtype=torch.int32, device="cuda")
    P = {k: v.double().requires_grad_() for k, v in net.params.items()}
    logits = logits_of(net, P, x, lengths)
    lp = torch.log_softmax(logits, -1).gather(-1, labels.long()[..., None])[..., 0]
    g = torch.Generator().manual_seed(1)
    adv = torch.randn(3, 37, generator=g).cuda()
    if loss == "distill":
        got, grads = net.loss_and_grads(x, ids, teacher, labels=labels, tau=2.0, alpha=0.6, lengths=lengths)
        p = torch.softmax(teacher.double() / 2, -1)
        lq = torch.log_softmax(logits / 2, -1).gather(-1, ids.long())
        want = 0.6 * 4 * (p * (p.log() - lq)).sum(-1) - 0.4 * lp
    else:
        # ratios of 0.7, 1 and 1.5 with a clip of 0.3 and 0.4: none near it
        move = torch.tensor([0.8, 1.0, 1.6]).log()[torch.randint(0, 3, (3, 37), generator=g)].cuda()
        old = (lp.detach() - move).float()
        ref = (lp.detach() + 0.3 * torch.randn(3, 37, generator=g).cuda()).float()
        got, logp, grads = net.policy_and_grads(x, labels, adv, old=old, ref=ref, clip=(0.3, 0.4), beta=0.2, lengths=lengths)
        assert ((logp.double() - lp.detach().reshape(-1)).norm() / lp.norm()).item() <= 5e-3
        r, u = torch.exp(lp - old.double()), ref.double() - lp
        want = -torch.minimum(r * adv, r.clamp(0.7, 1.4) * adv) + 0.2 * (torch.exp(u) - u - 1)
    want.mean().backward()
    assert ((got.double() - want.detach().reshape(-1)).norm() / want.norm()).item() <= 2e-2
    assert grads.keys() == P.keys()
    for k, v in grads.items():
        err = ((v.double() - P[k].grad).norm() / P[k].grad.norm()).item()
        assert err <= 2e-2, (k, err)


def test_generation_follows_the_prompt(net_of):
    """Logits token by token equal those of the whole sequence up to fp32
    reordering, and what it can move across bf16 rounding (1 %); the states behind
    a prompt are those that its steps leave."""
    net = net_of(80, 64, 2, heads=2, seed=7)
    x = case(8, 5, 19, 80, 2)[0].clamp(min=0)
    behind = []
    whole, states = net.forward(x, states=behind), net.new_states(5)
    for t in range(19):
        one = net.step(x[:, t].contiguous(), states)
        assert ((one - whole[:, t]).norm() / whole[:, t].norm()).item() <= 1e-2
    for a, b in zip(states, behind):
        assert ((a - b).norm() / b.norm()).item() <= 1e-2
    assert net.generate(x, 3).shape == (5, 3)
    assert net.generate(x, 0).shape == (5, 0)
    slots = torch.tensor([4, -1, 0], dtype=torch.int32, device="cuda")
    before = [s.clone() for s in states]
    net.step(x[:3, 0].contiguous(), states, slots=slots)
    for a, b in zip(states, before):
        assert torch.equal(a[1:4], b[1:4]) and not torch.equal(a[0], b[0]) and not torch.equal(a[4], b[4])


def test_steps_change_every_parameter(net_of):
    net = net_of(64, 64, 1, seed=5)
    x, ids, teacher, labels = case(6, 4, 32, 64, 4)
    for step in (lambda: net.train_step(0.1, x, ids, teacher), lambda: net.policy_step(0.1, x, labels, torch.ones(4, 32, device="cuda"))):
        before = {k: v.clone() for k, v in net.params.items()}
        step()
        for k, v in net.params.items():
            assert bool(torch.isfinite(v).all()) and not torch.equal(v, before[k]), k


def test_sizes_are_refused(net_of):
    for kw in (dict(heads=3), dict(heads=5)):
        with pytest.raises(ValueError):
            net_of(64, 64, 1, **kw)
    with pytest.raises(ValueError):
        net_of(64, 512, 1, heads=1)
    from paper_2103_08802_gb300.seqnet import SeqNet
    with pytest.raises(ValueError):
        SeqNet(64, 64, 1, mixer="other")

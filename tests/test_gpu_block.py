"""Linear attention, norms around a block and the policy loss on the GPU against
plain fp64 implementations (block_ref), at the sizes, types, strides and masks
where they can go wrong.  Bounds come from the arithmetic (block_ref); an
output in bf16 adds its one rounding, 2^-8 of the value."""
import math

import pytest
import torch

import block_ref as B
import seq_ref as R
from test_gpu_seq import held, randn

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
INF = math.inf


@pytest.fixture(scope="module")
def seq():
    from paper_2103_08802_gb300 import build
    build.build()
    from paper_2103_08802_gb300 import seq as S
    return S


def cuda(*ts):
    return [None if t is None else t.cuda() for t in ts]


def near(name, got, want, most):
    """Random signs: the error's norm against the result's."""
    got, want = got.detach().cpu().double(), want.double()
    if want.norm() == 0:
        assert got.norm() == 0, name
        return
    err = float((got - want).norm() / want.norm())
    assert err <= most, (name, err)


# ---------------------------------------------------------------- linear attention
def rows_of(g, b, t, h, d, dt):
    return randn(g, b, t, h, d, dtype=dt)


def decays(h):
    """Forgets at once, sees a token alone, keeps everything, and in between."""
    return torch.tensor(([0.97, 1.0, 0.0, 0.5, 0.999, 1e-30] * h)[:h])


ATTEND = [  # batch, time, heads, dk, dv, type, lengths
    (1, 1, 1, 1, 1, F32, None), (2, 5, 3, 8, 16, BF, None), (1, 33, 2, 20, 7, F32, None), (2, 64, 2, 64, 64, BF, None),
    (3, 127, 2, 64, 128, BF, [127, 0, 1]), (1, 300, 6, 128, 64, BF, None), (2, 129, 1, 128, 128, BF, [128, 129]),
    (1, 700, 2, 40, 72, F32, [533]), (1, 1031, 1, 64, 64, BF, [1029]), (2, 260, 2, 96, 80, BF, [0, 255]), (1, 130, 1, 256, 256, F32, None),
    (1, 200, 1, 200, 256, BF, None), (2, 90, 3, 33, 65, BF, [90, 40]), (1, 1600, 1, 128, 128, BF, None), (4, 257, 2, 72, 24, BF, [256, 257, 3, 0]),
    (1, 2100, 2, 16, 128, BF, [1700]), (1, 2100, 1, 64, 40, F32, [1700]), (6, 513, 40, 16, 16, BF, [513, 511, 256, 0, 1, 400]),
]


def attend_case(case, seed=1):
    b, t, h, dk, dv, dt, lengths = case
    g = torch.Generator().manual_seed(seed)
    q, k, v, do = (rows_of(g, b, t, h, d, dt) for d in (dk, dk, dv, dv))
    s0, ds = randn(g, b, h, dk, dv), randn(g, b, h, dk, dv)
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)
    return q, k, v, do, decays(h), s0, ds, ln


def hide(x, ln):
    """What lies behind a sequence must not be read: NaN there."""
    if ln is None:
        return x
    x = x.clone()
    for i, n in enumerate(ln.tolist()):
        x[i, max(n, 0):] = math.nan
    return x


@pytest.mark.parametrize("case", ATTEND, ids=str)
@pytest.mark.parametrize("state", [False, True], ids=["zero", "state"])
def test_attend(seq, case, state):
    q, k, v, do, a, s0, ds, ln = attend_case(case)
    if not state:
        s0 = ds = None
    scale = case[3] ** -0.5
    o, s = B.attend(q, k, v, a, s0, ln, scale)
    exact = (o, s) + B.attend_grad(q, k, v, a, do, s0, ds, ln, scale)
    bounds = B.attend_bounds(q, k, v, a, do, s0, ds, ln, scale)
    Q, K, V, D = cuda(*(hide(x, ln) for x in (q, k, v, do)))
    A, S0, DS, LN = cuda(a, s0, ds, ln)
    got = seq.attend(Q, K, V, A, s0=S0, lengths=LN, scale=scale) + seq.attend_grad(Q, K, V, A, D, s0=S0, ds_last=DS, lengths=LN, scale=scale)
    seq.sync()
    for name, x, want, bound in zip(("o", "s_last", "dq", "dk", "dv", "ds0"), got, exact, bounds):
        held(name, x, want, bound)
        state_ = name in ("s_last", "ds0")
        # random signs: the errors add up as the terms do.  bf16: one rounding inside, one of the output, of 2^-8 / sqrt(3)
        # of the value each at most in the mean; fp32 sums 2^-20
        near(name, x, want, R.U * 32 if state_ or case[5] == F32 else 2 ** -8)


def test_attend_of_padding_alone(seq):
    q, k, v, do, a, s0, ds, _ = attend_case((2, 40, 2, 64, 64, BF, None))
    ln = torch.tensor([0, -3], dtype=torch.int32)
    Q, K, V, D, A, S0, DS, LN = cuda(*(torch.full_like(x, math.nan) for x in (q, k, v, do)), a, s0, ds, ln)
    o, s = seq.attend(Q, K, V, A, s0=S0, lengths=LN)
    dq, dk, dv, ds0 = seq.attend_grad(Q, K, V, A, D, s0=S0, ds_last=DS, lengths=LN)
    assert torch.equal(s, S0) and torch.equal(ds0, DS)
    for x in (o, dq, dk, dv):
        assert bool((x == 0).all())


@pytest.mark.parametrize("dt", [BF, F32], ids=str)
def test_attend_strides(seq, dt):
    """q, k, v as slices of one packed projection, heads before time, one head for all, an offset that is not aligned;
    the output as a slice, what lies between its rows untouched."""
    g = torch.Generator().manual_seed(5)
    b, t, h, d = 2, 200, 3, 64
    packed = randn(g, b, t, 3, h, d, dtype=dt)
    q, k, v = packed.unbind(2)
    a = decays(h)
    base = seq.attend(*cuda(q.contiguous(), k.contiguous(), v.contiguous(), a))
    P = packed.cuda()
    A = a.cuda()
    exact, bounds = B.attend(q, k, v, a), B.attend_bounds(q, k, v, a)
    buf = torch.full((b, t, h, d + 8), 5.0, dtype=dt, device="cuda")
    o, s = seq.attend(*P.unbind(2), A, o=buf[..., :d])
    assert torch.equal(o, base[0]) and torch.equal(s, base[1]) and bool((buf[..., d:] == 5).all())
    turned = [x.transpose(1, 2).contiguous().cuda().transpose(1, 2) for x in (q, k, v)]
    o, s = seq.attend(*turned, A)
    assert torch.equal(o, base[0]) and torch.equal(s, base[1])
    for off in (1, 4):
        wide = [torch.zeros(b, t, h, d + 8, dtype=dt, device="cuda") for _ in range(3)]
        for w, x in zip(wide, (q, k, v)):
            w[..., off:off + d] = x.cuda()
        o, s = seq.attend(*(w[..., off:off + d] for w in wide), A)
        held("o", o, exact[0], bounds[0])
        held("s", s, exact[1], bounds[1])
    one = [x[:, :, :1].cuda().expand(b, t, h, d) for x in (k, v)]
    ks, vs = k[:, :, :1].expand(b, t, h, d), v[:, :, :1].expand(b, t, h, d)
    o, s = seq.attend(q.cuda(), *one, A)
    held("o", o, B.attend(q, ks, vs, a)[0], B.attend_bounds(q, ks, vs, a)[0])
    same = q[:1].cuda().expand(b, t, h, d)  # one sequence for all
    o, s = seq.attend(same, *cuda(k, v, a))
    held("o", o, B.attend(q[:1].expand(b, t, h, d), k, v, a)[0], B.attend_bounds(q[:1].expand(b, t, h, d), k, v, a)[0])


def test_attend_is_linear(seq):
    """o is linear in each of q, k, v, s0: differences of any size are its derivative, which the backward's products have to give."""
    q, k, v, do, a, s0, ds, _ = attend_case((1, 150, 2, 24, 40, F32, None))
    X = dict(zip(("q", "k", "v", "s0"), cuda(q, k, v, s0)))
    A, D, DS = cuda(a, do, ds)
    dq, dk, dv, ds0 = seq.attend_grad(X["q"], X["k"], X["v"], A, D, s0=X["s0"], ds_last=DS)
    f = lambda **kw: (lambda o, s: (o.double() * D.double()).sum() + (s.double() * DS.double()).sum())(  # noqa: E731
        *(lambda p: seq.attend(p["q"], p["k"], p["v"], A, s0=p["s0"]))({**X, **kw}))
    bo, bs, bq, bk, bv, b0 = B.attend_bounds(q, k, v, a, do, s0, ds)
    slack = float((bo * do.abs()).sum() + (bs * ds.abs()).sum())
    for name, grad, bound in (("q", dq, bq), ("k", dk, bk), ("v", dv, bv), ("s0", ds0, b0)):
        u = torch.randn(X[name].shape, generator=torch.Generator().manual_seed(3)).cuda()
        diff = (f(**{name: X[name] + u}) - f(**{name: X[name] - u})) / 2
        got = (grad.double() * u.double()).sum()
        # (x + u rounded: u of each argument; both sides within their bounds, of arguments up to 5 times as large)
        lim = 5 * slack + float((bound * u.cpu().abs()).sum()) + float((2 * R.U * (X[name].abs() + u.abs()).double() * grad.abs().double()).sum())
        assert abs(float(diff - got)) <= lim, (name, float(diff), float(got), lim)


STEP = [(1, 1, 1, 1, 1, F32), (3, 5, 2, 64, 64, BF), (7, 9, 3, 40, 72, F32), (40, 64, 16, 128, 128, BF), (2, 2, 1, 256, 256, BF), (5, 5, 2, 33, 19, BF)]


@pytest.mark.parametrize("case", STEP, ids=str)
def test_attend_step(seq, case):
    """One token on a pool: empty places, states nobody names untouched, and strided rows."""
    b, n, h, dk, dv, dt = case
    g = torch.Generator().manual_seed(2)
    wide = randn(g, b, h, 2 * dk + dv + 1, dtype=dt)
    q, k, v = wide[..., :dk], wide[..., dk:2 * dk], wide[..., 2 * dk:2 * dk + dv]
    pool, a = randn(g, n, h, dk, dv), decays(h)
    slots = torch.randperm(n, generator=g)[:b].int()
    if b > 2:
        slots[1] = -1
        slots[2] = n
    want, out = pool.double().clone(), torch.zeros(b, h, dv, dtype=torch.float64)
    bar, obar = pool.double().abs(), torch.zeros(b, h, dv, dtype=torch.float64)
    for i, s in enumerate(slots.tolist()):
        if 0 <= s < n:
            kv = k[i].double()[..., None] * v[i].double()[:, None]
            want[s] = a.double()[:, None, None] * want[s] + kv
            bar[s] = a.double()[:, None, None] * bar[s] + kv.abs()
            out[i] = 0.3 * torch.einsum("hk,hkv->hv", q[i].double(), want[s])
            obar[i] = 0.3 * torch.einsum("hk,hkv->hv", q[i].double().abs(), bar[s])
    W, P = wide.cuda(), pool.cuda()
    got = seq.attend_step(W[..., :dk], W[..., dk:2 * dk], W[..., 2 * dk:2 * dk + dv], a.cuda(), P, slots=slots.cuda(), scale=0.3)
    held("state", P, want, bar * 3 * R.U + R.TINY)
    held("o", got, out, obar * (dk + 8) * R.U + R.TINY)
    named = [s for s in slots.tolist() if 0 <= s < n]
    rest = [i for i in range(n) if i not in named]
    assert torch.equal(P.cpu()[rest], pool[rest])


def test_steps_follow_the_prompt(seq):
    """A prompt's state, continued token by token, is the whole sequence's: fp32 bounds of both sides."""
    q, k, v, _, a, s0, _, _ = attend_case((2, 90, 3, 32, 48, F32, None))
    Q, K, V, A = cuda(q, k, v, a)
    o, s = seq.attend(Q, K, V, A)
    _, state = seq.attend(Q[:, :80], K[:, :80], V[:, :80], A)
    bo, bs = B.attend_bounds(q, k, v, a)
    for i in range(80, 90):
        one = seq.attend_step(Q[:, i], K[:, i], V[:, i], A, state)
        held("o", one, o[:, i].cpu(), 2 * bo[:, i])
    held("s", state, s.cpu(), 2 * bs)


# ---------------------------------------------------------------- norms
NORM = [  # rows, width, x, res, weight, gate, vector scale, next
    (1, 1, F32, None, True, True, False, True), (3, 5, BF, F32, True, True, True, True), (100, 64, BF, None, True, True, False, False),
    (33, 128, BF, BF, True, False, True, True), (7, 1000, F32, F32, True, True, False, True), (5, 1001, BF, F32, False, True, True, True),
    (64, 258, BF, BF, True, True, True, True), (20, 2048, BF, F32, True, True, True, True), (9, 4100, F32, BF, True, False, False, True),
    (3, 8192, BF, BF, True, True, True, True), (2, 8200, BF, F32, True, True, True, True), (3, 16383, F32, F32, True, True, True, True),
    (1000, 24, F32, None, True, False, True, False), (300, 40, BF, F32, False, False, False, True), (5000, 16, BF, BF, True, True, True, True),
    (700, 512, BF, None, False, True, True, False), (2, 2050, F32, None, True, True, True, True),
    (20000, 33, BF, F32, True, True, True, True), (10007, 35, F32, BF, True, False, True, False), (1301, 1001, BF, BF, True, True, True, True),
    (1300, 1002, BF, F32, True, True, True, True), (310, 4101, BF, BF, True, True, True, True), (170, 8180, BF, F32, True, True, False, True),
    (40, 8187, F32, F32, True, False, True, True),
]


def norm_case(case, seed=3):
    r, w, dx, dr, post, gated, vector, nxt = case
    g = torch.Generator().manual_seed(seed)
    x = randn(g, r, w, dtype=dx)
    kw = dict(weight=1 + 0.3 * randn(g, w) if post else None, gate=2 * randn(g, r, w, dtype=dx) if gated else None,
              scale=0.5 + 0.2 * randn(g, w) if vector else -0.7, res=2 * randn(g, r, w, dtype=dr) if dr else None,
              next_weight=1 + 0.3 * randn(g, w) if nxt else None)
    dh, dn = randn(g, r, w, dtype=dr or dx), randn(g, r, w, dtype=dx) if nxt else None
    return x, kw, dh, dn


def on_gpu(kw):
    return {k: v.cuda() if torch.is_tensor(v) else v for k, v in kw.items()}


@pytest.mark.parametrize("case", NORM, ids=str)
def test_norm(seq, case):
    x, kw, dh, dn = norm_case(case)
    f64 = {k: v.double() if torch.is_tensor(v) else v for k, v in kw.items()}
    h, n = B.norm(x.double(), **f64)
    want = B.norm_grad(x, dh, dn, **kw)
    bounds = B.norm_bounds(x, dh, dn, **kw)
    got = seq.norm(x.cuda(), **on_gpu(kw))
    held("h", got[0], h, bounds["h"])
    assert (got[1] is None) == (n is None)
    if n is not None:
        held("n", got[1], n, bounds["n"])
    g = seq.norm_grad(x.cuda(), *cuda(dh, dn), **on_gpu(kw))
    for name, v in g._asdict().items():
        assert (v is None) == (name != "x" and not torch.is_tensor(kw[name])), name
        if v is not None:
            held(name, v, want[name], bounds[name])
    if case[7]:  # h goes nowhere but into the norm
        g = seq.norm_grad(x.cuda(), None, dn.cuda(), **on_gpu(kw))
        want, bounds = B.norm_grad(x, None, dn, **kw), B.norm_bounds(x, None, dn, **kw)
        for name, v in g._asdict().items():
            if v is not None:
                held(name, v, want[name], bounds[name])


def test_norm_shapes_rows_and_strides(seq):
    """Leading axes of any number, slices of wider buffers (aligned and not), no rows, zero rows and large eps."""
    g = torch.Generator().manual_seed(1)
    x, gate, w = randn(g, 6, 50, 128, dtype=BF).cuda(), randn(g, 6, 50, 128, dtype=BF).cuda(), torch.ones(128, device="cuda")
    base = seq.norm(x.view(300, 128), weight=w, gate=gate.view(300, 128))[0]
    assert torch.equal(seq.norm(x, weight=w, gate=gate)[0].view(300, 128), base)
    turned = x.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(seq.norm(turned, weight=w, gate=gate)[0].view(300, 128), base)
    for off in (1, 8):
        wide = torch.zeros(300, 140, dtype=BF, device="cuda")
        wide[:, off:off + 128] = x.view(300, 128)
        part = wide[:, off:off + 128]
        h, _ = seq.norm(part, weight=w, gate=gate.view(300, 128))
        ref, bound = B.norm(part.cpu().double(), weight=w.cpu().double(), gate=gate.view(300, 128).cpu().double()), B.norm_bounds(
            part.cpu(), weight=w.cpu(), gate=gate.view(300, 128).cpu())
        held("h", h, ref[0], bound["h"])
    one = torch.randn(128, generator=g).cuda()
    assert seq.norm(one, weight=w)[0].shape == (128,)
    none = seq.norm_grad(x[:0], x[:0], weight=w, gate=gate[:0])
    assert none.x.shape == (0, 50, 128) and bool((none.weight == 0).all())
    assert seq.norm(x[:0], weight=w)[0].shape == (0, 50, 128)
    z = torch.zeros(4, 128, device="cuda")
    h, n = seq.norm(z, weight=w, next_weight=w)
    assert bool((h == 0).all()) and bool((n == 0).all())
    d = seq.norm_grad(z, z + 1, z + 1, weight=w, next_weight=w, eps=0.25)
    # at zero both norms have the slope 1 / sqrt(eps) = 2: D = 1 + 2, dx = 2 D
    assert torch.allclose(d.x, torch.full_like(z, 6.0), rtol=1e-5)


def test_norm_gradient_against_differences(seq):
    """A direction's derivative against differences of the fp32 forward: off by what the same differences are off in
    fp64, and by the forward's own error over the step."""
    x, kw, dh, dn = norm_case((6, 96, F32, F32, True, True, True, True))
    g = seq.norm_grad(x.cuda(), *cuda(dh, dn), **on_gpu(kw))
    step = 2.0 ** -6
    args = {"x": x, **kw}
    bound = B.norm_bounds(x, **kw)
    err = float((bound["h"] * dh.abs() * 2 + bound["n"] * dn.abs() * 2).sum()) + R.U * float((B.norm(x.double(), **{k: v.double() for k, v in kw.items()})[0] * dh).abs().sum() * 4)
    for name, t in args.items():
        u = torch.randn(t.shape, generator=torch.Generator().manual_seed(8)) * t.abs().clamp(min=0.1)

        def f(sign, call, conv):
            a = {**args, name: t + sign * step * u}
            h, n = call(**{k: conv(v) for k, v in a.items()})
            return float((h.double().cpu() * dh).sum() + (n.double().cpu() * dn).sum())
        diff = (f(1, seq.norm, lambda v: v.cuda()) - f(-1, seq.norm, lambda v: v.cuda())) / (2 * step)
        exact = (f(1, B.norm, lambda v: v.double()) - f(-1, B.norm, lambda v: v.double())) / (2 * step)
        want = float((B.norm_grad(x, dh, dn, **kw)[name] * u.double()).sum())
        got = float((getattr(g, name).cpu().double() * u.double()).sum())
        assert abs(got - diff) <= abs(exact - want) + err / step + 1e-4 * abs(want), (name, got, diff, exact, want)


# ---------------------------------------------------------------- policy loss
POLICY = [  # rows, vocab, type, tau, old, ref, weight
    (1, 1, F32, 1.0, True, True, True), (5, 7, BF, 1.0, True, False, True), (9, 33, F32, 0.7, False, True, False), (6, 1000, F32, 1.0, True, True, True),
    (5, 2049, BF, 1.3, True, True, True), (3, 8193, F32, 1.0, True, True, False), (4, 9217, BF, 1.0, True, False, True), (3, 21505, BF, 2.0, True, True, True),
    (3, 40001, BF, 1.0, True, True, True), (2, 60000, F32, 1.0, False, False, True), (700, 130, BF, 1.0, True, True, True),
]


def policy_case(case, seed=4):
    r, v, dt, tau, has_old, has_ref, has_weight = case
    g = torch.Generator().manual_seed(seed)
    logits = (2 * randn(g, r, v)).to(dt)
    labels = torch.randint(0, v, (r,), generator=g).int()
    if v > 20:
        logits[:, v - v // 16:] = -INF
        labels = labels.clamp(max=v - v // 16 - 1)
    lp = torch.log_softmax(logits.double() / tau, 1).gather(1, labels.long()[:, None])[:, 0]
    d = 0.2 * randn(g, r).double()
    for edge in (math.log(0.9), math.log(1.3)):  # not on the border, where a rounding decides
        d = torch.where((d - edge).abs() < 1e-3, d + 4e-3, d)
    old = (lp - d).float() if has_old else None
    ref = (lp + 0.4 * randn(g, r).double()).float() if has_ref else None
    if r > 4:
        labels[1], labels[2] = -1, v
        if v > 20:
            labels[3] = v - 1  # masked
            logits[4] = -INF
    kw = dict(old=old, ref=ref, weight=torch.rand(r, generator=g) if has_weight else None, clip=(0.1, 0.3), beta=0.1 if has_ref else 0.0, tau=tau)
    return logits, labels, randn(g, r), kw


@pytest.mark.parametrize("case", POLICY, ids=str)
def test_policy(seq, case):
    logits, labels, adv, kw = policy_case(case)
    want, bounds = B.policy(logits, labels, adv, **kw)
    got = seq.policy(*cuda(logits, labels, adv), **on_gpu(kw))
    for name, x, w, b in zip(("loss", "logp", "dlogits"), got, want, bounds):
        held(name, x, w, b)
    alone = seq.policy(*cuda(logits, labels, adv), grad=False, **on_gpu(kw))
    assert alone[2] is None
    for name, x, w, b in zip(("loss", "logp"), alone, want, bounds):
        held(name, x, w, b)
    place = logits.cuda()  # the gradient in the logits' place
    inplace = seq.policy(place, *cuda(labels, adv), out=place, **on_gpu(kw))
    assert torch.equal(inplace[2], got[2]) and torch.equal(inplace[0], got[0])
    wide = torch.full((case[0], case[1] + 9), 7.0, dtype=case[2], device="cuda")
    wide[:, 3:3 + case[1]] = logits.cuda()
    off = seq.policy(wide[:, 3:3 + case[1]], *cuda(labels, adv), out=wide[:, 3:3 + case[1]], **on_gpu(kw))
    held("dlogits", off[2], want[2], bounds[2])
    assert bool((wide[:, :3] == 7).all()) and bool((wide[:, 3 + case[1]:] == 7).all())
    seq.sync()


def test_policy_at_the_clip(seq):
    """Ratios far inside, beyond either bound, of either sign; on the border the gradient holds."""
    logits = torch.tensor([[0.0, 0.0]] * 8)
    lp = math.log(0.5)
    ratio = torch.tensor([1.0, 2.0, 2.0, 0.25, 0.25, 1.0, 1.0, 1e9], dtype=torch.float64)
    adv = torch.tensor([1.0, 1.0, -1.0, 1.0, -1.0, 0.0, 1.0, 0.0])
    old = (lp - ratio.log()).float()
    loss, logp, d = seq.policy(*cuda(logits, torch.zeros(8).int(), adv), old=old.cuda(), clip=(0.5, 0.5))
    assert torch.allclose(logp.cpu(), torch.full((8,), lp))
    assert torch.allclose(loss.cpu(), torch.tensor([-1.0, -1.5, 2.0, -0.25, 0.5, 0.0, -1.0, 0.0]))
    slope = torch.tensor([-1.0, 0.0, 2.0, -0.25, 0.0, 0.0, -1.0, 0.0])
    assert torch.allclose(d.cpu(), slope[:, None] * torch.tensor([0.5, -0.5]))
    # the ratio is 1 exactly, and the clip lets nothing else through
    _, _, d = seq.policy(*cuda(logits[:1], torch.zeros(1).int(), adv[:1]), clip=(0.0, 0.0))
    assert torch.allclose(d.cpu(), torch.tensor([[-0.5, 0.5]]))
    loss, _, _ = seq.policy(*cuda(logits[:2], torch.zeros(2).int(), adv[:2]), old=old[:2].cuda(), clip=(1.0, INF))
    assert torch.allclose(loss.cpu(), torch.tensor([-1.0, -2.0]))


def test_policy_gradient_against_differences(seq):
    logits, labels, adv, kw = policy_case((6, 50, F32, 0.7, True, True, True))
    want, (bl, _, bd) = B.policy(logits, labels, adv, **kw)
    _, _, d = seq.policy(*cuda(logits, labels, adv), **on_gpu(kw))
    u = torch.randn(logits.shape, generator=torch.Generator().manual_seed(9))
    step = 2.0 ** -9
    w = kw["weight"].double()
    live = torch.isfinite(logits[:, 0]) & (labels >= 0) & (labels < 50) & (labels < 47)

    def f(sign, exact):
        x = logits + sign * step * u
        loss = B.policy(x, labels, adv, **kw)[0][0] if exact else seq.policy(*cuda(x, labels, adv), grad=False, **on_gpu(kw))[0].cpu().double()
        return loss * w
    diff, exact = (f(1, False) - f(-1, False)) / (2 * step), (f(1, True) - f(-1, True)) / (2 * step)
    finite = torch.isfinite(logits)
    got = torch.where(finite, d.cpu().double() * u, 0.0).sum(1)
    ref = torch.where(finite, want[2] * u, 0.0).sum(1)
    lim = (exact - ref).abs() + 3 * bl * w / step + torch.where(finite, bd * u.abs(), 0.0).sum(1) + R.U * 8
    assert bool(((got - diff).abs() <= lim)[live].all()), (got, diff, exact, lim)


# ---------------------------------------------------------------- streams, graphs
def test_block_calls_in_a_graph_and_on_a_stream(seq):
    """Every call captured together and replayed, on new values in the same buffers, beside the same calls on another stream."""
    q, k, v, do, a, s0, ds, ln = cuda(*attend_case((2, 700, 2, 64, 64, BF, [700, 300])))
    x, kw, dh, dn = norm_case((64, 256, BF, F32, True, True, True, True))
    x, dh, dn, kw = x.cuda(), dh.cuda(), dn.cuda(), on_gpu(kw)
    logits, labels, adv, pk = policy_case((6, 9000, BF, 1.0, True, True, True))
    logits, labels, adv, pk = logits.cuda(), labels.cuda(), adv.cuda(), on_gpu(pk)
    pool = randn(torch.Generator().manual_seed(1), 3, 2, 64, 64).cuda()

    def calls(stream=None):
        m = dict(stream=stream)
        return [*seq.attend(q, k, v, a, s0=s0, lengths=ln, **m), *seq.attend_grad(q, k, v, a, do, s0=s0, ds_last=ds, lengths=ln, **m),
                seq.attend_step(q[:, 0], k[:, 0], v[:, 0], a, pool, **m), *seq.norm(x, **kw, **m),
                *seq.norm_grad(x, dh, dn, **kw, **m), *seq.policy(logits, labels, adv, **pk, **m)]

    start = pool.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    first = [t.clone() for t in calls()]
    torch.cuda.synchronize()
    pool.copy_(start)
    torch.cuda.synchronize()
    other = calls(side)
    side.synchronize()
    for i, (p, r) in enumerate(zip(first, other)):
        assert torch.equal(p, r), i
    pool.copy_(start)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = calls()
    pool.copy_(start)
    graph.replay()
    torch.cuda.synchronize()
    for i, (p, r) in enumerate(zip(first, outs)):
        assert torch.equal(p, r), i
    q.mul_(2)
    pool.copy_(start)
    graph.replay()
    again = [t.clone() for t in outs]
    pool.copy_(start)
    for i, (p, r) in enumerate(zip(calls(), again)):
        assert torch.equal(p, r), i
    seq.sync()


def test_offsets_beyond_32_bits(seq):
    """Sequences and rows 2^31 values apart, and the last axis of time far behind the first: bit for bit what contiguous ones give."""
    big = torch.empty(2 ** 32 + 2 ** 20, dtype=BF, device="cuda")
    g = torch.Generator().manual_seed(6)
    for shape, stride in (((2, 70, 2, 64), (2 ** 31, 128, 64, 1)), ((1, 3, 1, 64), (64, 2 ** 31, 64, 1)), ((2, 70, 2, 50), (2 ** 31, 102, 50, 1))):
        q = randn(g, *shape, dtype=BF).cuda()
        far, out = big.as_strided(shape, stride), big.as_strided(shape, stride, 2 ** 19)
        far.copy_(q)
        a = torch.full((shape[2],), 0.9, device="cuda")
        for k in (1, 2):  # (as q alone, and as all three)
            o, s = seq.attend(far, far if k == 2 else q, far if k == 2 else q, a, o=out)
            want = seq.attend(q, q, q, a)
            if shape[3] == 64:
                assert torch.equal(o, want[0]) and torch.equal(s, want[1])
            near("o", o, want[0].cpu(), 2 ** -8)
            near("s", s, want[1].cpu(), 1e-6)
        grads = seq.attend_grad(far, far, far, a, far)
        for x, y in zip(grads, seq.attend_grad(q, q, q, a, q)):
            near("grad", x, y.cpu(), 2 ** -8)
    x = randn(g, 2, 200, dtype=BF).cuda()
    far = big.as_strided((2, 200), (2 ** 31, 1))
    far.copy_(x)
    w = torch.ones(200, device="cuda")
    h, n = seq.norm(far, weight=w, res=far, next_weight=w)
    want = seq.norm(x, weight=w, res=x, next_weight=w)
    assert torch.equal(h, want[0]) and torch.equal(n, want[1])
    for p, r in zip(seq.norm_grad(far, far, far, weight=w, res=far, next_weight=w), seq.norm_grad(x, x, x, weight=w, res=x, next_weight=w)):
        assert (p is None) == (r is None) and (p is None or torch.equal(p, r))
    label, adv = torch.tensor([3, 7], dtype=torch.int32, device="cuda"), torch.ones(2, device="cuda")
    out = big.as_strided((2, 200), (2 ** 31, 1), 2 ** 19)
    for p, r in zip(seq.policy(far, label, adv, out=out), seq.policy(x, label, adv)):
        assert torch.equal(p, r)
    seq.sync()


@pytest.mark.parametrize("a", [0.79, 0.81, 0.9, 0.1, 1.0])
def test_decays_on_either_side_of_the_row_scale(seq, a):
    """Decays whose 128th power is far below or above what one accumulator holds, over several chunks with a partial one."""
    q, k, v, do, _, s0, ds, _ = attend_case((2, 300, 1, 64, 128, BF, None), seed=9)
    dec, ln = torch.tensor([a]), torch.tensor([300, 131], dtype=torch.int32)
    o, s = B.attend(q, k, v, dec, s0, ln, 0.125)
    exact = (o, s) + B.attend_grad(q, k, v, dec, do, s0, ds, ln, 0.125)
    Q, K, V, D, A, S0, DS, LN = cuda(q, k, v, do, dec, s0, ds, ln)
    got = seq.attend(Q, K, V, A, s0=S0, lengths=LN, scale=0.125) + seq.attend_grad(Q, K, V, A, D, s0=S0, ds_last=DS, lengths=LN, scale=0.125)
    for name, x, want, bound in zip(("o", "s_last", "dq", "dk", "dv", "ds0"), got, exact, B.attend_bounds(q, k, v, dec, do, s0, ds, ln, 0.125)):
        held(name, x, want, bound)
        near(name, x, want, R.U * 32 if name in ("s_last", "ds0") else 2 ** -8)


@pytest.mark.parametrize("case", [(5, 1531, 7, 40, 72, F32), (1, 256, 1, 64, 64, F32), (1, 1500, 2, 256, 256, F32), (3, 1000, 8, 33, 65, BF), (1, 2048, 4, 64, 64, BF)], ids=str)
def test_workspace_does_not_depend_on_lengths(seq, case):
    """Lengths may be given after the workspace was asked for; results with full lengths are those without."""
    q, k, v, do, a, s0, ds, _ = attend_case((*case, None))
    ln = torch.full((case[0],), case[1], dtype=torch.int32)
    Q, K, V, D, A, S0, DS, LN = cuda(q, k, v, do, a, s0, ds, ln)
    lib = seq.load()
    for back in (0, 1):
        size = []
        for lengths in (None, LN):
            args = seq._attend_args(Q, K, V, A, S0, lengths, 1.0, Q.get_device())
            n = seq.C.c_size_t()
            assert lib.pnn_attend_workspace_bytes(seq.C.byref(args), back, seq.C.byref(n)) == 0
            size.append(n.value)
        assert size[0] == size[1]
    plain = seq.attend(Q, K, V, A, s0=S0) + seq.attend_grad(Q, K, V, A, D, s0=S0, ds_last=DS)
    given = seq.attend(Q, K, V, A, s0=S0, lengths=LN) + seq.attend_grad(Q, K, V, A, D, s0=S0, ds_last=DS, lengths=LN)
    bounds = B.attend_bounds(q, k, v, a, do, s0, ds)
    for name, x, y, bound in zip(("o", "s_last", "dq", "dk", "dv", "ds0"), given, plain, bounds):
        held(name, x, y.cpu().double(), 2 * bound + (2 * 2.0 ** -8 * y.cpu().double().abs() if y.dtype == BF else 0))


@pytest.mark.parametrize("case", [(1, 7, 4, 128, 128), (1, 1, 1, 64, 64), (2, 32, 2, 64, 128), (1, 29, 2, 128, 64), (2, 150, 1, 33, 65), (1, 90, 2, 200, 256)], ids=str)
def test_few_tokens_and_odd_heads_are_rounded_once(seq, case):
    """bf16 outputs there: their own rounding, of 2^-8 of the value at most and evenly spread, is 2^-8 / sqrt(3) of the norm; what was
    kept to 16 bits on the way adds 2^-15 a term."""
    q, k, v, do, a, s0, ds, _ = attend_case((*case, BF, None))
    exact = (B.attend(q, k, v, a, s0)[0],) + B.attend_grad(q, k, v, a, do, s0, ds)[:3]
    Q, K, V, D, A, S0, DS = cuda(q, k, v, do, a, s0, ds)
    got = (seq.attend(Q, K, V, A, s0=S0)[0],) + seq.attend_grad(Q, K, V, A, D, s0=S0, ds_last=DS)[:3]
    for name, x, want in zip(("o", "dq", "dk", "dv"), got, exact):
        near(name, x, want, 2 ** -8 / math.sqrt(3))

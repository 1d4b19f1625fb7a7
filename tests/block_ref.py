"""Plain fp64 implementations (torch, CPU) of the linear attention, the norms
around a block and the policy loss, and the error bounds their kernels are held
to.  u = 2^-24 (one fp32 rounding); a rounding to bf16 is at most 2^-8 of the value."""
import math

import torch

from seq_ref import TINY, U, ULP

BF = 2.0 ** -8


# ---------------------------------------------------------------- linear attention
def attend(q, k, v, decay, s0=None, lengths=None, scale=1.0):
    """(o, s_last), token by token."""
    b, t, h, dk = q.shape
    q, k, v, a = q.double(), k.double(), v.double(), decay.double()[:, None, None]
    n = torch.full((b,), t) if lengths is None else lengths.clamp(0, t).long()
    s = torch.zeros(b, h, dk, v.shape[3], dtype=torch.float64) if s0 is None else s0.double()
    o = torch.zeros_like(v)
    for i in range(t):
        on = (i < n)[:, None, None, None]
        s = torch.where(on, a * s + k[:, i, :, :, None] * v[:, i, :, None], s)
        o[:, i] = torch.where(on[..., 0], scale * torch.einsum("bhk,bhkv->bhv", q[:, i], s), 0.0)
    return o, s


def attend_grad(q, k, v, decay, do, s0=None, ds_last=None, lengths=None, scale=1.0):
    """(dq, dk, dv, ds0), token by token."""
    b, t, h, dk = q.shape
    q, k, v, do, a = q.double(), k.double(), v.double(), do.double(), decay.double()[:, None, None]
    n = torch.full((b,), t) if lengths is None else lengths.clamp(0, t).long()
    s = torch.zeros(b, h, dk, v.shape[3], dtype=torch.float64) if s0 is None else s0.double()
    g = torch.zeros_like(s) if ds_last is None else ds_last.double()
    dq, dk_, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for i in range(t):
        on = (i < n)[:, None, None, None]
        s = torch.where(on, a * s + k[:, i, :, :, None] * v[:, i, :, None], s)
        dq[:, i] = torch.where(on[..., 0], scale * torch.einsum("bhv,bhkv->bhk", do[:, i], s), 0.0)
    for i in range(t - 1, -1, -1):
        on = (i < n)[:, None, None, None]
        here = g + scale * q[:, i, :, :, None] * do[:, i, :, None]
        dk_[:, i] = torch.where(on[..., 0], torch.einsum("bhv,bhkv->bhk", v[:, i], here), 0.0)
        dv[:, i] = torch.where(on[..., 0], torch.einsum("bhk,bhkv->bhv", k[:, i], here), 0.0)
        g = torch.where(on, a * here, g)
    return dq, dk_, dv, g


def attend_bounds(q, k, v, decay, do=None, s0=None, ds_last=None, lengths=None, scale=1.0):
    """Bounds of (o, s_last[, dq, dk, dv, ds0]) before the outputs' own rounding.

    An output is a sum of products a^n x y z.  Its magnitude is that of the same
    formula on absolute values, and the error relative to it: the powers 4 u;
    operands as two tf32 numbers 2^-22 each, or as three bf16 numbers u; sums over
    the width and over a piece of 128 tokens at most, on an adder that may cut
    off instead of rounding (2 u an addition); a state is scaled and added to once
    every 32 tokens (2 u each).  bf16 rows: the scores, or the state, rounded to
    bf16 on their way into an output.  A state has none of that."""
    dk, dv, t = q.shape[3], v.shape[3], q.shape[1]
    m = lambda x: None if x is None else x.abs()  # noqa: E731
    c = (2 * 128 + 2 * (t / 32 + 1) + 32) * U
    out = (2 * max(dk, dv)) * U + c + (2 * BF if q.dtype == torch.bfloat16 else 0.0)
    o, s = attend(m(q), m(k), m(v), decay, m(s0), lengths, abs(scale))
    r = [o * out + TINY, s * c + TINY]
    if do is not None:
        g = attend_grad(m(q), m(k), m(v), decay, m(do), m(s0), m(ds_last), lengths, abs(scale))
        r += [x * out + TINY for x in g[:3]] + [g[3] * c + TINY]
    return r


# ---------------------------------------------------------------- norms
def norm(x, weight=None, gate=None, scale=1.0, res=None, next_weight=None, eps=1e-6):
    """(h, n) in fp64; differentiable."""
    unit = lambda v: v / (v.square().mean(-1, keepdim=True) + eps).sqrt()  # noqa: E731
    y = x if weight is None else unit(x) * weight
    if gate is not None:
        y = y * gate * torch.sigmoid(gate)
    h = y * scale if res is None else res + y * scale
    return h, None if next_weight is None else unit(h) * next_weight


def norm_grad(x, dh, dn=None, **kw):
    """Gradients of norm's tensor arguments by autograd, {name: gradient}."""
    v = {"x": x, **{k: t for k, t in kw.items() if k != "eps"}}
    v = {k: t.double().requires_grad_() if torch.is_tensor(t) else t for k, t in v.items()}
    h, n = norm(eps=kw.get("eps", 1e-6), **v)
    total = 0.0 if dh is None else (h * dh.double()).sum()
    if n is not None:
        total = total + (n * dn.double()).sum()
    names = [k for k, t in v.items() if torch.is_tensor(t)]
    return dict(zip(names, torch.autograd.grad(total, [v[k] for k in names], allow_unused=True)))


def norm_bounds(x, dh=None, dn=None, weight=None, gate=None, scale=1.0, res=None, next_weight=None, eps=1e-6):
    """{name: bound} of h, n and the gradients.

    The relative error of one product along any path: a mean of squares is a sum
    of 16 values a thread, of a warp and of 32 warps (26 roundings at most; half of that
    in the root), 2 ulp the root, the gate's exponential 2 + 1.16 |g| ulp, division 2
    ulp, and a dozen products and sums: e.  h carries e of |res| + |s y|, which
    against h itself is larger where the two cancel: n and all that the second
    norm gives back carry k e, k = the row's (mean hbar^2 / mean h^2)^(1/2), three
    times over (rh, its cube, h).  Gradients are bounded by e or 4 k e of their formula with
    every term taken by its absolute value; a column's sum over the rows adds a
    rounding for every row of a thread's, and 64."""
    f = lambda v: v.double() if torch.is_tensor(v) else v  # noqa: E731
    x, dh, dn, weight, gate, scale, res, w2 = map(f, (x, dh, dn, weight, gate, scale, res, next_weight))
    rows = x.shape[0]
    e = 64 * U + (0.0 if gate is None else (4 + 2 * 1.16 * gate.abs().clamp(max=90.0)) * ULP)
    one = torch.ones(())
    w = one if weight is None else weight.abs()
    rx = torch.ones(rows, 1, dtype=torch.float64) if weight is None else (x.square().mean(1, keepdim=True) + eps).rsqrt()
    act = one if gate is None else (gate * torch.sigmoid(gate)).abs()
    s = scale.abs() if torch.is_tensor(scale) else torch.tensor(abs(scale))
    y = (x * rx).abs() * w
    bar = y * act * s + (0.0 if res is None else res.abs())
    h, n = norm(x, weight, gate, scale, res, w2, eps)
    out = {"h": bar * e + TINY}
    k = 1.0
    if w2 is not None:
        ms = h.square().mean(1, keepdim=True) + eps
        k = (1.0 + (bar.square().mean(1, keepdim=True) / ms)).sqrt()
        rh = ms.rsqrt()
        out["n"] = rh * w2.abs() * bar * e * k * 2 + TINY
    if dh is None and dn is None:
        return out
    D = torch.zeros_like(x) if dh is None else dh.abs()
    if w2 is not None:
        d = (dn * w2).abs()
        D = D + rh * (d + bar * rh ** 2 * (d * bar).mean(1, keepdim=True))
    emax = (e if torch.is_tensor(e) else torch.full_like(x, e)).amax(1, keepdim=True)
    c = 4 * k * emax
    many = (rows + 64) * U
    out["res"] = D * c + TINY
    q = D * s
    out["scale"] = (D * act * y * (c + many)).sum(0) + TINY
    if gate is not None:
        sg = torch.sigmoid(gate)
        out["gate"] = q * y * (sg * (1 + gate.abs() * (1 - sg))) * c * 2 + TINY
    q = q * act
    xw = (x * rx).abs()
    out["weight"] = (q * xw * (c + many)).sum(0) + TINY
    if weight is None:
        out["x"] = q * c + TINY
    else:
        out["x"] = rx * (q * w + xw * (q * w * xw).mean(1, keepdim=True)) * c + TINY
    if w2 is not None:
        out["next_weight"] = (dn.abs() * rh * bar * (c + many)).sum(0) + TINY
    return out


# ---------------------------------------------------------------- policy loss
def policy(logits, labels, advantage, old=None, ref=None, weight=None, clip=(0.2, 0.2), beta=0.0, tau=1.0):
    """(loss, logp, dlogits) and their bounds, row by row, in fp64.

    An exponent carries 4 u of itself, its exponential (2 + 1.16 |y|) ulp, a row's
    sum chains of at most V / 32 + 64 roundings; the logarithm 1 ulp.  The
    ratio's relative error is that of lp - old, absolute, and 2 ulp of its exponential."""
    r, v = logits.shape
    f64 = lambda *s: torch.zeros(*s, dtype=torch.float64)  # noqa: E731
    loss, logp, d = f64(r), f64(r), f64(r, v)
    bl, bp, bd = f64(r) + TINY, f64(r) + TINY, f64(r, v) + TINY
    for i in range(r):
        a = int(labels[i])
        if not 0 <= a < v:
            continue
        s = logits[i].double() / tau
        if s[a] == -math.inf:
            logp[i] = -math.inf
            continue
        m = s.max()
        y = s - m
        e = torch.exp(y)
        p, mag = e / e.sum(), torch.where(e > 0, y.abs(), 0.0)
        each = (3 + 1.16 * mag) * ULP + 4 * U * mag
        total = float((p * each).sum()) + (v / 32 + 64) * U
        lp = float(y[a] - e.sum().log())
        elp = total + 4 * U * (1 + float(mag[a])) + 4 * U * float(e.sum().log())
        A, w = float(advantage[i]), 1.0 if weight is None else float(weight[i])
        gap = 0.0 if old is None else lp - float(old[i])
        ratio = math.exp(gap)
        er = 0.0 if old is None else elp + abs(gap) * U + 2 * ULP
        lo, hi = 1 - clip[0], 1 + clip[1]
        held = min(ratio, hi) if A > 0 else max(ratio, lo)
        slope = -A * ratio if held == ratio else 0.0
        loss[i], bl[i] = -A * held, bl[i] + abs(A) * held * (er + 4 * U)
        es = abs(slope) * (er + 4 * U)
        if ref is not None and beta:
            u = float(ref[i]) - lp
            k = math.expm1(u)
            eu = elp + 2 * U * abs(u)
            loss[i] += beta * (k - u)
            bl[i] += beta * (abs(k) * eu + (abs(k) + 2 * abs(u)) * 2 * ULP) + U * abs(float(loss[i]))
            slope -= beta * k
            es += beta * (math.exp(u) * eu + abs(k) * 2 * ULP + 2 * U * abs(k))
        logp[i], bp[i] = lp, bp[i] + elp
        hot = f64(v)
        hot[a] = 1.0
        c = w / tau * slope
        d[i] = c * (hot - p)
        bd[i] += abs(w) / tau * (es + 4 * U * abs(slope)) * (hot + p) + abs(c) * (p * (each + total + 8 * U) + 4 * U * hot)
    return (loss, logp, d), (bl, bp, bd)

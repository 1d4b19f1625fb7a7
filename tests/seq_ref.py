"""Plain fp64 implementations (torch, CPU) of the token-sequence operators and
the error bounds their fp32 kernels are held to.

Notation: u = 2^-24 (one fp32 rounding).  The kernels' exponential is CUDA's
__expf, documented to 2 + floor(1.16 |x|) ulp, an ulp at most 2 u of the
value twice over (2^-23), and their division to 2 ulp."""
import math

import torch

U = 2.0 ** -24
ULP = 2.0 ** -23
TINY = 1e-30


def out_round(dtype):
    """Relative rounding of an output: half a bf16 ulp is at most 2^-8 of the value."""
    return 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24


# ---------------------------------------------------------------- recurrence
def gate_error(z):
    """Relative error of f and of 1 - f: one exponential, one sum, one division, one product."""
    return (6.0 + 1.16 * z.abs().clamp(max=200.0)) * ULP


def recur(z, x, width, h0=None, lengths=None):
    """(h, h_last, before, f, g) in fp64; before[t] = h_{t-1}."""
    b, t, d = x.shape
    z = z.double().repeat_interleave(width, -1)
    f, g = 1 / (1 + torch.exp(-z)), 1 / (1 + torch.exp(z))
    n = torch.full((b,), t) if lengths is None else lengths.clamp(0, t).long()
    s = torch.zeros(b, d, dtype=torch.float64) if h0 is None else h0.double()
    h, before = torch.zeros(b, t, d, dtype=torch.float64), torch.zeros(b, t, d, dtype=torch.float64)
    for i in range(t):
        on = (i < n)[:, None]
        before[:, i] = s
        s = torch.where(on, f[:, i] * s + g[:, i] * x[:, i].double(), s)
        h[:, i] = torch.where(on, s, 0.0)
    return h, s, before, f, g


def recur_grad(z, x, width, dh, dh_last=None, h0=None, lengths=None):
    """(dz, dx, dh0), and G, in fp64."""
    b, t, d = x.shape
    _, _, before, f, g = recur(z, x, width, h0, lengths)
    n = torch.full((b,), t) if lengths is None else lengths.clamp(0, t).long()
    r = torch.zeros(b, d, dtype=torch.float64) if dh_last is None else dh_last.double()
    dz, dx = torch.zeros(b, t, d // width, dtype=torch.float64), torch.zeros(b, t, d, dtype=torch.float64)
    for i in range(t - 1, -1, -1):
        on = (i < n)[:, None]
        G = r + dh[:, i].double()
        dx[:, i] = torch.where(on, g[:, i] * G, 0.0)
        v = torch.where(on, f[:, i] * g[:, i] * G * (before[:, i] - x[:, i].double()), 0.0)
        dz[:, i] = v.reshape(b, -1, width).sum(-1)
        r = torch.where(on, f[:, i] * G, r)
    return dz, dx, r


def recur_bounds(z, x, width, h0=None, lengths=None, dh=None, dh_last=None):
    """Absolute fp32 error bounds (h, h_last, dz, dx, dh0).

    Whatever the order of the scan, h_t is a sum of products f_t ... f_{s+1}
    g_s x_s; a factor f_i carries gate_error(z_i) and the roundings of one
    product and one sum, so E_t = f_t E_{t-1} + (gate_error + 4 u) H_t with
    the majorant H_t = f_t H_{t-1} + g_t |x_t|.  The same along G with M_t =
    |dh_t| + f_{t+1} M_{t+1}; dz and dx follow by the product rule."""
    b, t, d = x.shape
    H, Hl, Hb, f, g = recur(z, x.abs(), width, None if h0 is None else h0.abs(), lengths)
    n = torch.full((b,), t) if lengths is None else lengths.clamp(0, t).long()
    c = gate_error(z.double().nan_to_num(200.0, 200.0, -200.0)).repeat_interleave(width, -1) + 4 * U
    E, Eb = torch.zeros_like(H), torch.zeros_like(H)
    e = torch.zeros(b, d, dtype=torch.float64)
    for i in range(t):
        on = (i < n)[:, None]
        Eb[:, i] = e
        e = torch.where(on, f[:, i] * e + c[:, i] * H[:, i], e)
        E[:, i] = torch.where(on, e, 0.0)
    out = [E + TINY, e + TINY]
    if dh is None:
        return out
    M = torch.zeros(b, d, dtype=torch.float64) if dh_last is None else dh_last.double().abs()
    e = torch.zeros_like(M)
    bz, bx = torch.zeros(b, t, d // width, dtype=torch.float64), torch.zeros_like(H)
    for i in range(t - 1, -1, -1):
        on = (i < n)[:, None]
        G, eG = M + dh[:, i].double().abs(), e + U * (M + dh[:, i].double().abs())
        bx[:, i] = torch.where(on, g[:, i] * (eG + c[:, i] * G), 0.0)
        span = Hb[:, i] + x[:, i].double().abs()
        v = f[:, i] * g[:, i] * (eG * span + G * Eb[:, i] + (2 * c[:, i] + (4 + width) * U) * G * span)
        bz[:, i] = torch.where(on, v, 0.0).reshape(b, -1, width).sum(-1)
        M, e = torch.where(on, f[:, i] * G, M), torch.where(on, f[:, i] * (eG + c[:, i] * G), e)
    return out + [bz + TINY, bx + TINY, e + TINY]


# ---------------------------------------------------------------- distillation
def distill(logits, ids, teacher, labels=None, weight=None, tau=1.0, alpha=1.0):
    """(loss, dlogits, loss bound, dlogits bound), row by row, in fp64.

    An exponent y = (s - m) / tau carries 4 u |y| (difference, reciprocal,
    product), its exponential (2 + 1.16 |y|) ulp more; a sum of V of them adds
    chains of at most V / 32 + 64 roundings (a row has 32 threads or more)."""
    r, v = logits.shape
    k = 0 if ids is None else ids.shape[1]
    loss, dl = torch.zeros(r, dtype=torch.float64), torch.zeros(r, v, dtype=torch.float64)
    bl, bd = torch.full((r,), TINY, dtype=torch.float64), torch.full((r, v), TINY, dtype=torch.float64)

    def soft(y):
        """softmax of y (entries may be -inf), log of its sum from the maximum,
        the relative error of each entry and the error of that log."""
        m = y.max()
        y = y - m
        e = torch.exp(y)
        q, a = e / e.sum(), torch.where(e > 0, y.abs(), 0.0)
        each = (3 + 1.16 * a) * ULP + 4 * U * a
        total = (q * each).sum() + (len(y) / 32 + 64) * U
        return q, y - e.sum().log(), each + total + 4 * ULP, total + 4 * U * (1 + a) + 4 * U * e.sum().log().abs()

    for i in range(r):
        s = logits[i].double()
        if (s == -math.inf).all():
            continue
        w = 1.0 if weight is None else float(weight[i])
        here = [(int(c), float(t)) for c, t in zip(ids[i].tolist(), teacher[i].double().tolist())
                if 0 <= c < v and t != -math.inf] if k else []
        if alpha > 0 and here:
            at, t = torch.tensor([c for c, _ in here]), torch.tensor([t for _, t in here], dtype=torch.float64)
            q, lq, eq, elq = soft(s / tau)
            p, lp, ep, elp = soft(t / tau)
            gap = torch.where(p > 0, lp - lq[at], 0.0)
            loss[i] += alpha * tau ** 2 * (p * gap).sum()
            slack = ep * gap.abs() + elp + elq[at] + 8 * U * (lp.abs() + lq[at].abs()) + (k + 8) * U * gap.abs()
            bl[i] += alpha * tau ** 2 * torch.where(p > 0, p * slack, 0.0).sum()
            target = torch.zeros(v, dtype=torch.float64).index_add_(0, at, p)
            etarget = torch.zeros(v, dtype=torch.float64).index_add_(0, at, p * (ep + k * U))
            dl[i] += w * alpha * tau * (q - target)
            bd[i] += abs(w) * alpha * tau * (q * (eq + 8 * U) + etarget + 8 * U * target)
        label = -1 if labels is None else int(labels[i])
        if alpha < 1 and 0 <= label < v:
            q, lq, eq, elq = soft(s)
            loss[i] -= (1 - alpha) * lq[label]
            bl[i] += (1 - alpha) * (elq[label] + 8 * U * lq[label].abs())
            hot = torch.zeros(v, dtype=torch.float64)
            hot[label] = 1.0
            dl[i] += w * (1 - alpha) * (q - hot)
            bd[i] += abs(w) * (1 - alpha) * (q * (eq + 8 * U) + 8 * U * hot)
    return loss, dl, bl, bd

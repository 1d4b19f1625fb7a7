"""Workloads of linear attention with a decay for each head, of the norms around a block with its gate
and residual scale, and of the clipped policy loss.

A case is a dict of plain values; its "op" names the operator:

  attend        S_t = a_h S_{t-1} + k_t v_t^T, o_t = scale q_t^T S_t over whole prompts
  attend_train  the same and its backward pass
  attend_step   one token of it on a pool of states
  norm          h = res + scale norm(x) silu(gate), n = norm(h)
  norm_train    the same and its backward pass
  policy        loss and gradient of the clipped policy ratio with a KL term
  policy_loss   its loss and log-probabilities alone

Labels and slots outside their range stand for padding: no loss term, no gradient, no state.
"""
import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
EPS = 1e-6


def listed():
    return [
        # one generated token of a single sequence, small heads: latency
        dict(name="attend_token", op="attend_step", slots=1, batch=1, heads=8, dk=64, dv=64, dtype="bf16"),
        # one generated token for each of 96 active sequences of a pool of 128
        dict(name="attend_serve", op="attend_step", slots=128, batch=96, heads=16, dk=128, dv=128, dtype="bf16"),
        # a batch of prompts that continue from kept states
        dict(name="attend_prompt", op="attend", batch=4, time=4096, heads=16, dk=64, dv=64, dtype="bf16", ragged=False, state=True),
        # one long document: few heads, a long time axis
        dict(name="attend_long", op="attend", batch=1, time=65536, heads=8, dk=128, dv=128, dtype="bf16", ragged=False, state=False),
        # an ordinary training batch
        dict(name="attend_train", op="attend_train", batch=8, time=4096, heads=16, dk=128, dv=128, dtype="bf16", ragged=False, state=False),
        # ragged sequences (empty and one-token ones among them), odd heads, fp32
        dict(name="attend_ragged", op="attend_train", batch=5, time=1531, heads=7, dk=40, dv=72, dtype="f32", ragged=True, state=True),
        # a decoding step's rows
        dict(name="norm_token", op="norm", rows=64, width=1000, x="f32", res="f32", post=True, gate=True, scale="number", next=True),
        # the norm of every head of 128 with its gate, as it follows linear attention: short rows, no residual
        dict(name="norm_heads", op="norm_train", rows=524288, width=128, x="bf16", res=None, post=True, gate=True, scale="number", next=False),
        # everything around a block: norm, gate, learned residual scale, fp32 residual stream, norm of the next block
        dict(name="norm_block", op="norm_train", rows=16384, width=2048, x="bf16", res="f32", post=True, gate=True, scale="vector", next=True),
        # a classifier of 1000 classes in fp32
        dict(name="policy_classes", op="policy", rows=256, vocab=1000, dtype="f32", tau=1.0, ref=True, old=True, beta=0.04),
        # a training batch of generated tokens, held to a reference policy
        dict(name="policy_tokens", op="policy", rows=4096, vocab=32000, dtype="bf16", tau=1.0, ref=True, old=True, beta=0.04),
        # a large vocabulary whose rows start at odd addresses, no reference, sampled at another temperature
        dict(name="policy_large", op="policy", rows=4096, vocab=128003, dtype="bf16", tau=0.7, ref=False, old=True, beta=0.0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attend", "attend_train", "attend_step", "norm", "norm_train", "policy", "policy_loss"])
    two = lambda: rng.choice(["bf16", "f32"])  # noqa: E731
    if op in ("attend", "attend_train", "attend_step"):
        dk = rng.choice([64, 128, 64, 128, 16, 24, 32, 40, 80, 96, 100, 33])
        dv = rng.choice([dk, dk, dk, 64, 128, 32, 72, 256, 19])
        heads, dtype = _log(rng, 1, 32), rng.choice(["bf16", "bf16", "f32"])
        if op == "attend_step":
            slots = _log(rng, 1, 256)
            return dict(op=op, slots=slots, batch=rng.randint(1, slots), heads=heads, dk=dk, dv=dv, dtype=dtype)
        batch = _log(rng, 1, 16)
        most = 50_000_000 // (batch * heads * max(dk, dv)) // (2 if dtype == "f32" else 1)
        return dict(op=op, batch=batch, time=_log(rng, 1, min(65536, most)), heads=heads, dk=dk, dv=dv, dtype=dtype, ragged=rng.random() < 0.4,
                    state=rng.random() < 0.5)
    if op in ("norm", "norm_train"):
        width = _log(rng, 16, 8192)
        rows = _log(rng, 1, min(524288, 33_000_000 // width))
        post, nxt = rng.choice([(True, True), (True, False), (False, True)])
        res = rng.choice([None, "bf16", "f32"]) if post else two()
        return dict(op=op, rows=rows, width=width, x=two(), res=res, post=post, gate=rng.random() < 0.5, scale=rng.choice(["number", "vector"]), next=nxt)
    vocab = _log(rng, 10, 200_000)
    rows, ref = _log(rng, 1, min(16384, 200_000_000 // vocab)), rng.random() < 0.6
    return dict(op=op, rows=rows, vocab=vocab, dtype=two(), tau=rng.choice([1.0, 1.0, 0.7, 1.3]), ref=ref, old=rng.random() < 0.8, beta=0.04 if ref else 0.0)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _lengths(g, case):
    """Lengths of a ragged batch: anything from 0 to time, an empty and a one-token sequence among them."""
    b, t = case["batch"], case["time"]
    ln = (torch.rand(b, generator=g, device="cuda") * (t + 1)).int().clamp_(0, t)
    ln[0] = t
    if b > 1:
        ln[1] = 0
    if b > 2:
        ln[2] = min(1, t)
    return ln


def prepare(case, seed):
    g, op = _gen(seed), case["op"]
    rand = lambda *s, dtype=torch.float32: torch.randn(*s, generator=g, device="cuda").to(dtype)  # noqa: E731
    s = {"case": case}
    if op.startswith("attend"):
        b, h, dk, dv, dt = case["batch"], case["heads"], case["dk"], case["dv"], DT[case["dtype"]]
        at = (b, h) if op == "attend_step" else (b, case["time"], h)
        s["q"], s["k"], s["v"] = rand(*at, dk, dtype=dt), rand(*at, dk, dtype=dt), rand(*at, dv, dtype=dt)
        s["scale"] = dk ** -0.5
        # heads forget within 16 to 1000 tokens; the last of several keeps everything
        s["decay"] = 1.0 - torch.exp2(-torch.linspace(4.0, 10.0, h, device="cuda"))
        if h > 3:
            s["decay"][-1] = 1.0
        if op == "attend_step":
            n = case["slots"]
            s["pool"] = rand(n, h, dk, dv)
            s["slots"] = torch.randperm(n, generator=g, device="cuda")[:b].int()
            if b > 8:
                s["slots"][b // 2] = -1  # a place of the batch without a sequence
            return s
        s["lengths"] = _lengths(g, case) if case["ragged"] else None
        s["s0"] = 2.0 * rand(b, h, dk, dv) if case["state"] else None
        if op == "attend_train":
            s["do"] = rand(*at, dv, dtype=dt)
            s["ds_last"] = rand(b, h, dk, dv) if case["state"] else None
    elif op.startswith("norm"):
        r, w, dx = case["rows"], case["width"], DT[case["x"]]
        s["x"] = rand(r, w, dtype=dx)
        s["gate"] = rand(r, w, dtype=dx) if case["gate"] else None
        s["weight"] = 1.0 + 0.2 * rand(w) if case["post"] else None
        s["next"] = 1.0 + 0.2 * rand(w) if case["next"] else None
        s["scale"] = 0.5 + 0.1 * rand(w) if case["scale"] == "vector" else 0.7
        s["res"] = 2.0 * rand(r, w, dtype=DT[case["res"]]) if case["res"] else None
        if op == "norm_train":
            dh = DT[case["res"]] if case["res"] else dx
            s["dh"] = rand(r, w, dtype=dh)
            s["dn"] = rand(r, w, dtype=dx) if case["next"] else None
    else:
        r, v, tau = case["rows"], case["vocab"], case["tau"]
        real = v - v // 128  # the vocabulary is padded: its last places are masked
        logits = 2.0 * rand(r, v)
        labels = torch.randint(0, real, (r,), generator=g, device="cuda")
        logits.scatter_add_(1, labels[:, None], 4.0 + rand(r, 1))  # what was generated was likely
        logits[:, real:] = -math.inf
        s["logits"] = logits.to(DT[case["dtype"]])
        lp = torch.empty(r, dtype=torch.float64, device="cuda")
        for i in range(0, r, 512):
            x = s["logits"][i:i + 512].double() / tau
            lp[i:i + 512] = x.gather(1, labels[i:i + 512, None])[:, 0] - x.logsumexp(1)
        # the policy has moved a little since it generated: about a fifth of the ratios are beyond the clip.
        # (None lies within 0.2 % of it, where one more rounding decides whether a row has a gradient.)
        d = 0.15 * rand(r).double()
        lo, hi = math.log(0.8), math.log(1.25)
        d = torch.where((d - lo).abs() < 2e-3, d - 4e-3, torch.where((d - hi).abs() < 2e-3, d + 4e-3, d))
        s["old"] = (lp - d).float() if case["old"] else None
        s["ref"] = (lp + 0.3 * rand(r).double()).float() if case["ref"] else None
        s["advantage"] = rand(r)
        s["labels"] = torch.where(torch.rand(r, generator=g, device="cuda") < 0.05, -1, labels).int()  # padding
        s["weight"] = torch.rand(r, generator=g, device="cuda") / r
    return s


# ---------------------------------------------------------------- plain forms
CHUNK = 64


def _powers(decay, n):
    """decay ** n for every head: heads x the shape of n."""
    return torch.pow(decay.double().view(-1, *([1] * n.dim())), n.double()).float()


def _chunks(x, fill):
    return torch.nn.functional.pad(x, (0, 0, 0, fill)).unflatten(2, (-1, CHUNK))


def _attend(q, k, v, decay, s0=None):
    """sum over j <= i of a^(i - j) (q_i . k_j) v_j, and a^(i + 1) q_i^T s0, of batch x heads x time x width in fp32,
    in chunks: the scores of a chunk, and the state before it from the sums of all chunks before that one."""
    t = q.shape[2]
    fill = -t % CHUNK
    q, k, v = _chunks(q, fill), _chunks(k, fill), _chunks(v, fill)
    i = torch.arange(CHUNK, device=q.device)
    near = (i[:, None] - i).clamp(min=0)
    inside = torch.where(i[:, None] >= i, _powers(decay, near), 0.0)  # heads x chunk x chunk
    out = ((q @ k.transpose(-1, -2)) * inside[:, None]) @ v
    sums = (k * _powers(decay, CHUNK - 1 - i)[:, None, :, None]).transpose(-1, -2) @ v  # batch x heads x chunks x dk x dv
    n = sums.shape[2]
    c = torch.arange(n, device=q.device)
    gap = (c[:, None] - c - 1).clamp(min=0)
    across = torch.where(c[:, None] > c, _powers(decay, gap * CHUNK), 0.0)  # heads x chunks x chunks
    before = (across @ sums.flatten(-2)).view_as(sums)
    if s0 is not None:
        before = before + _powers(decay, c * CHUNK)[:, :, None, None] * s0[:, :, None]
    out = out + (q * _powers(decay, i + 1)[:, None, :, None]) @ before
    return out.flatten(2, 3)[:, :, :t]


def _to_end(decay, n, t):
    """a ** (n - 1 - j) for the tokens j < n of every sequence, else 0: batch x heads x time x 1; and a ** n."""
    j = torch.arange(t, device=decay.device)
    e = n[:, None] - 1 - j
    w = torch.pow(decay.double()[None, :, None], e.clamp(min=0)[:, None].double())
    return torch.where((e >= 0)[:, None], w, 0.0).float()[..., None], torch.pow(decay.double(), n[:, None].double()).float()[..., None, None]


def _plain_attend(s):
    case, dt, a = s["case"], s["q"].dtype, s["decay"]
    t = case["time"]
    n = torch.full((case["batch"],), t, device="cuda") if s["lengths"] is None else s["lengths"].long()
    live = (torch.arange(t, device="cuda") < n[:, None])[:, None, :, None]
    real = lambda x: torch.where(live, x.float().transpose(1, 2), 0.0)  # noqa: E731
    back = lambda x: torch.where(live, x, 0.0).transpose(1, 2).to(dt)  # noqa: E731
    q, k, v, scale = real(s["q"]), real(s["k"]), real(s["v"]), s["scale"]
    o = back(scale * _attend(q, k, v, a, s["s0"]))
    w, whole = _to_end(a, n, t)
    last = (k * w).transpose(-1, -2) @ v
    if s["s0"] is not None:
        last = last + whole * s["s0"]
    if case["op"] == "attend":
        return o, last
    do = scale * real(s["do"])
    flip = lambda x: x.flip(2)  # noqa: E731
    dq = _attend(do, v, k, a, None if s["s0"] is None else s["s0"].transpose(-1, -2))
    dk = flip(_attend(flip(v), flip(do), flip(q), a))
    dv = flip(_attend(flip(k), flip(q), flip(do), a))
    ds0 = (q * _powers(a, torch.arange(1, t + 1, device="cuda"))[None, ..., None]).transpose(-1, -2) @ do
    if s["ds_last"] is not None:
        dk = dk + w * (v @ s["ds_last"].transpose(-1, -2))
        dv = dv + w * (k @ s["ds_last"])
        ds0 = ds0 + whole * s["ds_last"]
    return o, last, back(dq), back(dk), back(dv), ds0


def _plain_step(s):
    slots = s["slots"].long()
    live = (slots >= 0)[:, None, None]
    state = s["pool"][slots.clamp(min=0)]
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    new = s["decay"][:, None, None] * state + k[..., None] * v[..., None, :]
    spare = torch.zeros_like(state[:1])  # a row behind the pool takes what the empty places give
    pool = torch.cat([s["pool"], spare])
    pool[torch.where(slots >= 0, slots, len(pool) - 1)] = new
    s["pool"].copy_(pool[:-1])
    o = s["scale"] * (q[..., None, :] @ new)[..., 0, :]
    return torch.where(live, o, 0.0).to(s["q"].dtype), s["pool"]


def _plain_norm(s):
    case, x, dt = s["case"], s["x"].float(), s["x"].dtype
    w, w2, scale = s["weight"], s["next"], s["scale"]
    rx = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
    y = x if w is None else x * rx * w
    g = None if s["gate"] is None else s["gate"].float()
    sig = None if g is None else torch.sigmoid(g)
    a = y if g is None else y * (g * sig)
    h = a * scale if s["res"] is None else s["res"].float() + a * scale
    out = [h.to(dt if s["res"] is None else s["res"].dtype)]
    if w2 is not None:
        rh = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
        out.append((h * rh * w2).to(dt))
    if case["op"] == "norm":
        return out
    d = s["dh"].float()
    if w2 is not None:
        dn = s["dn"].float()
        d = d + rh * (dn * w2 - h * (rh * rh) * (dn * w2 * h).mean(1, keepdim=True))
        out.append((dn * h * rh).sum(0))
    if s["res"] is not None:
        out.append(d.to(s["res"].dtype))
    if case["scale"] == "vector":
        out.append((d * a).sum(0))
    da = d * scale
    if g is not None:
        out.append((da * y * (sig * (1 + g * (1 - sig)))).to(dt))
        da = da * (g * sig)
    if w is not None:
        out.append((da * x * rx).sum(0))
        da = rx * (da * w - x * (rx * rx) * (da * w * x).mean(1, keepdim=True))
    return out + [da.to(dt)]


def _plain_policy(s):
    case, tau = s["case"], s["case"]["tau"]
    x, label = s["logits"].float(), s["labels"].long()
    real = label >= 0
    at = label.clamp(min=0)[:, None]
    y = (x - x.amax(1, keepdim=True)) / tau
    e = torch.exp(y)
    total = e.sum(1, keepdim=True)
    lp = (y.gather(1, at) - total.log())[:, 0]
    A, old = s["advantage"], lp if s["old"] is None else s["old"]
    r = torch.exp(lp - old)
    loss = -torch.minimum(r * A, r.clamp(0.8, 1.25) * A)
    out = ((A > 0) & (r > 1.25)) | ((A < 0) & (r < 0.8))
    d = torch.where(out, 0.0, -A * r)
    if s["ref"] is not None:
        u = s["ref"] - lp
        loss = loss + case["beta"] * (torch.expm1(u) - u)
        d = d - case["beta"] * torch.expm1(u)
    loss, logp = torch.where(real, loss, 0.0), torch.where(real, lp, 0.0)
    if case["op"] == "policy_loss":
        return loss, logp
    d = torch.where(real, d, 0.0) * s["weight"] / tau
    p = (e / total).scatter_add(1, at, torch.full_like(total, -1.0))
    return loss, logp, (-d[:, None] * p).to(s["logits"].dtype)


def _plain(s):
    op = s["case"]["op"]
    if op == "attend_step":
        return _plain_step(s)
    if op.startswith("attend"):
        return _plain_attend(s)
    return _plain_norm(s) if op.startswith("norm") else _plain_policy(s)


def run(state):
    if not own:
        return _plain(state)
    from paper_2103_08802_gb300 import seq
    s, case = state, state["case"]
    op = case["op"]
    if op == "attend_step":
        return seq.attend_step(s["q"], s["k"], s["v"], s["decay"], s["pool"], slots=s["slots"], scale=s["scale"]), s["pool"]
    if op.startswith("attend"):
        o, last = seq.attend(s["q"], s["k"], s["v"], s["decay"], s0=s["s0"], lengths=s["lengths"], scale=s["scale"])
        if op == "attend":
            return o, last
        return (o, last) + seq.attend_grad(s["q"], s["k"], s["v"], s["decay"], s["do"], s0=s["s0"], ds_last=s["ds_last"], lengths=s["lengths"], scale=s["scale"])
    if op.startswith("norm"):
        h, n = seq.norm(s["x"], weight=s["weight"], gate=s["gate"], scale=s["scale"], res=s["res"], next_weight=s["next"], eps=EPS)
        out = [h] if n is None else [h, n]
        if op == "norm":
            return out
        g = seq.norm_grad(s["x"], s["dh"], dn=s["dn"], weight=s["weight"], gate=s["gate"], scale=s["scale"], res=s["res"], next_weight=s["next"], eps=EPS)
        return out + [v for v in (g.next_weight, g.res, g.scale, g.gate, g.weight, g.x) if v is not None]
    r = seq.policy(s["logits"], s["labels"], s["advantage"], old=s["old"], ref=s["ref"], weight=s["weight"] if op == "policy" else None,
                   clip=(0.2, 0.25), beta=case["beta"], tau=case["tau"], grad=op == "policy")
    return r if op == "policy" else r[:2]


def work(case):
    op = case["op"]
    if op.startswith("attend"):
        b, h, dk, dv, e = case["batch"], case["heads"], case["dk"], case["dv"], SIZE[case["dtype"]]
        if op == "attend_step":
            return {"bytes": b * h * (8 * dk * dv + (2 * dk + 2 * dv) * e) + 4 * b, "flops": 5 * b * h * dk * dv}
        t, train = case["time"], op == "attend_train"
        live = (t + (b - 2) * t / 2) / b if case["ragged"] and b > 1 else t
        read, wrote = 2 * dk + dv + (dv if train else 0), dv + (2 * dk + dv if train else 0)
        ends = b * h * dk * dv * 4 * ((2 if case["state"] else 1) + ((2 if case["state"] else 1) if train else 0))
        return {"bytes": b * h * (live * read + t * wrote) * e + ends, "flops": b * h * live * dk * dv * (16 if train else 5)}
    if op.startswith("norm"):
        n, ex, er = case["rows"] * case["width"], SIZE[case["x"]], SIZE[case["res"] or case["x"]]
        gate, res, nxt = bool(case["gate"]), bool(case["res"]), bool(case["next"])
        bytes_ = n * (ex * (1 + gate + nxt) + er * (1 + res))
        if op == "norm_train":
            bytes_ += n * (ex * (1 + gate + nxt) + er * (1 + res))
        return {"bytes": bytes_, "flops": n * (30 if op == "norm_train" else 10)}
    r, v = case["rows"], case["vocab"]
    return {"bytes": r * v * SIZE[case["dtype"]] * (2 if op == "policy" else 1) + r * 28, "flops": r * v * (8 if op == "policy" else 4)}


# ---------------------------------------------------------------- the definitions in fp64
def _exact_attend(s):
    """Token by token forwards for the states, and token by token backwards for what reaches them."""
    case, scale = s["case"], s["scale"]
    b, t, h, dk, dv = (case[n] for n in ("batch", "time", "heads", "dk", "dv"))
    train, ragged = case["op"] == "attend_train", s["lengths"] is not None
    if train and t > 30000:
        return None
    a = s["decay"].double().view(1, h, 1, 1)
    new = lambda d: torch.zeros(b, t, h, d, dtype=torch.float64, device="cuda")  # noqa: E731
    S = torch.zeros(b, h, dk, dv, dtype=torch.float64, device="cuda") if s["s0"] is None else s["s0"].double()
    o, dq, dk_, dv_ = new(dv), new(dk) if train else None, new(dk) if train else None, new(dv) if train else None
    on = torch.arange(t, device="cuda")[:, None, None, None, None] < (s["lengths"].view(1, b, 1, 1, 1) if ragged else t)
    for i in range(t):
        k, v = s["k"][:, i].double(), s["v"][:, i].double()
        after = torch.addcmul(S * a, k[..., None], v[:, :, None])
        S = torch.where(on[i], after, S) if ragged else after
        o[:, i] = scale * torch.einsum("bhk,bhkv->bhv", s["q"][:, i].double(), S)
        if train:
            dq[:, i] = scale * torch.einsum("bhv,bhkv->bhk", s["do"][:, i].double(), S)
    mask = (lambda x: torch.where(on[:, :, :, 0].transpose(0, 1), x, 0.0)) if ragged else (lambda x: x)
    if not train:
        return mask(o), S
    G = torch.zeros_like(S) if s["ds_last"] is None else s["ds_last"].double()
    for i in range(t - 1, -1, -1):
        q, do = s["q"][:, i].double(), s["do"][:, i].double()
        here = torch.addcmul(G, q[..., None], do[:, :, None], value=scale)
        dk_[:, i] = torch.einsum("bhv,bhkv->bhk", s["v"][:, i].double(), here)
        dv_[:, i] = torch.einsum("bhk,bhkv->bhv", s["k"][:, i].double(), here)
        G = torch.where(on[i], here * a, G) if ragged else here * a
    return mask(o), S, mask(dq), mask(dk_), mask(dv_), G


def _exact_norm(s):
    """The forward pass in fp64, its gradients by autograd."""
    case = s["case"]
    names = [n for n in ("next", "res", "scale", "gate", "weight", "x") if torch.is_tensor(s[n])]
    v = {n: s[n].double().requires_grad_(case["op"] == "norm_train") if torch.is_tensor(s[n]) else s[n] for n in ("next", "res", "scale", "gate", "weight", "x")}
    unit = lambda x: x / (x.square().mean(-1, keepdim=True) + EPS).sqrt()  # noqa: E731
    a = v["x"] if v["weight"] is None else unit(v["x"]) * v["weight"]
    if v["gate"] is not None:
        a = a * torch.nn.functional.silu(v["gate"])
    h = a * v["scale"]
    if v["res"] is not None:
        h = h + v["res"]
    out = [h] if v["next"] is None else [h, unit(h) * v["next"]]
    if case["op"] == "norm":
        return out
    grads = torch.autograd.grad(out, [v[n] for n in names], [s["dh"].double()] + ([] if v["next"] is None else [s["dn"].double()]))
    return [x.detach() for x in out] + list(grads)


def _exact_policy(s):
    case, tau = s["case"], s["case"]["tau"]
    parts = []
    for i in range(0, case["rows"], 1024):
        x = s["logits"][i:i + 1024].double()
        label, A = s["labels"][i:i + 1024].long(), s["advantage"][i:i + 1024].double()
        there = label >= 0
        hot = torch.zeros_like(x).scatter_(1, label.clamp(min=0)[:, None], 1.0)
        ls = torch.log_softmax(x / tau, 1)
        lp = ls.gather(1, label.clamp(min=0)[:, None])[:, 0]
        ratio = torch.ones_like(lp) if s["old"] is None else torch.exp(lp - s["old"][i:i + 1024].double())
        bound = torch.where(A > 0, ratio.clamp(max=1.25), ratio.clamp(min=0.8))
        loss, slope = -A * bound, torch.where(bound == ratio, -A * ratio, 0.0)
        if s["ref"] is not None:
            back = torch.exp(s["ref"][i:i + 1024].double() - lp)
            loss, slope = loss + case["beta"] * (back - back.log() - 1), slope + case["beta"] * (1 - back)
        part = [loss * there, torch.where(there, lp, 0.0)]
        if case["op"] == "policy":
            part.append((hot - ls.exp()) * (slope * there * s["weight"][i:i + 1024].double() / tau)[:, None])
        parts.append(part)
    return [torch.cat(p) for p in zip(*parts)]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "attend_step":
        pool = s["pool"].double()
        out = torch.zeros(s["v"].shape, dtype=torch.float64, device="cuda")
        for i, slot in enumerate(s["slots"].tolist()):
            if slot >= 0:
                pool[slot] = s["decay"].double()[:, None, None] * pool[slot] + s["k"][i].double()[..., None] * s["v"][i].double()[:, None]
                out[i] = s["scale"] * torch.einsum("hk,hkv->hv", s["q"][i].double(), pool[slot])
        return out, pool
    if op.startswith("attend"):
        return _exact_attend(s)
    return _exact_norm(s) if op.startswith("norm") else _exact_policy(s)

"""Workloads of the token-sequence operators: embedding lookup and its gradient, the gated linear
recurrence (scan, backward pass, single-token step) and distillation from a teacher's top logits.

A case is a dict of plain values; its "op" names the operator:

  embed       out[n] = scale * table[ids[n]]
  embed_grad  dtable[v] (+)= scale * sum of dout[n] over the tokens n with ids[n] = v
  recur       h_t = f_t h_{t-1} + (1 - f_t) x_t, f = sigmoid(z): the forward scan
  train       the forward scan and its backward pass
  step        one token of the recurrence on a pool of states
  distill     loss and gradient of the mixed teacher / label cross entropy
  eval        its loss alone

Ids, labels and slots outside their range stand for padding: a zero row, no gradient, no loss term.
"""
import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


def listed():
    return [
        # one decoding step's tokens of a serving batch: latency
        dict(name="embed_decode", op="embed", n=64, vocab=32000, d=1024, table="bf16", out="bf16", ids=32),
        # a prefill / training batch of 16 sequences of 2048 tokens over a large vocabulary
        dict(name="embed_batch", op="embed", n=32768, vocab=128000, d=2048, table="bf16", out="bf16", ids=64),
        # gradient of a small training batch into a dense fp32 table, width not a power of two
        dict(name="embed_grad", op="embed_grad", n=8192, vocab=32000, d=1000, dout="bf16", dtable="f32", acc=False, ids=32),
        # gradient of a large batch added into the table that the tied output layer has already written
        dict(name="embed_grad_acc", op="embed_grad", n=65536, vocab=128000, d=2048, dout="bf16", dtable="f32", acc=True, ids=64),
        # one generated token for each of 96 active sequences of a pool of 128
        dict(name="recur_step", op="step", slots=128, batch=96, heads=2048, width=1, dtype="bf16"),
        # one long document: few rows, a long time axis
        dict(name="recur_long", op="recur", batch=1, time=65536, heads=1024, width=1, dtype="bf16", ragged=False, state=True),
        # an ordinary training batch
        dict(name="recur_train", op="train", batch=8, time=4096, heads=2048, width=1, dtype="bf16", ragged=False, state=False),
        # ragged sequences (empty and one-token ones among them), one gate for each head of 48 channels, fp32
        dict(name="recur_heads", op="train", batch=5, time=1531, heads=25, width=48, dtype="f32", ragged=True, state=True),
        # a classifier of 1000 classes learning from a teacher's best five
        dict(name="distill_classes", op="distill", rows=256, vocab=1000, k=5, dtype="f32", tau=4.0, alpha=0.9, labels=True),
        # a training batch of tokens, teacher and labels mixed
        dict(name="distill_tokens", op="distill", rows=4096, vocab=32000, k=32, dtype="bf16", tau=2.0, alpha=0.5, labels=True),
        # the same with a large vocabulary whose rows start at odd addresses, teacher alone
        dict(name="distill_large", op="distill", rows=4096, vocab=128003, k=64, dtype="bf16", tau=1.0, alpha=1.0, labels=False),
        # validation loss over held-out tokens
        dict(name="distill_eval", op="eval", rows=2048, vocab=50001, k=16, dtype="bf16", tau=1.0, alpha=0.5, labels=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "recur", "train", "step", "distill", "eval"])
    two = lambda: rng.choice(["bf16", "f32"])  # noqa: E731
    if op in ("embed", "embed_grad"):
        d = _log(rng, 16, 8192)
        vocab = _log(rng, 200, min(256000, 262_144_000 // d))
        n = _log(rng, 1, min(65536, 67_000_000 // d))
        if op == "embed":
            return dict(op=op, n=n, vocab=vocab, d=d, table=two(), out=two(), ids=rng.choice([32, 64]))
        return dict(op=op, n=n, vocab=vocab, d=d, dout=two(), dtable=rng.choice(["bf16", "f32"]), acc=rng.random() < 0.3, ids=rng.choice([32, 64]))
    if op in ("recur", "train"):
        batch = _log(rng, 1, 16)
        width = rng.choice([1, 1, 1, 5, 16, 32, 48, 64, 128])
        heads = _log(rng, max(1, 32 // width), 4096 // width)
        time = _log(rng, 1, min(65536, 33_000_000 // (batch * heads * width)))
        return dict(op=op, batch=batch, time=time, heads=heads, width=width, dtype=two(), ragged=rng.random() < 0.4, state=rng.random() < 0.5)
    if op == "step":
        slots = _log(rng, 1, 512)
        width = rng.choice([1, 1, 5, 16, 64])
        return dict(op=op, slots=slots, batch=rng.randint(1, slots), heads=_log(rng, max(1, 32 // width), 8192 // width), width=width, dtype=two())
    vocab = _log(rng, 10, 200_000)
    rows = _log(rng, 1, min(16384, 200_000_000 // vocab))
    return dict(op=op, rows=rows, vocab=vocab, k=_log(rng, 1, min(128, vocab // 2)), dtype=two(), tau=rng.choice([0.7, 1.0, 1.0, 1.5, 2.0, 4.0]), alpha=rng.choice([0.5, 0.9, 1.0]),
                labels=rng.random() < 0.7)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _tokens(g, n, vocab, bits):
    """Token ids as text has them: a few are frequent, most are rare (p ~ 1 / rank); about 1 % padding."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    rank = torch.exp(u * math.log(vocab + 1.0)).long().clamp_(1, vocab) - 1
    ids = (rank * 7919 + 13) % vocab if vocab % 7919 else rank
    ids = torch.where(torch.rand(n, generator=g, device="cuda") < 0.01, -1, ids)
    return ids.to(torch.int64 if bits == 64 else torch.int32)


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
    if op in ("embed", "embed_grad"):
        n, vocab, d = case["n"], case["vocab"], case["d"]
        s["ids"] = _tokens(g, n, vocab, case["ids"])
        s["scale"] = math.sqrt(d)
        if op == "embed":
            s["table"] = (rand(vocab, d) / math.sqrt(d)).to(DT[case["table"]])
        else:
            s["dout"] = rand(n, d, dtype=DT[case["dout"]])
            if case["acc"]:
                s["dtable"] = rand(vocab, d, dtype=DT[case["dtable"]])
    elif op in ("recur", "train"):
        b, t, h, d, dt = case["batch"], case["time"], case["heads"], case["heads"] * case["width"], DT[case["dtype"]]
        z = 2.0 + 2.0 * rand(b, t, h)
        # about one token in 200 is skipped (+inf: the state passes), one in 2000 starts afresh (-inf)
        u = torch.rand(b, t, 1, generator=g, device="cuda")
        z = torch.where(u < 0.005, math.inf, torch.where(u > 0.9995, -math.inf, z))
        s["z"], s["x"] = z.to(dt), rand(b, t, d, dtype=dt)
        s["lengths"] = _lengths(g, case) if case["ragged"] else None
        s["h0"] = rand(b, d) if case["state"] else None
        if op == "train":
            s["dh"] = rand(b, t, d, dtype=dt)
            s["dh_last"] = rand(b, d) if case["state"] else None
    elif op == "step":
        b, n, h, d, dt = case["batch"], case["slots"], case["heads"], case["heads"] * case["width"], DT[case["dtype"]]
        s["z"], s["x"] = (2.0 + 2.0 * rand(b, h)).to(dt), rand(b, d, dtype=dt)
        s["pool"] = rand(n, d)
        s["slots"] = torch.randperm(n, generator=g, device="cuda")[:b].int()
        if b > 8:
            s["slots"][b // 2] = -1  # a place of the batch without a sequence
    else:
        r, v, k, dt = case["rows"], case["vocab"], case["k"], DT[case["dtype"]]
        real = v - v // 128  # the vocabulary is padded: its last places are masked
        first = torch.randint(0, real, (r, 1), generator=g, device="cuda")
        ids = (first + torch.arange(k, device="cuda") * max(1, real // k)) % real
        s["teacher"] = (6.0 - 0.2 * torch.arange(k, device="cuda") + 0.5 * rand(r, k)).to(dt)
        logits = 1.5 * rand(r, v)
        logits.scatter_add_(1, ids, 0.5 * s["teacher"].float())
        logits[:, real:] = -math.inf
        s["logits"] = logits.to(dt)
        u = torch.rand(r, 1, generator=g, device="cuda")
        ids = torch.where(u < 0.03, -1, ids)  # rows without a teacher
        if k > 2:
            ids[r // 2, k - k // 3:] = -1  # a shorter list
        s["ids"] = ids.int()
        s["labels"] = None
        if case["labels"]:
            label = torch.where(torch.rand(r, generator=g, device="cuda") < 0.5, first[:, 0], torch.randint(0, real, (r,), generator=g, device="cuda"))
            s["labels"] = torch.where(torch.rand(r, generator=g, device="cuda") < 0.05, -1, label).int()
        s["weight"] = torch.rand(r, generator=g, device="cuda") / r
    return s


def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t along dim 1, from zero: by doubling, log2(time) passes over the whole."""
    k = 1
    while k < a.shape[1]:
        b = torch.cat([b[:, :k], a[:, k:] * b[:, :-k] + b[:, k:]], 1)
        a = torch.cat([a[:, :k], a[:, k:] * a[:, :-k]], 1)
        k *= 2
    return b


def _gates(s):
    """f, 1 - f (both exact where the other is small), x and the mask of real tokens, in fp32."""
    case = s["case"]
    z = s["z"].float().repeat_interleave(case["width"], -1)
    x, live = s["x"].float(), None
    f, g = torch.sigmoid(z), torch.sigmoid(-z)
    if s["lengths"] is not None:
        live = (torch.arange(case["time"], device="cuda") < s["lengths"][:, None])[..., None]
        f, g, x = torch.where(live, f, 1.0), torch.where(live, g, 0.0), torch.where(live, x, 0.0)
    return f, g, x, live


def _plain_recur(s):
    case, dt = s["case"], s["x"].dtype
    f, g, x, live = _gates(s)
    u = g * x
    if s["h0"] is not None:
        u[:, 0] += f[:, 0] * s["h0"]
    h = _scan(f, u)
    last = h[:, -1].clone()
    out = h if live is None else torch.where(live, h, 0.0)
    if case["op"] == "recur":
        return out.to(dt), last
    h0 = torch.zeros_like(last) if s["h0"] is None else s["h0"]
    before = torch.cat([h0[:, None], h[:, :-1]], 1)
    dh = s["dh"].float() if live is None else torch.where(live, s["dh"].float(), 0.0)
    if s["dh_last"] is not None:
        dh = torch.cat([dh[:, :-1], dh[:, -1:] + s["dh_last"][:, None]], 1)
    later = torch.cat([f[:, 1:], torch.ones_like(f[:, :1])], 1)  # G_t = dh_t + f_{t+1} G_{t+1}
    G = _scan(later.flip(1), dh.flip(1)).flip(1)
    dx = g * G
    dz = (f * g * G * (before - x)).unflatten(-1, (case["heads"], case["width"])).sum(-1)
    if live is not None:
        dx, dz = torch.where(live, dx, 0.0), torch.where(live, dz, 0.0)
    return out.to(dt), last, dz.to(dt), dx.to(dt), f[:, 0] * G[:, 0]


def _plain_step(s):
    z = s["z"].float().repeat_interleave(s["case"]["width"], -1)
    slots = s["slots"].long()
    live = (slots >= 0)[:, None]
    h = s["pool"][slots.clamp(min=0)]
    new = torch.sigmoid(z) * h + torch.sigmoid(-z) * s["x"].float()
    spare = torch.zeros_like(h[:1])  # a row behind the pool takes what the empty places give
    pool = torch.cat([s["pool"], spare])
    pool[torch.where(slots >= 0, slots, len(pool) - 1)] = new
    s["pool"].copy_(pool[:-1])
    return torch.where(live, new, 0.0).to(s["x"].dtype), s["pool"]


def _plain_distill(s):
    case = s["case"]
    tau, alpha, v = case["tau"], case["alpha"], case["vocab"]
    x, t, ids = s["logits"].float(), s["teacher"].float(), s["ids"].long()
    y = x - x.amax(1, keepdim=True)
    e = torch.exp(y / tau)
    total = e.sum(1, keepdim=True)
    there = (ids >= 0) & (ids < v)
    t = torch.where(there, t, -math.inf) / tau
    any_ = there.any(1, keepdim=True)
    t = torch.where(any_, t, 0.0)
    t = t - t.amax(1, keepdim=True)
    w = torch.exp(t)
    p = torch.where(any_, w / w.sum(1, keepdim=True), 0.0)
    at = ids.clamp(0, v - 1)
    logp, logq = t - w.sum(1, keepdim=True).log(), y.gather(1, at) / tau - total.log()
    loss = alpha * tau * tau * torch.where(p > 0, p * (logp - logq), 0.0).sum(1)
    train = case["op"] == "distill"
    if train:
        d = (alpha * tau) * torch.where(any_, (e / total).scatter_add(1, at, -p), 0.0)
    if s["labels"] is not None and alpha < 1:
        label = s["labels"].long()
        known = label >= 0
        at = label.clamp(min=0)[:, None]
        e = torch.exp(y)
        total = e.sum(1, keepdim=True)
        loss = loss + (1 - alpha) * torch.where(known, (total.log() - y.gather(1, at))[:, 0], 0.0)
        if train:
            one = (e / total).scatter_add(1, at, torch.full_like(total, -1.0))
            d = d + (1 - alpha) * torch.where(known[:, None], one, 0.0)
    if not train:
        return loss
    return loss, (d * s["weight"][:, None]).to(s["logits"].dtype)


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "embed":
        ids = s["ids"].long()
        rows = s["table"][ids.clamp(min=0)].float() * s["scale"]
        return torch.where((ids >= 0)[:, None], rows, 0.0).to(DT[case["out"]])
    if op == "embed_grad":
        ids = s["ids"].long()
        d = torch.where((ids >= 0)[:, None], s["dout"].float() * s["scale"], 0.0)
        if not case["acc"]:
            return torch.zeros(case["vocab"], case["d"], device="cuda").index_add_(0, ids.clamp(min=0), d).to(DT[case["dtable"]])
        return s["dtable"].copy_(s["dtable"].float().index_add_(0, ids.clamp(min=0), d)) if case["dtable"] != "f32" else s["dtable"].index_add_(0, ids.clamp(min=0), d)
    if op in ("recur", "train"):
        return _plain_recur(s)
    return _plain_step(s) if op == "step" else _plain_distill(s)


def run(state):
    if not own:
        return _plain(state)
    from paper_2103_08802_gb300 import seq
    s, case = state, state["case"]
    op = case["op"]
    if op == "embed":
        return seq.embed(s["ids"], s["table"], scale=s["scale"], dtype=DT[case["out"]])
    if op == "embed_grad":
        if case["acc"]:
            return seq.embed_grad(s["ids"], s["dout"], scale=s["scale"], dtable=s["dtable"], accumulate=True)
        return seq.embed_grad(s["ids"], s["dout"], vocab=case["vocab"], scale=s["scale"], dtype=DT[case["dtable"]])
    if op == "recur":
        return seq.recur(s["z"], s["x"], h0=s["h0"], lengths=s["lengths"])
    if op == "train":
        h, last, saved = seq.recur(s["z"], s["x"], h0=s["h0"], lengths=s["lengths"], save=True)
        dz, dx, dh0 = seq.recur_grad(s["z"], s["x"], saved, s["dh"], dh_last=s["dh_last"], lengths=s["lengths"])
        return h, last, dz, dx, dh0
    if op == "step":
        return seq.recur_step(s["z"], s["x"], s["pool"], slots=s["slots"]), s["pool"]
    r = seq.distill(s["logits"], s["ids"], s["teacher"], labels=s["labels"], tau=case["tau"], alpha=case["alpha"],
                    weight=s["weight"] if op == "distill" else None, grad=op == "distill")
    return r if op == "distill" else r[0]


def work(case):
    op = case["op"]
    if op in ("embed", "embed_grad"):
        n, vocab, d = case["n"], case["vocab"], case["d"]
        # distinct tokens of n draws with p ~ 1 / rank: the rows that have to be touched
        ranks = range(1, vocab + 1) if vocab <= 4096 else [math.exp((i + 0.5) * math.log(vocab) / 4096) for i in range(4096)]
        each = 1.0 if vocab <= 4096 else None
        c = 1.0 / math.log(vocab + 1.0)
        rows = sum((each or r * math.log(vocab) / 4096) * -math.expm1(n * math.log1p(-min(0.999, c * math.log1p(1.0 / r)))) for r in ranks)
        if op == "embed":
            return {"bytes": n * case["ids"] / 8 + rows * d * SIZE[case["table"]] + n * d * SIZE[case["out"]], "flops": n * d}
        grad = (2 * rows if case["acc"] else vocab) * d * SIZE[case["dtable"]]
        return {"bytes": n * case["ids"] / 8 + n * d * SIZE[case["dout"]] + grad, "flops": 2 * n * d}
    if op in ("recur", "train"):
        b, t, h, d = case["batch"], case["time"], case["heads"], case["heads"] * case["width"]
        live = (t + (b - 2) * t / 2) / b if case["ragged"] and b > 1 else t
        read, wrote = h + d + (d if op == "train" else 0), d + (d + h if op == "train" else 0)
        ends = b * d * 4 * ((3 if case["state"] else 1) + (1 if op == "train" else 0) - (1 if op == "recur" and case["state"] else 0))
        return {"bytes": SIZE[case["dtype"]] * b * (live * read + t * wrote) + ends, "flops": b * live * d * (20 if op == "train" else 8)}
    if op == "step":
        b, h, d = case["batch"], case["heads"], case["heads"] * case["width"]
        return {"bytes": b * ((h + 2 * d) * SIZE[case["dtype"]] + 8 * d + 4), "flops": 8 * b * d}
    r, v = case["rows"], case["vocab"]
    side = r * (case["k"] * (4 + SIZE[case["dtype"]]) + 12)
    return {"bytes": r * v * SIZE[case["dtype"]] * (2 if op == "distill" else 1) + side, "flops": r * v * (10 if op == "distill" else 4)}


def _exact_recur(s):
    """The recurrence token by token, and its gradient by the chain rule backwards, in fp64."""
    case = s["case"]
    b, t, d, p = case["batch"], case["time"], case["heads"] * case["width"], case["width"]
    n = [t] * b if s["lengths"] is None else s["lengths"].tolist()
    hs = torch.zeros(b, t, d, dtype=torch.float64, device="cuda")
    h = torch.zeros(b, d, dtype=torch.float64, device="cuda") if s["h0"] is None else s["h0"].double()
    live = torch.arange(t, device="cuda")[:, None] < torch.tensor(n, device="cuda")  # [t, b]
    first = h
    for i in range(t):
        z = s["z"][:, i].double()[..., None].expand(-1, -1, p).reshape(b, d)
        new = h / (1 + torch.exp(-z)) + s["x"][:, i].double() / (1 + torch.exp(z))
        h = torch.where(live[i][:, None], new, h) if s["lengths"] is not None else new
        hs[:, i] = h
    show = hs * live.t()[..., None] if s["lengths"] is not None else hs
    if case["op"] == "recur":
        return show, h
    last = h
    dz = torch.zeros(b, t, case["heads"], dtype=torch.float64, device="cuda")
    dx = torch.zeros(b, t, d, dtype=torch.float64, device="cuda")
    grad = torch.zeros(b, d, dtype=torch.float64, device="cuda") if s["dh_last"] is None else s["dh_last"].double()
    for i in range(t - 1, -1, -1):
        on = live[i][:, None]
        z = s["z"][:, i].double()[..., None].expand(-1, -1, p).reshape(b, d)
        f, g = 1 / (1 + torch.exp(-z)), 1 / (1 + torch.exp(z))
        here = grad + s["dh"][:, i].double()
        prev = hs[:, i - 1] if i else first
        dx[:, i] = torch.where(on, g * here, 0.0)
        dz[:, i] = torch.where(on, f * g * here * (prev - s["x"][:, i].double()), 0.0).reshape(b, -1, p).sum(-1)
        grad = torch.where(on, f * here, grad)
    return show, last, dz, dx, grad


def _exact_distill(s):
    case = s["case"]
    tau, a, v = case["tau"], case["alpha"], case["vocab"]
    losses, grads = [], []
    for i in range(0, case["rows"], 1024):
        x = s["logits"][i:i + 1024].double()
        ids, t = s["ids"][i:i + 1024].long(), s["teacher"][i:i + 1024].double()
        rows = torch.arange(len(x), device="cuda")[:, None]
        there = ids >= 0
        any_ = there.any(1)
        lq = torch.log_softmax(x / tau, 1)
        lp = torch.log_softmax(torch.where(any_[:, None], torch.where(there, t, -math.inf), 0.0) / tau, 1)
        p = lp.exp() * any_[:, None]
        loss = a * tau ** 2 * torch.where(there, p * (lp - lq[rows, ids.clamp(min=0)]), 0.0).sum(1)
        target = torch.zeros_like(x).index_put_((rows.expand_as(ids), ids.clamp(min=0)), p, accumulate=True)
        d = a * tau * (lq.exp() - target) * any_[:, None]
        if s["labels"] is not None and a < 1:
            label = s["labels"][i:i + 1024].long()
            l1 = torch.log_softmax(x, 1)
            hot = torch.zeros_like(x).index_put_((rows[:, 0], label.clamp(min=0)), torch.ones((), dtype=torch.float64, device="cuda"))
            known = (label >= 0).double()
            loss = loss - (1 - a) * known * l1[rows[:, 0], label.clamp(min=0)]
            d = d + (1 - a) * known[:, None] * (l1.exp() - hot)
        losses.append(loss)
        if case["op"] == "distill":
            grads.append(d * s["weight"][i:i + 1024, None].double())
    return (torch.cat(losses), torch.cat(grads)) if grads else torch.cat(losses)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "embed":
        ids = s["ids"].long()
        out = s["table"].double()[ids.clamp(min=0)] * s["scale"]
        out[ids < 0] = 0
        return out
    if op == "embed_grad":
        ids = s["ids"].long()
        keep = ids >= 0
        out = s["dtable"].double() if case["acc"] else torch.zeros(case["vocab"], case["d"], dtype=torch.float64, device="cuda")
        return out.index_put_((ids[keep],), s["dout"][keep].double() * s["scale"], accumulate=True)
    if op in ("recur", "train"):
        return _exact_recur(s)
    if op == "step":
        h = s["pool"].double()
        out = torch.zeros(s["x"].shape, dtype=torch.float64, device="cuda")
        for i, slot in enumerate(s["slots"].tolist()):
            if slot >= 0:
                z = s["z"][i].double()[:, None].expand(-1, case["width"]).reshape(-1)
                h[slot] = out[i] = h[slot] / (1 + torch.exp(-z)) + s["x"][i].double() / (1 + torch.exp(z))
        return out, h
    return _exact_distill(s)

"""A small token network on the library's calls: embedding, layers between 1x1
convolutions (the linear layers, pnn.conv_run), trained by distillation from a
teacher's top logits or by a policy's advantages.

    h = embed(tokens);  logits = W_v h behind the layers
    mixer="recur":   h += W_o recur(W_z h, W_x h)
    mixer="attend":  h += s norm(W_o (norm(attend(W_q n, W_k n, W_v n)) silu(W_g n))),
                     n = norm(h), and W_v reads norm(h) too

Activations are fp32, convolution operands are rounded to bf16 by the
convolutions, states and sums are fp32.  `train_step` and `policy_step` run
forward, loss, backward and an SGD update; `generate` feeds tokens one by one
through the mixer's single-token step on a pool of states.  All of it runs on
torch's current stream; every convolution waits for that stream before it returns.

    python -m paper_2103_08802_gb300.seqnet      trains a student on synthetic
                                                 text from a larger teacher
"""
from __future__ import annotations

import math

import torch

from . import pnn, seq

__all__ = ["SeqNet"]


def _rows(x):
    """The geometry of a 1x1 convolution over the rows of x (... x channels)."""
    return dict(batch=1, h=1, w=x.numel() // x.shape[-1], ksize=1, stride=1)


def _conv(mode, g):
    """One convolution on torch's current stream, where the sequence operators run."""
    pnn.conv_run(mode, [g], stream=torch.cuda.current_stream())


class SeqNet:
    """vocab and width must be multiples of 8.  mixer "recur": a layer has
    `heads` gates (of width / heads channels each); "attend": `heads` heads of
    linear attention of width / heads each (by default width // 64 heads, or the
    fewest more that divide the width), whose decays keep from 16 to 1000 tokens."""

    mixer = "recur"

    def __init__(self, vocab, width, layers, heads=None, seed=0, mixer="recur"):
        self.vocab, self.width, self.layers, self.mixer = vocab, width, layers, mixer
        if mixer not in ("recur", "attend"):
            raise ValueError("mixer is recur or attend")
        if not heads:
            heads = width if mixer == "recur" else next(n for n in range(max(1, width // 64), width + 1) if width % n == 0)
        self.heads = heads
        if vocab % 8 or width % 8 or width % self.heads or (mixer == "recur" and self.heads % 8):
            raise ValueError("vocab, width and a recurrence's heads must be multiples of 8, and width one of heads")
        self.head = width // self.heads
        g = torch.Generator().manual_seed(seed)
        shape = {"embed": (vocab, width), "out": (vocab, width)}
        for i in range(layers):
            if mixer == "recur":
                shape |= {f"z{i}": (self.heads, width), f"x{i}": (width, width), f"o{i}": (width, width)}
            else:
                shape |= {f"{n}{i}": (width, width) for n in "qkvgo"}
        # N(0, 1 / width): the embedding is scaled by sqrt(width) when it is looked up
        self.params = {k: (torch.randn(*s, generator=g) / math.sqrt(width)).cuda() for k, s in shape.items()}
        self.scale = math.sqrt(width)
        if mixer == "attend":
            if self.head > 256:
                raise ValueError("a head is at most 256 wide")
            ones = {f"pre{i}": (width,) for i in range(layers + 1)} | {f"post{i}": (width,) for i in range(layers)} | {f"head{i}": (self.head,) for i in range(layers)}
            self.params |= {k: torch.ones(s, device="cuda") for k, s in ones.items()}
            self.params |= {f"res{i}": torch.full((width,), 0.5, device="cuda") for i in range(layers)}
            self.decay = 1.0 - torch.exp2(-torch.linspace(4.0, 10.0, self.heads, device="cuda"))

    # ------------------------------------------------------------ linear layers
    def _linear(self, x, name, res=None):
        w = self.params[name]
        y = torch.empty(*x.shape[:-1], w.shape[0], device=x.device)
        _conv("forward", dict(_rows(x), c=w.shape[1], k=w.shape[0], x=x, wt=w.to(torch.bfloat16), y=y, res=res))
        return y

    def _linear_grad(self, x, name, dy, grads, dx=None):
        """Adds dy W to dx (a new tensor without one); dW into grads."""
        w = self.params[name]
        new = dx is None
        if new:
            dx = torch.empty_like(x)
        grads[name] = torch.empty_like(w)
        g = dict(_rows(x), c=w.shape[1], k=w.shape[0], wt=w.to(torch.bfloat16), dy=dy)
        _conv("dgrad", dict(g, dx=dx, accumulate=0 if new else 1))
        _conv("wgrad", dict(g, x=x, dw=grads[name]))
        return dx

    # ------------------------------------------------------------ training
    def forward(self, tokens, lengths=None, keep=None, states=None):
        """Logits (batch x time x vocab) of tokens (batch x time int32; -1:
        padding).  keep: a list that receives what the backward needs, states:
        one that receives each layer's state behind the tokens."""
        h = seq.embed(tokens, self.params["embed"], scale=self.scale)
        if self.mixer == "attend":
            return self._attend_forward(h, lengths, keep, states)
        for i in range(self.layers):
            z, x = self._linear(h, f"z{i}"), self._linear(h, f"x{i}")
            r, last, saved = seq.recur(z, x, lengths=lengths, save=True)
            if keep is not None:
                keep.append((h, z, x, r, saved))
            if states is not None:
                states.append(last)
            h = self._linear(r, f"o{i}", res=h)
        if keep is not None:
            keep.append(h)
        return self._linear(h, "out")

    def _split(self, x):
        return x.view(*x.shape[:-1], self.heads, self.head)

    def _attend_forward(self, x, lengths, keep, states):
        P, scale = self.params, self.head ** -0.5
        h, n = seq.norm(x, next_weight=P["pre0"])
        if keep is not None:
            keep.append(x)
        for i in range(self.layers):
            q, k, v, g = (self._linear(n, f"{m}{i}") for m in "qkvg")
            o, last = seq.attend(self._split(q), self._split(k), self._split(v), self.decay, lengths=lengths, scale=scale)
            y, _ = seq.norm(o, weight=P[f"head{i}"], gate=self._split(g))
            b = self._linear(y.view_as(x), f"o{i}")
            if keep is not None:
                keep.append((h, n, q, k, v, g, o, y, b))
            if states is not None:
                states.append(last)
            h, n = seq.norm(b, weight=P[f"post{i}"], scale=P[f"res{i}"], res=h, next_weight=P[f"pre{i + 1}"])
        if keep is not None:
            keep.append(n)
        return self._linear(n, "out")

    def _attend_backward(self, dn, keep, grads, lengths):
        """The gradient of the embedded tokens from that of the last norm."""
        P, scale, dh = self.params, self.head ** -0.5, None
        for i in reversed(range(self.layers)):
            h, n, q, k, v, g, o, y, b = keep.pop()
            d = seq.norm_grad(b, dh, dn, weight=P[f"post{i}"], scale=P[f"res{i}"], res=h, next_weight=P[f"pre{i + 1}"])
            grads[f"post{i}"], grads[f"res{i}"], grads[f"pre{i + 1}"], dh = d.weight, d.scale, d.next_weight, d.res
            dy = self._linear_grad(y.view_as(b), f"o{i}", d.x, grads)
            d = seq.norm_grad(o, self._split(dy), weight=P[f"head{i}"], gate=self._split(g))
            grads[f"head{i}"] = d.weight
            dq, dk, dv, _ = seq.attend_grad(self._split(q), self._split(k), self._split(v), self.decay, d.x, lengths=lengths, scale=scale)
            dn = None
            for m, t in zip("qkvg", (dq, dk, dv, d.gate)):
                dn = self._linear_grad(n, f"{m}{i}", t.view_as(b), grads, dn)
        d = seq.norm_grad(keep.pop(), dh, dn, next_weight=P["pre0"])
        grads["pre0"] = d.next_weight
        return d.x

    def _backward(self, tokens, d, keep, lengths):
        """Gradients of all parameters from that of the logits (rows x vocab)."""
        grads = {}
        dh = self._linear_grad(keep.pop(), "out", d.view(*tokens.shape, self.vocab), grads)
        if self.mixer == "attend":
            dh = self._attend_backward(dh, keep, grads, lengths)
        else:
            for i in reversed(range(self.layers)):
                h, z, x, r, saved = keep.pop()
                dr = self._linear_grad(r, f"o{i}", dh, grads)
                dz, dx, _ = seq.recur_grad(z, x, saved, dr, lengths=lengths)
                self._linear_grad(h, f"z{i}", dz, grads, dh)  # dh already has the residual's share
                self._linear_grad(h, f"x{i}", dx, grads, dh)
        grads["embed"] = seq.embed_grad(tokens, dh, vocab=self.vocab, scale=self.scale)
        return grads

    @staticmethod
    def _flat(v, n, *s):
        return None if v is None else v.reshape(n, *s)

    def _weights(self, weight, n, device):
        return torch.full((n,), 1.0 / n, device=device) if weight is None else weight.reshape(n)

    def loss_and_grads(self, tokens, ids, teacher, labels=None, weight=None, tau=1.0, alpha=1.0, lengths=None):
        """Losses of every token and the gradients of their sum weighted by
        `weight` (batch x time; None: the mean).  ids, teacher: batch x time x
        k pairs, or None with alpha = 0 (the labels alone)."""
        keep, n = [], tokens.numel()
        logits = self.forward(tokens, lengths, keep).view(n, self.vocab)
        loss, d = seq.distill(logits, self._flat(ids, n, -1), self._flat(teacher, n, -1), labels=self._flat(labels, n),
                              weight=self._weights(weight, n, logits.device), tau=tau, alpha=alpha, out=logits)  # the gradient takes the logits' place
        return loss, self._backward(tokens, d, keep, lengths)

    def policy_and_grads(self, tokens, actions, advantage, old=None, ref=None, weight=None, clip=(0.2, 0.2), beta=0.0, tau=1.0, lengths=None):
        """Losses and log-probabilities of every token's action (the token that
        was drawn behind it; -1: none), and the gradients of the losses' sum
        weighted by `weight` (None: the mean).  advantage, old (None: the present
        policy drew them), ref: batch x time."""
        keep, n = [], tokens.numel()
        logits = self.forward(tokens, lengths, keep).view(n, self.vocab)
        loss, logp, d = seq.policy(logits, actions.reshape(n), advantage.reshape(n), old=self._flat(old, n), ref=self._flat(ref, n),
                                   weight=self._weights(weight, n, logits.device), clip=clip, beta=beta, tau=tau, out=logits)
        return loss, logp, self._backward(tokens, d, keep, lengths)

    def _descend(self, lr, grads):
        for k, g in grads.items():
            self.params[k].add_(g, alpha=-lr)

    def train_step(self, lr, *args, **kw):
        """One SGD step of distillation; returns the losses of the tokens before it."""
        loss, grads = self.loss_and_grads(*args, **kw)
        self._descend(lr, grads)
        return loss

    def policy_step(self, lr, *args, **kw):
        """One SGD step of the policy loss; returns losses and log-probabilities before it."""
        loss, logp, grads = self.policy_and_grads(*args, **kw)
        self._descend(lr, grads)
        return loss, logp

    # ------------------------------------------------------------ generation
    def new_states(self, slots):
        """States of `slots` sequences, one tensor a layer."""
        shape = (slots, self.width) if self.mixer == "recur" else (slots, self.heads, self.head, self.head)
        return [torch.zeros(shape, device="cuda") for _ in range(self.layers)]

    def step(self, tokens, states, slots=None):
        """Logits after one more token of each sequence (tokens: int32, batch);
        states advance in place.  slots: each sequence's place in them."""
        h = seq.embed(tokens, self.params["embed"], scale=self.scale)
        if self.mixer == "attend":
            P = self.params
            h, n = seq.norm(h, next_weight=P["pre0"])
            for i in range(self.layers):
                q, k, v, g = (self._split(self._linear(n, f"{m}{i}")) for m in "qkvg")
                o = seq.attend_step(q, k, v, self.decay, states[i], slots=slots, scale=self.head ** -0.5)
                y, _ = seq.norm(o, weight=P[f"head{i}"], gate=g)
                h, n = seq.norm(self._linear(y.view_as(h), f"o{i}"), weight=P[f"post{i}"], scale=P[f"res{i}"], res=h, next_weight=P[f"pre{i + 1}"])
            return self._linear(n, "out")
        for i in range(self.layers):
            z, x = self._linear(h, f"z{i}"), self._linear(h, f"x{i}")
            h = self._linear(seq.recur_step(z, x, states[i], slots=slots), f"o{i}", res=h)
        return self._linear(h, "out")

    def generate(self, prompt, steps):
        """Greedy continuation of prompts (batch x time int32, time >= 1): batch x steps."""
        if prompt.dim() != 2 or prompt.shape[1] == 0:
            raise ValueError("a prompt is batch x time with a token at least")
        if self.mixer == "attend":  # the whole prompt at once leaves the states that the steps go on from
            states = []
            logits = self.forward(prompt.contiguous(), states=states)[:, -1]
        else:
            states = self.new_states(prompt.shape[0])
            for t in range(prompt.shape[1]):
                logits = self.step(prompt[:, t].contiguous(), states)
        out = []
        for _ in range(steps):
            out.append(logits.argmax(1).int())
            logits = self.step(out[-1], states)
        return torch.stack(out, 1) if out else prompt[:, :0]


def _text(batch, time, vocab, seed):
    """Synthetic text: from every token one of four successors, the first of them half of the time."""
    g = torch.Generator().manual_seed(seed)
    nxt = torch.randint(0, vocab, (vocab, 4), generator=torch.Generator().manual_seed(1))
    t = torch.zeros(batch, time + 1, dtype=torch.int64)
    t[:, 0] = torch.randint(0, vocab, (batch,), generator=g)
    pick = torch.tensor([0, 0, 1, 2, 3, 0])[torch.randint(0, 6, (batch, time), generator=g)]
    for i in range(time):
        t[:, i + 1] = nxt[t[:, i], pick[:, i]]
    t = t.int().cuda()
    return t[:, :-1].contiguous(), t[:, 1:].contiguous()


def main(steps=200, vocab=512, k=16):
    teacher, student = SeqNet(vocab, 256, 2, seed=1), SeqNet(vocab, 128, 2, heads=16, seed=2)
    for i in range(steps):  # the teacher learns from the labels alone
        x, y = _text(16, 128, vocab, i)
        loss = teacher.train_step(0.2, x, None, None, labels=y, alpha=0.0)
    print("teacher: cross entropy %.3f (uniform %.3f)" % (loss.mean().item(), math.log(vocab)))
    for i in range(steps):
        x, y = _text(16, 128, vocab, 1000 + i)
        top = teacher.forward(x).topk(k, -1)
        loss = student.train_step(0.2, x, top.indices.int(), top.values, labels=y, tau=2.0, alpha=0.5)
        if i % 50 == 0 or i == steps - 1:
            print("student: step %d, loss %.3f" % (i, loss.mean().item()))
    policy = SeqNet(vocab, 128, 2, heads=2, seed=3, mixer="attend")
    for i in range(steps):  # a policy that is rewarded for the commonest successor
        x, y = _text(16, 128, vocab, i)
        loss = policy.train_step(0.2, x, None, None, labels=y, alpha=0.0)
    print("linear attention: cross entropy %.3f" % loss.mean().item())
    nxt = torch.randint(0, vocab, (vocab, 4), generator=torch.Generator().manual_seed(1))[:, 0].int().cuda()
    for i in range(steps // 4):
        x, _ = _text(16, 128, vocab, 2000 + i)
        p = torch.softmax(policy.forward(x).view(-1, vocab), 1)
        drawn = torch.multinomial(p, 1).int().view_as(x)
        reward = (drawn == nxt[x.long()]).float()
        _, logp = policy.policy_step(0.5, x, drawn, reward - reward.mean(), beta=0.0)
        if i % 10 == 0:
            print("policy: step %d, reward %.3f" % (i, reward.mean().item()))
    seq.sync()
    print("continued:", student.generate(_text(1, 8, vocab, 7)[0], 8)[0].tolist())


if __name__ == "__main__":
    main()

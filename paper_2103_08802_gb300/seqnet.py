"""A small token network on the library's calls: embedding, layers of gated
recurrence between 1x1 convolutions (the linear layers, pnn.conv_run), and
distillation from a teacher's top logits.

    h = embed(tokens);  per layer: h += W_o recur(W_z h, W_x h);  logits = W_v h

Activations are fp32, convolution operands are rounded to bf16 by the
convolutions, states and sums are fp32.  `train_step` runs forward, loss,
backward and an SGD update; `generate` feeds tokens one by one through the
recurrence's single-token step on a pool of states.  All of it runs on torch's
current stream; every convolution waits for that stream before it returns.

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
    """vocab and width must be multiples of 8; a layer has `heads` gates (of
    width / heads channels each)."""

    def __init__(self, vocab, width, layers, heads=None, seed=0):
        self.vocab, self.width, self.layers = vocab, width, layers
        self.heads = heads or width
        if vocab % 8 or width % 8 or self.heads % 8 or width % self.heads:
            raise ValueError("vocab, width and heads must be multiples of 8, and width one of heads")
        g = torch.Generator().manual_seed(seed)
        shape = {"embed": (vocab, width), "out": (vocab, width)}
        for i in range(layers):
            shape |= {f"z{i}": (self.heads, width), f"x{i}": (width, width), f"o{i}": (width, width)}
        # N(0, 1 / width): the embedding is scaled by sqrt(width) when it is looked up
        self.params = {k: (torch.randn(*s, generator=g) / math.sqrt(width)).cuda() for k, s in shape.items()}
        self.scale = math.sqrt(width)

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
    def forward(self, tokens, lengths=None, keep=None):
        """Logits (batch x time x vocab) of tokens (batch x time int32; -1:
        padding).  keep: a list that receives what the backward needs."""
        h = seq.embed(tokens, self.params["embed"], scale=self.scale)
        for i in range(self.layers):
            z, x = self._linear(h, f"z{i}"), self._linear(h, f"x{i}")
            r, _, saved = seq.recur(z, x, lengths=lengths, save=True)
            if keep is not None:
                keep.append((h, z, x, r, saved))
            h = self._linear(r, f"o{i}", res=h)
        if keep is not None:
            keep.append(h)
        return self._linear(h, "out")

    def loss_and_grads(self, tokens, ids, teacher, labels=None, weight=None, tau=1.0, alpha=1.0, lengths=None):
        """Losses of every token and the gradients of their sum weighted by
        `weight` (batch x time; None: the mean).  ids, teacher: batch x time x
        k pairs, or None with alpha = 0 (the labels alone)."""
        keep, grads, n = [], {}, tokens.numel()
        logits = self.forward(tokens, lengths, keep).view(n, self.vocab)
        if weight is None:
            weight = torch.full((n,), 1.0 / n, device=logits.device)
        flat = lambda v, *s: None if v is None else v.reshape(n, *s)  # noqa: E731
        weight = flat(weight)
        loss, d = seq.distill(logits, flat(ids, -1), flat(teacher, -1), labels=flat(labels), weight=weight, tau=tau, alpha=alpha,
                              out=logits)  # the gradient takes the logits' place
        dh = self._linear_grad(keep.pop(), "out", d.view(*tokens.shape, self.vocab), grads)
        for i in reversed(range(self.layers)):
            h, z, x, r, saved = keep.pop()
            dr = self._linear_grad(r, f"o{i}", dh, grads)
            dz, dx, _ = seq.recur_grad(z, x, saved, dr, lengths=lengths)
            self._linear_grad(h, f"z{i}", dz, grads, dh)  # dh already has the residual's share
            self._linear_grad(h, f"x{i}", dx, grads, dh)
        grads["embed"] = seq.embed_grad(tokens, dh, vocab=self.vocab, scale=self.scale)
        return loss, grads

    def train_step(self, lr, *args, **kw):
        """One SGD step; returns the losses of the tokens before it."""
        loss, grads = self.loss_and_grads(*args, **kw)
        for k, g in grads.items():
            self.params[k].add_(g, alpha=-lr)
        return loss

    # ------------------------------------------------------------ generation
    def new_states(self, slots):
        """States of `slots` sequences, one tensor a layer."""
        return [torch.zeros(slots, self.width, device="cuda") for _ in range(self.layers)]

    def step(self, tokens, states, slots=None):
        """Logits after one more token of each sequence (tokens: int32, batch);
        states advance in place.  slots: each sequence's place in them."""
        h = seq.embed(tokens, self.params["embed"], scale=self.scale)
        for i in range(self.layers):
            z, x = self._linear(h, f"z{i}"), self._linear(h, f"x{i}")
            h = self._linear(seq.recur_step(z, x, states[i], slots=slots), f"o{i}", res=h)
        return self._linear(h, "out")

    def generate(self, prompt, steps):
        """Greedy continuation of prompts (batch x time int32, time >= 1): batch x steps."""
        if prompt.dim() != 2 or prompt.shape[1] == 0:
            raise ValueError("a prompt is batch x time with a token at least")
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
    seq.sync()
    print("continued:", student.generate(_text(1, 8, vocab, 7)[0], 8)[0].tolist())


if __name__ == "__main__":
    main()

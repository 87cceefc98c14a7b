"""A small language model whose layers forget by their data: token embeddings, then layers of norm_before (the residual sum and its norm), projections,
norms of the heads' queries and keys, rotary positions, the gated delta rule and norm_after with the heads' gate; trained by their backward passes, then
decoded token by token from the kept states.

    python examples/delta_language_model.py [--steps 150] [--width 128] [--layers 2] [--type bf16]

The data are sequences of two random Markov chains over 64 tokens that take turns, so that a token follows from the one before the last; their entropy is
known, and a trained model's loss comes near it.
"""
import argparse
import os
import sys

import torch
from torch.nn.functional import linear, logsigmoid

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2510_03426_amd import Goom, rotary_frequencies  # noqa: E402


class Embed(torch.autograd.Function):
    @staticmethod
    def forward(ctx, g, table, tokens):
        tokens = tokens.contiguous()
        ctx.g, ctx.tokens, ctx.vocab = g, tokens, table.shape[0]
        return g.embedding(table, tokens)

    @staticmethod
    def backward(ctx, grad):
        return None, ctx.g.embedding_backward(ctx.tokens, grad.contiguous(), ctx.vocab), None


class Before(torch.autograd.Function):
    """(norm(h) weight, h), h = residual + x."""

    @staticmethod
    def forward(ctx, g, x, residual, weight):
        y, h, _, rstd = g.norm_before(x, residual=residual, weight=weight, want_stats=True)
        ctx.g, ctx.alone = g, residual is None
        ctx.save_for_backward(h, rstd, weight)
        return y, h.view_as(h) if ctx.alone else h

    @staticmethod
    def backward(ctx, grad_y, grad_h):
        h, rstd, weight = ctx.saved_tensors
        gres, gx, _, gw, _, _ = ctx.g.norm_before_backward(h, h, grad_y.contiguous(), None, rstd, grad_h=grad_h.contiguous(), weight=weight)
        return None, gx, None if ctx.alone else gres, gw


class After(torch.autograd.Function):
    """norm(x) weight silu(gate), each head by itself."""

    @staticmethod
    def forward(ctx, g, x, groups, weight, gate):
        y, _, rstd = g.norm_after(x, groups, weight=weight, gate=gate, want_stats=True)
        ctx.g, ctx.groups, ctx.gated = g, groups, gate is not None
        ctx.save_for_backward(*([x, rstd, weight] + ([gate] if ctx.gated else [])))
        return y

    @staticmethod
    def backward(ctx, grad):
        x, rstd, weight = ctx.saved_tensors[:3]
        gx, ggate, gw, _, _ = ctx.g.norm_after_backward(x, grad.contiguous(), None, rstd, ctx.groups, weight=weight, gate=ctx.saved_tensors[3] if ctx.gated else None)
        return None, gx, None, gw, ggate


class Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, g, q, k, positions, frequencies):
        ctx.g, ctx.positions, ctx.frequencies = g, positions, frequencies
        return g.rotary(q, k, positions, frequencies)

    @staticmethod
    def backward(ctx, grad_q, grad_k):
        return (None,) + ctx.g.rotary_backward(grad_q.contiguous(), grad_k.contiguous(), ctx.positions, ctx.frequencies) + (None, None)


class Delta(torch.autograd.Function):
    @staticmethod
    def forward(ctx, g, q, k, v, log_decay, beta):
        ctx.g = g
        ctx.save_for_backward(q, k, v, log_decay, beta)
        return g.gated_delta(q, k, v, log_decay, beta)

    @staticmethod
    def backward(ctx, grad):
        return (None,) + ctx.g.gated_delta_backward(*ctx.saved_tensors, grad.contiguous())[:5]


class Model:
    """A layer: h = residual + what the last layer gave; q, k, v, gate, decay and beta from norm(h); the heads' q and k of length one, turned by
    their positions; the gated delta rule; the heads' norm with the gate; a projection."""

    def __init__(self, g, vocab, width, heads, layers, dtype=torch.bfloat16, seed=0):
        gen = torch.Generator().manual_seed(seed)
        self.g, self.vocab, self.width, self.heads, self.dtype = g, vocab, width, heads, dtype
        self.frequencies = rotary_frequencies(width // heads // 2, device="cuda")[0]

        def draw(*s):
            return (torch.randn(s, generator=gen) * s[-1] ** -0.5).cuda().requires_grad_()

        def full(n, value):
            return torch.full((n,), float(value), device="cuda", requires_grad=True)
        self.table, self.out = draw(vocab, width), draw(vocab, width)
        unit = (width // heads) ** -0.5  # a head whose mean square is one, times this: of length one
        self.blocks = [dict(norm=full(width, 1), qk=draw(2 * width, width), unit=full(2 * width, unit), v=draw(width, width), gate=draw(width, width),
                            ab=draw(2 * heads, width), keep=full(heads, 4), heads=full(width, 1), proj=draw(width, width)) for _ in range(layers)]
        self.last = dict(norm=full(width, 1))

    def parameters(self):
        return [self.table, self.out] + [p for b in self.blocks + [self.last] for p in b.values()]

    def _open(self, block, x, residual):
        """norm(residual + x) and that sum; x: [..., width]."""
        return Before.apply(self.g, x, residual, block["norm"])

    def _inputs(self, block, y, positions):
        """q, k, v [..., heads, width / heads], the decays' logarithms and betas [..., heads] and the gate [..., width]."""
        qk = After.apply(self.g, linear(y, block["qk"].to(y.dtype)), 2 * self.heads, block["unit"], None)
        q, k = (t.unflatten(-1, (self.heads, -1)) for t in qk.split(self.width, dim=-1))
        q, k = Rotary.apply(self.g, q, k, positions, self.frequencies)
        v = linear(y, block["v"].to(y.dtype)).unflatten(-1, (self.heads, -1))
        a, b = linear(y, block["ab"].to(y.dtype)).float().split(self.heads, dim=-1)
        return q, k, v, logsigmoid(a + block["keep"]), torch.sigmoid(b), linear(y, block["gate"].to(y.dtype))

    def _close(self, block, o, gate):
        return linear(After.apply(self.g, o.flatten(-2), self.heads, block["heads"], gate), block["proj"].to(o.dtype))

    def _logits(self, x, residual):
        return linear(self._open(self.last, x, residual)[0], self.out.to(x.dtype)).float()

    def forward(self, tokens, states=None):
        """tokens [batch, T] -> logits [batch, T, vocab]; a list `states` receives the layers' final states."""
        x, h = Embed.apply(self.g, self.table.to(self.dtype), tokens), None
        positions = torch.arange(tokens.shape[1], device=tokens.device).expand(tokens.shape).contiguous()
        for block in self.blocks:
            y, h = self._open(block, x, h)
            *inputs, gate = self._inputs(block, y, positions)
            if states is None:
                o = Delta.apply(self.g, *(t.contiguous() for t in inputs))
            else:
                o, s = self.g.gated_delta(*(t.contiguous() for t in inputs), want_state=True)
                states.append(s)
            x = self._close(block, o, gate)
        return self._logits(x, h)

    def step(self, tokens, positions, states):
        """One token of each sequence: tokens, positions [batch] -> logits [batch, vocab]; the states move on in place."""
        x, h = self.g.embedding(self.table.to(self.dtype), tokens.contiguous()), None
        for block, s in zip(self.blocks, states):
            y, h = self._open(block, x, h)
            *inputs, gate = self._inputs(block, y, positions)
            x = self._close(block, self.g.gated_delta_step(*(t.contiguous() for t in inputs), s), gate)
        return self._logits(x, h)


def chain(vocab, seed=1):
    """Transition probabilities of the chains, and their entropy."""
    p = torch.softmax(4 * torch.randn(vocab, vocab, generator=torch.Generator().manual_seed(seed)), -1)
    return p.cuda(), float(-(p * p.clamp_min(1e-30).log()).sum(-1).mean())


def sample(p, batch, length, gen):
    t = torch.randint(0, p.shape[0], (batch, 2), device="cuda", generator=gen)
    for _ in range(length - 2):
        t = torch.cat([t, torch.multinomial(p[t[:, -2]], 1, generator=gen)], 1)
    return t


def main(argv=None):
    a = argparse.ArgumentParser()
    a.add_argument("--steps", type=int, default=150)
    a.add_argument("--width", type=int, default=128)
    a.add_argument("--heads", type=int, default=4)
    a.add_argument("--layers", type=int, default=2)
    a.add_argument("--vocab", type=int, default=64)
    a.add_argument("--batch", type=int, default=32)
    a.add_argument("--length", type=int, default=65)
    a.add_argument("--type", choices=("bf16", "f16", "f32"), default="bf16")
    a = a.parse_args(argv)
    g = Goom(0)
    model = Model(g, a.vocab, a.width, a.heads, a.layers, {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[a.type])
    gen = torch.Generator(device="cuda").manual_seed(2)
    p, entropy = chain(a.vocab)
    opt = torch.optim.Adam(model.parameters(), lr=3e-3)
    for i in range(a.steps):
        t = sample(p, a.batch, a.length, gen)
        loss = torch.nn.functional.cross_entropy(model.forward(t[:, :-1])[:, 1:].reshape(-1, a.vocab), t[:, 2:].reshape(-1))
        opt.zero_grad()
        loss.backward()
        opt.step()
        if i % 25 == 0 or i == a.steps - 1:
            print(f"step {i}: loss {loss.item():.3f} (the chains' entropy: {entropy:.3f})", flush=True)
    # a prompt at once, then token by token from its states: the same logits as all tokens at once
    with torch.no_grad():
        t = sample(p, 4, a.length, gen)
        whole = model.forward(t)
        states, n = [], t.shape[1] - 10
        parts = [model.forward(t[:, :n], states)[:, -1]]
        for i in range(n, n + 10):
            parts.append(model.step(t[:, i], torch.full((4,), i, device="cuda"), states))
        off = float((torch.stack(parts, 1) - whole[:, n - 1:]).abs().max() / whole.std())
        print(f"ten tokens decoded from kept states: logits within {off:.3g} spreads of those at once", flush=True)
    g.close()
    return off


if __name__ == "__main__":
    main()

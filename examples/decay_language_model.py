"""A small recurrent language model made of the library's layer operators: token embeddings, linear attention with a decay for each
head and group norm with an activation, trained by their backward passes, then decoded token by token from the kept states.

    python examples/decay_language_model.py [--steps 150] [--width 128] [--layers 2]

The data are sequences of a random Markov chain over 256 tokens, whose entropy is known: a trained model's loss comes near it.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2510_03426_amd import Goom  # noqa: E402


class Embed(torch.autograd.Function):
    @staticmethod
    def forward(ctx, g, table, tokens, scale):
        tokens = tokens.contiguous()
        ctx.g, ctx.tokens, ctx.vocab, ctx.scale = g, tokens, table.shape[0], scale
        return g.embedding(table, tokens, scale=scale)

    @staticmethod
    def backward(ctx, grad):
        return None, ctx.g.embedding_backward(ctx.tokens, grad.contiguous(), ctx.vocab, scale=ctx.scale), None, None


class Attend(torch.autograd.Function):
    @staticmethod
    def forward(ctx, g, q, k, v, log_decay):
        ctx.g = g
        ctx.save_for_backward(q, k, v, log_decay)
        return g.linear_attention(q, k, v, log_decay, scale=q.shape[-1] ** -0.5)

    @staticmethod
    def backward(ctx, grad):
        q, k, v, log_decay = ctx.saved_tensors
        return (None,) + ctx.g.linear_attention_backward(q, k, v, log_decay, grad.contiguous(), scale=q.shape[-1] ** -0.5)[:3] + (None,)


class Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, g, x, groups, weight, bias, activation):
        y, mean, rstd = g.group_norm(x, groups, weight, bias, activation=activation, want_stats=True)
        ctx.g, ctx.groups, ctx.activation = g, groups, activation
        ctx.save_for_backward(x, mean, rstd, weight, bias)
        return y

    @staticmethod
    def backward(ctx, grad):
        x, mean, rstd, weight, bias = ctx.saved_tensors
        gx, gw, gb = ctx.g.group_norm_backward(x, grad.contiguous(), mean, rstd, ctx.groups, weight, bias, activation=ctx.activation)
        return None, gx, None, gw, gb, None


class Model:
    """Layers of: norm, projection to q, k, v, linear attention, norm of each head with SiLU, projection, residual sum."""

    def __init__(self, g, vocab, width, heads, layers, seed=0):
        gen = torch.Generator().manual_seed(seed)
        self.g, self.vocab, self.width, self.heads, self.layers = g, vocab, width, heads, layers
        # heads from forgetting within two tokens to remembering some hundred
        self.log_decay = torch.log1p(-torch.exp2(-torch.linspace(1, 7, heads))).cuda()
        def draw(*s):
            return (torch.randn(s, generator=gen) * s[-1] ** -0.5).cuda().requires_grad_()

        def ones():
            return torch.ones(width, device="cuda", requires_grad=True)

        def zeros():
            return torch.zeros(width, device="cuda", requires_grad=True)
        self.table, self.out = draw(vocab, width), draw(vocab, width)
        self.blocks = [dict(w1=ones(), b1=zeros(), qkv=draw(3 * width, width), w2=ones(), b2=zeros(), proj=draw(width, width)) for _ in range(layers)]
        self.last = dict(w=ones(), b=zeros())

    def parameters(self):
        return [self.table, self.out] + [p for b in self.blocks + [self.last] for p in b.values()]

    def _norm(self, x, groups, w, b, act="none"):
        return Norm.apply(self.g, x.reshape(-1, self.width), groups, w, b, act).reshape(x.shape)

    def _heads(self, block, x):
        """q, k, v as slices of one projection's output: [..., heads, width / heads] each."""
        h = self._norm(x, 1, block["w1"], block["b1"])
        qkv = torch.nn.functional.linear(h, block["qkv"].to(x.dtype))
        return [t.unflatten(-1, (self.heads, -1)) for t in qkv.split(self.width, dim=-1)]

    def _rest(self, block, x, o):
        h = self._norm(o.flatten(-2), self.heads, block["w2"], block["b2"], "silu")
        return x + torch.nn.functional.linear(h, block["proj"].to(x.dtype))

    def _logits(self, x):
        return torch.nn.functional.linear(self._norm(x, 1, self.last["w"], self.last["b"]), self.out.to(x.dtype)).float()

    def forward(self, tokens, states=None):
        """tokens [batch, T] -> logits [batch, T, vocab]; a list `states` receives the layers' final states."""
        x = Embed.apply(self.g, self.table.to(torch.bfloat16), tokens, math.sqrt(self.width))
        for block in self.blocks:
            q, k, v = self._heads(block, x)
            if states is None:
                o = Attend.apply(self.g, q, k, v, self.log_decay)
            else:
                o, s = self.g.linear_attention(q, k, v, self.log_decay, scale=q.shape[-1] ** -0.5, want_state=True)
                states.append(s)
            x = self._rest(block, x, o)
        return self._logits(x)

    def step(self, tokens, states):
        """One token of each sequence: tokens [batch] -> logits [batch, vocab]; the states move on in place."""
        x = self.g.embedding(self.table.to(torch.bfloat16), tokens.contiguous(), scale=math.sqrt(self.width))
        for block, s in zip(self.blocks, states):
            q, k, v = self._heads(block, x)
            x = self._rest(block, x, self.g.linear_attention_step(q, k, v, self.log_decay, s, scale=q.shape[-1] ** -0.5))
        return self._logits(x)


def chain(vocab, seed=1):
    """Transition probabilities of the chain, and their entropy."""
    p = torch.softmax(4 * torch.randn(vocab, vocab, generator=torch.Generator().manual_seed(seed)), -1)
    return p.cuda(), float(-(p * p.clamp_min(1e-30).log()).sum(-1).mean())


def sample(p, batch, length, gen):
    t = torch.randint(0, p.shape[0], (batch, 1), device="cuda", generator=gen)
    for _ in range(length - 1):
        t = torch.cat([t, torch.multinomial(p[t[:, -1]], 1, generator=gen)], 1)
    return t


def main(argv=None):
    a = argparse.ArgumentParser()
    a.add_argument("--steps", type=int, default=150)
    a.add_argument("--width", type=int, default=128)
    a.add_argument("--heads", type=int, default=4)
    a.add_argument("--layers", type=int, default=2)
    a.add_argument("--vocab", type=int, default=256)
    a.add_argument("--batch", type=int, default=32)
    a.add_argument("--length", type=int, default=129)
    a = a.parse_args(argv)
    torch.manual_seed(0)
    g = Goom(0)
    model = Model(g, a.vocab, a.width, a.heads, a.layers)
    p, entropy = chain(a.vocab)
    gen = torch.Generator(device="cuda").manual_seed(2)
    opt = torch.optim.Adam(model.parameters(), lr=3e-3)
    first = loss = None
    for i in range(a.steps):
        t = sample(p, a.batch, a.length, gen)
        loss = torch.nn.functional.cross_entropy(model.forward(t[:, :-1]).reshape(-1, a.vocab), t[:, 1:].reshape(-1))
        opt.zero_grad()
        loss.backward()
        opt.step()
        first = loss.item() if first is None else first
        if i % 25 == 0 or i == a.steps - 1:
            print(f"step {i}: loss {loss.item():.3f} (the chain's entropy: {entropy:.3f})", flush=True)
    # a prompt at once, then token by token from its states: the same logits as all tokens at once
    with torch.no_grad():
        t = sample(p, 4, 100, gen)
        whole = model.forward(t)
        states = []
        parts = [model.forward(t[:, :90], states)[:, -1]] + [model.step(t[:, i], states) for i in range(90, 100)]
        off = float((torch.stack(parts, 1) - whole[:, 89:]).abs().max() / whole.std())
        print(f"ten tokens decoded from kept states: logits within {off:.3f} spreads of those at once", flush=True)
    g.close()
    return first, loss.item(), entropy, off


if __name__ == "__main__":
    main()

"""The operators of a layer that forgets by its data, together as they are used: the example model's loss, its gradients and its decoding, and a
decoded layer captured into graphs.

Tolerances, in float32 (u = 2^-24): a value passes through at most 2 layers of some ten operators each, every one a sum of at most W = 64 + 48 terms of
either sign (rounded W^(1/2) times independently: 11 u of the sum's terms' size), whose errors the next operators pass on with a factor near one (norms
divide by the size of what they are given; decays, betas and gates have slopes of at most one).  Forward: 20 x 11 u x 4 (the largest of some thousand
values lies four deviations out) = 900 u = 5e-5 of the logits' spread.  Gradients pass as many operators again and take the forward values, twice that:
1e-4 of the largest entry of the parameter's gradient, and again as much for entries summed over all tokens whose terms cancel: 2e-4.
Slopes by differences: with steps e and 2 e, D(e) = slope + c e^2 + d e^4 + .., so that (4 D(e) - D(2 e)) / 3 = slope - 4 d e^4.  All parameters moving at once
by e = 1e-4 of their mean size are a long way: against the 64-bit formulas' own slope D(e) is off by 2.7e-4, the extrapolated value by 4e-5, which
leaves most of the gradients' 2e-4; the 64-bit losses' rounding, 1e-15 / 1e-4, is nothing.
bfloat16: activations are rounded at the same places the two ways, and differ where sums in another order round to a neighbour (2^-8), passed on
through 2 layers of residual sums: a few hundredths of the logits' spread; 0.1 is allowed."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "delta_language_model.py")
    spec = importlib.util.spec_from_file_location("delta_language_model", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.fixture(scope="module")
def g():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2510_03426_amd import Goom
    g = Goom(0)
    yield g
    g.close()


def _plain(p, frequencies, heads, layers, tokens):
    """The model's logits in 64 bits from its formulas, token after token; p: its parameters in their order."""
    import torch
    p = list(p)
    table, out = p[:2]
    names = ("norm", "qk", "unit", "v", "gate", "ab", "keep", "heads", "proj")
    blocks = [dict(zip(names, p[2 + 9 * i:])) for i in range(layers)]
    rms = lambda x: x / (x.square().mean(-1, keepdim=True) + 1e-5).sqrt()  # noqa: E731
    split = lambda x: x.unflatten(-1, (heads, -1))  # noqa: E731
    h = table[tokens]
    angle = torch.arange(tokens.shape[1], dtype=torch.float64)[:, None, None] * frequencies.double().cpu()
    cos, sin = angle.cos(), angle.sin()

    def turn(x):
        a, b = x.chunk(2, dim=-1)
        return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    for b in blocks:
        y = rms(h) * b["norm"]
        qk = (rms((y @ b["qk"].T).unflatten(-1, (2 * heads, -1))).flatten(-2) * b["unit"]).chunk(2, dim=-1)
        q, k = (turn(split(x)) for x in qk)
        v = split(y @ b["v"].T)
        a, beta = (y @ b["ab"].T).chunk(2, dim=-1)
        decay, beta = torch.sigmoid(a + b["keep"]), torch.sigmoid(beta)
        S, o = torch.zeros(tokens.shape[0], heads, q.shape[-1], v.shape[-1], dtype=torch.float64), []
        for t in range(tokens.shape[1]):
            S = decay[:, t, :, None, None] * S
            u = beta[:, t, :, None] * (v[:, t] - (k[:, t, :, None, :] @ S)[..., 0, :])
            S = S + k[:, t, :, :, None] * u[..., None, :]
            o.append((q[:, t, :, None, :] @ S)[..., 0, :])
        gate = y @ b["gate"].T
        h = h + (rms(torch.stack(o, 1)).flatten(-2) * b["heads"] * gate * torch.sigmoid(gate)) @ b["proj"].T
    return (rms(h) * p[-1]) @ out.T


def test_gradients_of_the_example(example, g):
    import torch
    from torch.nn.functional import cross_entropy
    heads, layers, vocab = 2, 2, 48
    model = example.Model(g, vocab, 64, heads, layers, torch.float32)
    tokens = torch.randint(0, vocab, (2, 70), generator=torch.Generator().manual_seed(3))
    loss_of = lambda logits: cross_entropy(logits[:, :-1].reshape(-1, vocab), tokens.to(logits.device)[:, 1:].reshape(-1))  # noqa: E731
    logits = model.forward(tokens.cuda())
    loss_of(logits).backward()
    params = [p.detach().double().cpu().requires_grad_() for p in model.parameters()]
    plain = lambda ps: _plain(ps, model.frequencies, heads, layers, tokens)  # noqa: E731
    want = plain(params)
    loss_of(want).backward()
    assert (logits.double().cpu() - want).abs().max() < 5e-5 * want.std()
    got = [p.grad.double().cpu() for p in model.parameters()]
    for i, (a, b) in enumerate(zip(got, params)):
        assert (a - b.grad).abs().max() <= 2e-4 * b.grad.abs().max(), i
    # slopes along the gradients' signs, by differences
    with torch.no_grad():
        way = [a.sign() * p.abs().mean() for a, p in zip(got, params)]
        once, twice = ((loss_of(plain([p + e * w for p, w in zip(params, way)])) - loss_of(plain([p - e * w for p, w in zip(params, way)]))) / (2 * e) for e in (1e-4, 2e-4))
        slope = sum((a * w).sum() for a, w in zip(got, way))
        assert abs((4 * once - twice) / 3 - slope) < 2e-4 * abs(slope)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_example_runs_and_decodes(example, dtype):
    off = example.main(["--steps", "3", "--type", dtype])
    assert off < (0.1 if dtype == "bf16" else 5e-5)


def _layer(g, x, res, gate, ld, beta, state, at, freq, heads):
    """One decoded token through a layer without projections: [batch, width] each; the state moves on in place."""
    width = x.shape[-1]
    y, h = g.norm_before(x, residual=res)
    qk = g.norm_after(y, heads)
    q, k = g.rotary(qk.view(-1, heads, width // heads), y.view(-1, heads, width // heads), at, freq)
    o = g.gated_delta_step(q, k, y.view(-1, heads, width // heads), ld, beta, state, scale=0.125)
    return g.norm_after(o.view(-1, width), heads, gate=gate, residual=h)


def test_two_graphs_of_one_handle(g):
    """A prompt's layer with its gradients and a decoded token's, each captured from one handle, replayed with eager calls between and then side by side
    on two streams: the same bits as eager calls."""
    import torch
    from paper_2510_03426_amd import Goom, rotary_frequencies
    heads, d, batch, n = 4, 32, 3, 200
    width = heads * d
    gen = torch.Generator(device="cuda").manual_seed(4)
    new = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    freq = rotary_frequencies(d // 2, device="cuda")[0]
    x, res, gate = (new(batch, width).bfloat16() for _ in range(3))
    ld, beta, at = -new(batch, heads).abs(), torch.sigmoid(new(batch, heads)), torch.arange(batch, device="cuda")
    px, pgate, go = (new(batch, n, width).bfloat16() for _ in range(3))
    pld, pbeta, pat = -new(batch, n, heads).abs() - 1, 0.02 * torch.sigmoid(new(batch, n, heads)), torch.arange(n, device="cuda").expand(batch, n).contiguous()

    def prompt(c):
        w = torch.ones(width, device="cuda")
        y, h, _, rs = c.norm_before(px, residual=pgate, weight=w, want_stats=True)
        q, k = c.rotary(y.view(batch, n, heads, d), h.view(batch, n, heads, d), pat, freq, interleaved=True)
        v = y.view(batch, n, heads, d)
        o, last = c.gated_delta(q, k, v, pld, pbeta, scale=0.1, want_state=True)
        z, _, ro = c.norm_after(o.view(batch, n, width), heads, weight=w, gate=pgate, residual=h, want_stats=True)
        gz, ggate, gw, _, _ = c.norm_after_backward(o.view(batch, n, width), go, None, ro, heads, weight=w, gate=pgate)
        gq, gk, gv, ga, gb, _ = c.gated_delta_backward(q, k, v, pld, pbeta, gz.view(batch, n, heads, d), scale=0.1)
        gq, gk = c.rotary_backward(gq, gk, pat, freq, interleaved=True)
        gx = c.norm_before_backward(h, h, (gq + gv).view(batch, n, width), None, rs, grad_h=gk.view(batch, n, width), weight=w)
        return [z, last, ggate, gw, ga, gb, gx[0], gx[3]]
    state = torch.zeros(batch, heads, d, d, device="cuda")
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], []
    with torch.cuda.stream(side):
        c = Goom(0, side)
        for call in (prompt, lambda c: [_layer(c, x, res, gate, ld, beta, state, at, freq, heads)]):
            call(c)
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                outs.append(call(c))
            graphs.append(graph)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    state.zero_()
    mine = torch.zeros_like(state)
    for i in range(4):
        x.mul_(1.25).add_(0.125)
        px.mul_(-0.75).add_(0.25)
        at.add_(1)
        torch.cuda.synchronize()
        if i < 2:
            graphs[0].replay()
            torch.cuda.synchronize()
            graphs[1].replay()
        else:
            for graph, stream in zip(graphs, (side, other)):
                with torch.cuda.stream(stream):
                    graph.replay()
        torch.cuda.synchronize()
        want = prompt(g), [_layer(g, x, res, gate, ld, beta, mine, at, freq, heads), mine]
        torch.cuda.synchronize()
        for got, w in zip((outs[0], outs[1] + [state]), want):
            assert all(torch.equal(a, b) for a, b in zip(got, w)), i
        assert all(bool(torch.isfinite(a.float()).all()) for a in outs[0])
    c.close()

"""The operators of a layer that forgets by its data where element offsets pass 32 bits: parts at both ends of the long tensors against the same parts
alone.  Tolerances: the parts may be cut into other segments, so that sums are taken in another order: two roundings to bfloat16 of values that differ by
float roundings, 2^-7 of the larger, and, near zero, 2^-7 of the outputs' spread; decays' and betas' gradients are floats: 2^-7 of the spread."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def g():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2510_03426_amd import Goom
    g = Goom(0)
    yield g
    g.close()
    torch.cuda.empty_cache()


def _close(a, b):
    import torch
    a, b = a.float(), b.float()
    assert bool(((a - b).abs() <= 2.0 ** -7 * torch.maximum(a.abs(), b.std())).all()), float((a - b).abs().max())


def test_gated_delta_and_rotary(g):
    import torch
    from paper_2510_03426_amd import rotary_frequencies
    n, H, d = 540000, 64, 128  # 4.4e9 elements of v
    assert n * H * d > 2 ** 32
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k = (torch.nn.functional.normalize(torch.empty(n, 4, 32, dtype=torch.bfloat16, device="cuda").normal_(generator=gen), dim=-1) for _ in range(2))
    v, do = (torch.empty(n, H, d, dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(2))
    ld = -0.2 * torch.rand(n, H, device="cuda", generator=gen)
    beta = torch.rand(n, H, device="cuda", generator=gen)
    offsets = torch.tensor([0, 1000, n - 60000, n - 700, n], device="cuda")  # (tokens 1000 .. are a long sequence of one more)
    o = g.gated_delta(q, k, v, ld, beta, offsets=offsets)
    ends = slice(0, 1000), slice(n - 700, n)
    for part in ends:
        _close(o[part], g.gated_delta(*(t[part].contiguous()[None] for t in (q, k, v, ld, beta)))[0])
    del o
    grads = g.gated_delta_backward(q, k, v, ld, beta, do, offsets=offsets)[:5]
    for part in ends:
        want = g.gated_delta_backward(*(t[part].contiguous()[None] for t in (q, k, v, ld, beta, do)))
        for a, b in zip(grads, want):
            _close(a[part], b[0])
    del grads, do
    at, freq = torch.arange(n, device="cuda"), rotary_frequencies(d // 2, device="cuda")[0]
    turned = g.rotary(v, None, at, freq)[0]
    for part in ends:
        assert torch.equal(turned[part], g.rotary(v[part].contiguous(), None, at[part], freq)[0])


def test_block_norm(g):
    import torch
    C, tokens = 4096, 1100000
    assert tokens * C > 2 ** 32
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, gate = (torch.empty(tokens, C, dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(2))
    kw = dict(groups=32, kind="layer")
    y, mean, rstd = g.norm_after(x, gate=gate, want_stats=True, **kw)
    gx, ggate = g.norm_after_backward(x, y, mean, rstd, gate=gate, **kw)[:2]
    z, h = g.norm_before(x, residual=gate, **kw)
    for part in (slice(0, 3), slice(tokens - 3, tokens)):
        p, t, dy = x[part], gate[part], y[part]
        a, m, r = g.norm_after(p, gate=t, want_stats=True, **kw)
        assert torch.equal(a, y[part])
        for one, whole in zip(g.norm_after_backward(p, dy, m, r, gate=t, **kw), (gx, ggate)):
            assert torch.equal(one, whole[part])
        for one, whole in zip(g.norm_before(p, residual=t, **kw), (z, h)):
            assert torch.equal(one, whole[part])

"""The layer operators where element offsets pass 32 bits: parts at both ends of the long tensors against the same parts alone.
Tolerances: the parts are computed with other segment lengths, so sums are taken in another order: two roundings to bfloat16 of values
that differ by float roundings, 2^-7 of the larger, and, near zero, 2^-7 of the outputs' spread."""
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


def test_linear_attention(g):
    import torch
    n, H, d = 540000, 64, 128  # 4.4e9 elements a tensor
    assert n * H * d > 2 ** 32
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v, do = (torch.empty(n, H, d, dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(4))
    ld = torch.linspace(-0.5, -0.02, H, device="cuda")
    offsets = torch.tensor([0, 1000, n - 700, n], device="cuda")
    o = g.linear_attention(q, k, v, ld, offsets=offsets)
    grads = g.linear_attention_backward(q, k, v, ld, do, offsets=offsets)[:3]
    for part in (slice(0, 1000), slice(n - 700, n)):
        args = [t[part].contiguous()[None] for t in (q, k, v)]
        _close(o[part], g.linear_attention(*args, ld)[0])
        for a, b in zip(grads, g.linear_attention_backward(*args, ld, do[part].contiguous()[None])):
            _close(a[part], b[0])


def test_group_norm(g):
    import torch
    C = 4096
    for items, length in ((1100000, 1), (1100, 1000)):
        assert items * length * C > 2 ** 32
        gen = torch.Generator(device="cuda").manual_seed(2)
        x = torch.empty(items, length, C, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
        y, mean, rstd = g.group_norm(x, 32, activation="silu", want_stats=True)
        gx = g.group_norm_backward(x, y, mean, rstd, 32, activation="silu")[0]
        for part in (slice(0, 3), slice(items - 3, items)):
            z, m, r = g.group_norm(x[part].contiguous(), 32, activation="silu", want_stats=True)
            _close(y[part], z)
            _close(gx[part], g.group_norm_backward(x[part].contiguous(), z, m, r, 32, activation="silu")[0])
        del x, y, gx


def test_embedding(g):
    import torch
    n, width, vocab = 4300000, 1000, 1000
    assert n * width > 2 ** 32
    table = torch.arange(vocab, device="cuda", dtype=torch.float32)[:, None].bfloat16().repeat(1, width)
    tokens = torch.arange(n, device="cuda") % vocab
    rows = g.embedding(table, tokens)
    assert torch.equal(rows[-vocab:], table) and torch.equal(rows[:vocab], table)
    rows.fill_(1.0)
    rows[-1] = 2.0  # (the last token's)
    grad = g.embedding_backward(tokens, rows, vocab, dtype=torch.float32)
    want = torch.full((vocab, width), float(n // vocab), device="cuda")
    want[(n - 1) % vocab] += 1.0
    assert torch.equal(grad, want)

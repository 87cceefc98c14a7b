"""Token embeddings and their gradient against plain sums in 64 bits.  Tolerances, u = 2^-24: a row is one product, rounded to a
float and then to the type; a token's gradient is a sum of k floats in a fixed order, at most k u relative to the sum of their
magnitudes, times the scale (u), rounded to the type (2^-8 bfloat16, 2^-11 half)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
ROUND = {"f32": U, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


@pytest.fixture(scope="module")
def g():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2510_03426_amd import Goom
    g = Goom(0)
    yield g
    g.close()


def _types():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _tokens(kind, n, vocab, rng):
    if kind == "uniform":
        return rng.integers(0, vocab, n)
    if kind == "frequent":  # a few tokens take most positions
        return np.minimum((vocab ** rng.random(n)).astype(np.int64), vocab) - 1
    if kind == "one":
        return np.full(n, vocab - 1)
    t = rng.integers(-3, vocab + 3, n)  # some outside
    t[::7] = -(2 ** 40)
    t[::11] = 2 ** 40
    return t


@pytest.mark.parametrize("dtype,gtype", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("kind,n,vocab,width", [("uniform", 1, 5, 1), ("uniform", 1, 60000, 8), ("uniform", 300, 1000, 33), ("outside", 500, 70, 20), ("frequent", 3000, 50257, 6), ("one", 1000, 3, 130),
                                                ("frequent", 5000, 300, 264), ("uniform", 64, 1, 16), ("outside", 2048, 700000, 2)])
def test_rows_and_gradient(g, dtype, gtype, kind, n, vocab, width):
    import torch
    from oracle import layer_oracle as lo
    rng = np.random.default_rng(n + width)
    t = _tokens(kind, n, vocab, rng)
    scale = -1.75
    table = torch.from_numpy(rng.standard_normal((vocab, width)).astype(np.float32)).to(_types()[dtype])
    grad = torch.from_numpy(rng.standard_normal((n, width)).astype(np.float32)).to(_types()[dtype])
    tokens = torch.from_numpy(t).cuda()
    rows = g.embedding(table.cuda(), tokens, scale=scale).double().cpu().numpy()
    want = lo.embedding(table.double().numpy(), t, scale)
    assert (np.abs(rows - want) <= (ROUND[dtype] + U) * np.abs(want) + (2.0 ** -25 if dtype == "f16" else 0)).all()
    out = g.embedding_backward(tokens, grad.cuda(), vocab, scale=scale, dtype=_types()[gtype])
    assert out.dtype == _types()[gtype]
    want = lo.embedding_backward(t, grad.double().numpy(), vocab, scale)
    mag = lo.embedding_backward(t, np.abs(grad.double().numpy()), vocab, abs(scale))
    count = np.bincount(t[(t >= 0) & (t < vocab)], minlength=vocab)[:, None]
    tol = ROUND[gtype] * np.abs(want) + (count + 1) * U * mag + (2.0 ** -25 if gtype == "f16" else 0)
    got = out.double().cpu().numpy()
    assert (np.abs(got - want) <= tol).all(), np.argwhere(~(np.abs(got - want) <= tol))[:3]
    assert torch.equal(out, g.embedding_backward(tokens, grad.cuda(), vocab, scale=scale, dtype=_types()[gtype]))  # a fixed order


@pytest.mark.parametrize("n", [31, 256, 257, 4095, 4096, 4097, 65536, 65537, 200001])
def test_many_positions(g, n):
    """Whole numbers, whose sums are exact in any order: every position has to be counted once."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(n)
    vocab = 5003
    tokens = torch.exp(torch.rand(n, device="cuda", generator=gen, dtype=torch.float64) * np.log(vocab)).long().clamp(1, vocab) - 1
    grad = torch.randint(-8, 9, (n, 4), device="cuda", generator=gen).float()
    want = torch.zeros(vocab, 4, device="cuda", dtype=torch.float64).index_add_(0, tokens, grad.double())
    assert torch.equal(g.embedding_backward(tokens, grad, vocab).double(), want)
    if n > 65000:  # and with three sorting passes
        wide = tokens * 60
        assert torch.equal(g.embedding_backward(wide, grad, 60 * vocab)[::60].double(), want)


def test_odd_addresses_and_nothing(g):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(5)
    flat = torch.randn(20 * 16 + 1, device="cuda", generator=gen).bfloat16()
    table, tokens = flat[1:].view(20, 16), torch.arange(19, -1, -1, device="cuda").view(4, 5)
    assert torch.equal(g.embedding(table, tokens), table.flip(0).view(4, 5, 16))
    assert torch.equal(g.embedding_backward(tokens, table.view(4, 5, 16), 20), table.flip(0))
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    assert g.embedding(table, none).shape == (0, 16)
    assert torch.equal(g.embedding_backward(none, torch.empty(0, 16, device="cuda"), 7), torch.zeros(7, 16, device="cuda"))


def test_a_nan_stays_with_its_token(g):
    import torch
    tokens = torch.tensor([1, 2, 1, 0], device="cuda")
    grad = torch.ones(4, 8, device="cuda")
    grad[1, 3] = float("nan")
    out = g.embedding_backward(tokens, grad, 4)
    assert out[2, 3].isnan() and out.isnan().sum() == 1 and torch.equal(out[:2], torch.tensor([[1.0], [2.0]], device="cuda").expand(2, 8))

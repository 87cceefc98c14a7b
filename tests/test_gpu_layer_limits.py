"""The layer operators where a launch has more threads than 32 bits count along one axis of a grid.  Whole numbers, whose sums are exact,
or parts of a large call against the same parts alone."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def g():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2510_03426_amd import Goom
    g = Goom(0)
    yield g
    g._ws = None
    g.close()
    torch.cuda.empty_cache()


@pytest.mark.parametrize("vocab", [(1 << 26) + 3, (1 << 31) - 1])
@pytest.mark.parametrize("n", [100, 1000])
def test_tables_of_many_rows(g, n, vocab):
    """A wave for every table row: 2^32 threads from 2^26 rows on.  Up to 256 positions take one launch, more the sort and the runs."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(n)
    tokens = torch.randint(0, vocab, (n,), device="cuda", generator=gen)
    tokens[:50] = vocab - 1
    tokens[50:60] = 0
    tokens[60:70] = (1 << 26) + 1
    grad = torch.randint(1, 9, (n, 1), device="cuda", generator=gen).float()
    out = g.embedding_backward(tokens, grad, vocab, dtype=torch.bfloat16)[:, 0]
    rows, at = tokens.unique(return_inverse=True)
    want = torch.zeros(rows.numel(), device="cuda").index_add_(0, at, grad[:, 0])
    assert torch.equal(out[rows], want.bfloat16())
    assert int((out != 0).sum()) == rows.numel()


def test_group_norm_gradient_of_many_groups(g):
    """A workgroup for the means of every item and group: 2^24 of them are 2^32 threads."""
    import torch
    items, length, C = 9 * 8192, 513, 256
    x = torch.empty(items, length, C, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(4))
    _, mean, rstd = g.group_norm(x, C, activation="silu", want_stats=True)
    gx, gw, _ = g.group_norm_backward(x, x, mean, rstd, C, activation="silu")
    total = torch.zeros(C, dtype=torch.float64, device="cuda")
    for a in range(0, items, 8192):
        part = x[a:a + 8192]
        px, pw, _ = g.group_norm_backward(part, part, mean[a:a + 8192], rstd[a:a + 8192], C, activation="silu")
        assert torch.equal(px, gx[a:a + 8192])
        total += pw.double()
    assert torch.allclose(gw.double(), total, rtol=1e-5)


def test_linear_attention_of_many_short_sequences(g):
    """2^20 sequences of one token and 16 heads of one entry: three walks each, 2^32.6 threads.  One token: o = scale q (k v + decay s), and
    the gradients are products of the others, all of small whole numbers and exact."""
    import torch
    n, H = 1 << 20, 16
    gen = torch.Generator(device="cuda").manual_seed(6)
    q, k, v, do, s0, ds = (torch.randint(-3, 4, (n, 1, H, 1), device="cuda", generator=gen).float() for _ in range(6))
    ld = torch.zeros(H, device="cuda")
    state, dstate = s0.reshape(n, H, 1, 1), ds.reshape(n, H, 1, 1)
    o, last = g.linear_attention(q, k, v, ld, state=state, scale=2.0, want_state=True)
    assert torch.equal(last.reshape(q.shape), k * v + s0) and torch.equal(o, 2 * q * (k * v + s0))
    gq, gk, gv, gs = g.linear_attention_backward(q, k, v, ld, do, state=state, grad_state=dstate, scale=2.0)
    u = 2 * q * do + ds  # the state's adjoint
    assert torch.equal(gq, 2 * do * (k * v + s0)) and torch.equal(gk, u * v) and torch.equal(gv, u * k) and torch.equal(gs.reshape(q.shape), u)


def test_linear_attention_past_32_bit_offsets(g):
    """The last of 4.3e9 elements against the recurrence in 64 bits, with the tolerances of test_gpu_linear_attention.py."""
    import numpy as np
    import torch
    from oracle import layer_oracle as lo
    from test_gpu_linear_attention import _f64, _near
    n, H, d, T = 530000, 64, 128, 300
    assert (n - T) * H * d > 2 ** 32
    gen = torch.Generator(device="cuda").manual_seed(8)
    q, k, v, do = (torch.empty(n, H, d, dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(4))
    ld = torch.linspace(-0.5, -0.02, H, device="cuda")
    offsets = torch.tensor([0, 1000, n - T, n], device="cuda")
    o = g.linear_attention(q, k, v, ld, offsets=offsets)
    grads = g.linear_attention_backward(q, k, v, ld, do, offsets=offsets)[:3]
    args = [_f64(x[n - T:]) for x in (q, k, v)]
    mags = [np.abs(x) for x in args]
    terms = d + 64 + T // 64 + 32
    _near(o[n - T:], lo.attention(*args, _f64(ld))[0], lo.attention(*mags, _f64(ld))[0], "bf16", terms, False, "o")
    want, mag = lo.attention_backward(*args, _f64(ld), _f64(do[n - T:])), lo.attention_backward(*mags, _f64(ld), np.abs(_f64(do[n - T:])))
    for name, got, w, m in zip(("grad_q", "grad_k", "grad_v"), grads, want, mag):
        _near(got[n - T:], w, m, "bf16", terms, False, name)

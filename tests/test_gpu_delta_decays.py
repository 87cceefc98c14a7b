"""The gated delta rule's decays by themselves: with beta = 0 a state is its initial one times all decays so far, entry by entry, and a token's output the
query times that.

Tolerances, u = 2^-24, relative to each entry.  A decay's exponent is a product and a sum in 64 bits; its whole part scales exactly, its fraction is rounded to
2^-25 of log 2 (u / 3), the hardware's exponential is off by at most one unit of the last place (2 u), a product with the state rounds once (u): 4 u a factor.  In a step the state has one factor.
Through chunks it has one for each chunk, of operands in three bf16 parts (24 bits, u more each): 6 u a chunk.  Segments' maps are products with sums of zeros: as many more."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def g():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2510_03426_amd import Goom
    g = Goom(0)
    yield g
    g.close()


def _case(n, H, d, dtype, seed):
    import torch
    gen = torch.Generator().manual_seed(seed)
    q, k, v = (torch.randn(n, H, d, generator=gen).to(dtype) for _ in range(3))
    state = 1 + torch.rand(n, H, d, d, generator=gen)
    return q, k, v, state


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_step(g, dtype):
    """log_decay from -5 to -60 (and the ends of the range of floats): every entry of the next state to a few units of itself."""
    import torch
    t = getattr(torch, dtype)
    ld = torch.cat([-torch.linspace(5, 60, 200), -torch.rand(50) * 80, torch.tensor([0.0, 0.5, 3.0, 30.0, -1e-6, -80.0, -87.0])]).reshape(-1, 1)
    n, H, d = len(ld), 1, 24
    q, k, v, state = _case(n, H, d, t, 1)
    zero = torch.zeros(n, H)
    out = torch.empty_like(state).cuda()
    o = g.gated_delta_step(q.cuda(), k.cuda(), v.cuda(), ld.cuda(), zero.cuda(), state.cuda(), scale=0.7, out_state=out)
    want = np.exp(ld.double().numpy())[:, :, None, None] * state.double().numpy()
    assert (np.abs(out.double().cpu().numpy() - want) <= 4 * U * want).all()
    terms = q.double().numpy()[:, :, :, None] * want
    size = 0.7 * np.abs(terms).sum(2)
    tol = (d + 8) * U * size + torch.finfo(t).eps / 2 * np.abs(0.7 * terms.sum(2)) + (2.0 ** -25 if dtype == "float16" else 0)
    got, want = o.double().cpu().numpy(), 0.7 * terms.sum(2)
    beyond = np.abs(want) >= 65520 if dtype == "float16" else np.zeros(want.shape, bool)  # (e^30 times a number is none of a half's, whose last is 65504: infinity)
    assert ((np.abs(got - want) <= tol) | (beyond & (got == np.copysign(math.inf, want)))).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,rate", [(1, 20.0), (1, 60.0), (7, 9.0), (40, 1.5), (64, 1.25), (100, 0.7), (700, 0.1)])
def test_chunks(g, dtype, n, rate):
    import torch
    t = getattr(torch, dtype)
    H, d = 3, 32
    q, k, v, state = _case(n, H, d, t, n)
    state = state[:1]
    gen = torch.Generator().manual_seed(n)
    ld = -rate * (0.5 + torch.rand(1, n, H, generator=gen))
    b = np.cumsum(ld.double().numpy()[0], 0)  # [n, H]
    o, last = g.gated_delta(*(x[None].cuda() for x in (q, k, v)), ld.cuda(), torch.zeros(1, n, H).cuda(), state=state.cuda(), scale=0.7, want_state=True)
    chunks = -(-n // 32) + 1
    want = np.exp(b[-1])[:, None, None] * state.double().numpy()[0]
    assert want.min() > 1e-37
    assert (np.abs(last.double().cpu().numpy()[0] - want) <= 12 * chunks * U * want).all()
    terms = 0.7 * q.double().numpy()[:, :, :, None] * np.exp(b)[:, :, None, None] * state.double().numpy()
    tol = (12 * chunks + d + 8) * U * np.abs(terms).sum(2) + torch.finfo(t).eps / 2 * np.abs(terms.sum(2))
    assert (np.abs(o.double().cpu().numpy()[0] - terms.sum(2)) <= tol).all()


def test_what_is_forgotten_and_what_is_not(g):
    """Decays at and beyond the ends: zero below -110; infinity far above, which times a beta of zero is NaN in the formula itself (beta (v - a k . S)); NaN for NaN."""
    import torch
    ld = torch.tensor([-math.inf, -3e38, -111.0, -120.0, 0.0, 200.0, 3e38, math.inf, math.nan]).reshape(-1, 1)
    n, d = len(ld), 8
    q, k, v, state = _case(n, 1, d, torch.float32, 2)
    k = k * 0 + 1
    out = torch.empty_like(state).cuda()
    g.gated_delta_step(q.cuda(), k.cuda(), v.cuda(), ld.cuda(), torch.zeros(n, 1).cuda(), state.cuda(), out_state=out)
    out = out.cpu()
    assert (out[:4] == 0).all() and torch.equal(out[4], state[4]) and not out[5:].isfinite().any()


@pytest.mark.parametrize("dtype,n,rate,dk,dv", [("bfloat16", 64, 1.2, 64, 64), ("float32", 32, 2.4, 32, 40), ("float16", 20, 0.3, 50, 20), ("float32", 200, 0.4, 128, 128), ("bfloat16", 700, 0.11, 32, 32), ("bfloat16", 3, 25.0, 16, 16)])
def test_growing_decays(g, dtype, n, rate, dk, dv):
    """Decays above one, up to e^80 in all.  An error grows as the decays' product from where it is made, by matrices a (I - beta k k^T) of norms of at most a:
    E_t = max(a_t E_{t-1}, S_t + |v_t|) stands for the largest state in test_gpu_gated_delta.py's bound, twelve random roundings of sums of dk + 136 terms a token.
    Pairs' weights round their exponents: half a unit of b - b' <= 116 bits, 116 u log 2 = 80 u of a weight, less than the 12 sqrt(dk + 136) >= 147 u that are allowed for a single token.
    Gradients: finite, and within four such bounds, over all entries of a state, of the largest of their kind."""
    import torch
    from oracle import layer_oracle as lo
    t = getattr(torch, dtype)
    gen = torch.Generator().manual_seed(n)
    H = 2
    q, k, v, go = (torch.randn(1, n, H, d, generator=gen) for d in (dk, dk, dv, dv))
    q, k = (torch.nn.functional.normalize(x, dim=-1) for x in (q, k))
    q, k, v, go = (x.to(t) for x in (q, k, v, go))
    ld, beta = rate * (1 - 0.1 * torch.rand(1, n, H, generator=gen)), torch.rand(1, n, H, generator=gen)
    scale = 1e-3 if dtype == "float16" else 1.0  # (halves end at 65504)
    f = lambda x: x.double().numpy()[0]  # noqa: E731
    o, last = g.gated_delta(*(x.cuda() for x in (q, k, v, ld, beta)), scale=scale, want_state=True)
    E, S, share = np.zeros((n, H)), np.zeros((H, dk, dv)), np.arange(H)
    for i in range(n):
        S = lo._delta_step(S, f(k)[i], f(v)[i], f(ld)[i], f(beta)[i])[0]
        E[i] = np.maximum(np.exp(f(ld)[i]) * E[i - 1] if i else 0, np.sqrt((S * S).sum((1, 2))) + np.linalg.norm(f(v)[i], axis=-1))
    want, wl, _ = lo.gated_delta(*(f(x) for x in (q, k, v, ld, beta)), None, None, scale)
    err = 12 * U * math.sqrt(n * (dk + 136.0))
    qn = np.linalg.norm(f(q), axis=-1)
    assert (np.abs(f(o.cpu()) - want) <= torch.finfo(t).eps / 2 * np.abs(want) + err * scale * (qn * E)[..., None] + 2.0 ** -25).all()
    assert (np.abs(last.double().cpu().numpy()[0] - wl[0]) <= err * E[-1][:, None, None]).all()
    grads = g.gated_delta_backward(*(x.cuda() for x in (q, k, v, ld, beta, go)), scale=scale)[:5]
    wants = lo.gated_delta_backward(*(f(x) for x in (q, k, v, ld, beta, go)), scale=scale)[:5]
    for name, y, w in zip(("q", "k", "v", "log_decay", "beta"), grads, wants):
        y, most = f(y.cpu()), np.abs(w).max()
        assert np.isfinite(y).all(), name
        assert np.abs(y - w).max() <= (torch.finfo(t).eps / 2 if name in "qkv" else 0) * most + 4 * err * math.sqrt(dk * dv) * most, name

"""The gated delta rule's gradients against the recurrence's adjoint in 64 bits, every one within a small part of itself: for each head, and within it for each 32
tokens, the norm of what a gradient is off by against bounds made of the states, adjoints and rows that stand in that token's formula.

Tolerances, u = 2^-24.  After n tokens a state's and an adjoint's error has a norm of err = 12 u sqrt(n (dk + 136)) of theirs (the derivation in test_gpu_gated_delta.py:
sums of dk products, the solve's 2 x 64 terms and eight roundings a token, at random, by matrices of norms of at most one).  These errors are sums of roundings of their own in every entry,
so that a row of a gradient, the error times a vector, has err / sqrt(m), m = min(dk, dv), of the product of the norms; the twelve in err is the allowance for what is not that even.  The rows, S and D being norms of the state and its adjoint, e and w
the value's and the output's rows:
    grad_q = scale S' do: |scale| S' |do|,   grad_v = beta w, w = D^T k: |beta| D |k|,   grad_beta = w . e: D |k| |e| + |w| (|v| + a S |k|),
    grad_k = D beta e - a S grad_v: |beta| D (|e| + |v| + a S |k|) + a S (|grad_v| + |beta| D |k|),
    grad_log_decay, sums over the rest of a chunk of q . grad_q - v . grad_v and <D, S> at its end: these rows' bounds times |q| and |v|, in squares, and D S.
What is stored in 16 bits is rounded once more, eps / 2 of itself.  Every bound must be below 1 % of the gradient's own norm, that of the decays' (whose sums cancel where
decays are strong) below 15 %, which is asserted: zeros, and a term left out, are far outside."""
import math

import numpy as np
import pytest

from test_gpu_gated_delta import HALF, U, _f64, _inputs, _torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def g():
    torch, _ = _torch()
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2510_03426_amd import Goom
    g = Goom(0)
    yield g
    g.close()


def _rows(r, spans, scale, chunk):
    """The bounds' sizes [tokens, H] of every gradient, by the recurrence, and the sequences' adjoints' norms."""
    q, k, v, ld, be, go = (r[x] for x in ("q", "k", "v", "log_decay", "beta", "grad_o"))
    n, H, _ = v.shape
    share = np.arange(H) // (H // q.shape[1])
    vec, mat = (lambda x: np.sqrt((x * x).sum(-1))), (lambda x: np.sqrt((x * x).sum((-1, -2))))
    z = {x: np.zeros((n, H)) for x in "qkvab"}
    first = np.zeros((len(spans) - 1, H))
    for s, (a, b) in enumerate(zip(spans[:-1], spans[1:])):
        S, D = r["state"][s], r["grad_state"][s]
        states, errors = [S], []
        for t in range(a, b):
            S = np.exp(ld[t])[:, None, None] * S
            errors.append(v[t] - np.einsum("hk,hkv->hv", k[t, share], S))
            S = S + k[t, share][:, :, None] * (be[t][:, None] * errors[-1])[:, None]
            states.append(S)
        for t in range(b - 1, a - 1, -1):
            if (t - a) % chunk == chunk - 1 or t == b - 1:  # a chunk's end
                rest, end = 0.0, mat(D) * mat(states[t - a + 1])
            kk, qq, e, beta, decay = k[t, share], q[t, share], errors[t - a], np.abs(be[t]), np.exp(ld[t])
            D = D + scale * qq[:, :, None] * go[t][:, None]
            w = np.einsum("hk,hkv->hv", kk, D)
            S, old = mat(states[t - a + 1]), decay * mat(states[t - a])
            z["q"][t] = abs(scale) * S * vec(go[t])
            z["v"][t] = beta * mat(D) * vec(kk)
            z["b"][t] = mat(D) * vec(kk) * vec(e) + vec(w) * (vec(v[t]) + old * vec(kk))
            z["k"][t] = beta * mat(D) * (vec(e) + vec(v[t]) + old * vec(kk)) + old * (beta * vec(w) + z["v"][t])
            rest = rest + (vec(qq) * z["q"][t]) ** 2 + (vec(v[t]) * z["v"][t]) ** 2
            z["a"][t] = np.sqrt(rest) + end
            D = decay[:, None, None] * (D - kk[:, :, None] * (be[t][:, None] * w)[:, None])
        first[s] = mat(D)
    return z, first


def _norms(x, heads, spans):
    """[tokens, heads, ...] -> squares' sums of each head over 32 tokens of a sequence, and over everything."""
    x = (x * x).reshape(len(x), heads, -1).sum(-1)
    at = sorted({t for a, b in zip(spans[:-1], spans[1:]) for t in range(a, b, 32)} | set(spans))
    parts = np.array([x[a:b].sum(0) for a, b in zip(at[:-1], at[1:])])
    return np.sqrt(parts), np.sqrt(x.sum(0))


@pytest.mark.parametrize("dtype,n,H,Q,dk,dv,offsets,scale", [
    ("bf16", 1500, 1, 1, 64, 40, None, 1.0), ("f32", 1500, 1, 1, 64, 40, None, 1.0), ("f16", 1500, 1, 1, 64, 40, None, 1.0),
    ("bf16", 1300, 2, 1, 100, 100, [0, 700, 700, 705, 1300], 1.0), ("f32", 1300, 2, 1, 100, 100, [0, 700, 700, 705, 1300], 1.0),
    ("f16", 1300, 2, 1, 100, 100, [0, 700, 700, 705, 1300], 1.0),
    ("bf16", 140, 4, 2, 128, 128, None, 128 ** -0.5), ("f32", 70, 4, 2, 128, 128, None, 128 ** -0.5), ("f16", 97, 3, 3, 128, 72, None, 0.3),
    ("f32", 600, 2, 2, 32, 64, None, 1.0), ("bf16", 400, 6, 3, 32, 32, [0, 3, 64, 64, 200, 400], 0.5), ("f32", 130, 4, 4, 50, 72, [0, 33, 130], -0.7),
    ("bf16", 2100, 1, 1, 128, 64, None, 0.1), ("f32", 2100, 1, 1, 128, 128, None, 0.1)])
def test_gradients_within_a_small_part_of_themselves(g, dtype, n, H, Q, dk, dv, offsets, scale):
    torch, _ = _torch()
    from oracle import layer_oracle as lo
    spans = offsets or [0, n]
    x = _inputs(dtype, n, H, Q, dk, dv, len(spans) - 1, seed=n + dk)
    r = {name: _f64(t) for name, t in x.items()}
    names = ("q", "k", "v", "log_decay", "beta")
    *want, _ = lo.gated_delta_backward(*[r[a] for a in names + ("grad_o", "state", "grad_state")], spans, scale)
    z, first = _rows(r, spans, scale, 64 if dtype == "bf16" else 32)
    err = 12 * U * math.sqrt(max(np.diff(spans)) * (dk + 136.0)) / math.sqrt(min(dk, dv))
    dev = {name: t.cuda() for name, t in x.items()}
    if offsets:
        off = torch.tensor(offsets, dtype=torch.int64).cuda()
    else:
        off, dev = None, {name: t if "state" in name else t[None] for name, t in dev.items()}
    got = g.gated_delta_backward(*[dev[a] for a in names], dev["grad_o"], state=dev["state"], grad_state=dev["grad_state"], offsets=off, scale=scale)
    for name, heads, size, y, w in zip(("grad_q", "grad_k", "grad_v", "grad_log_decay", "grad_beta"), (Q, Q, H, H, H), "qkvab", got, want):
        y = _f64(y).reshape(w.shape)
        s = np.sqrt((z[size] ** 2).reshape(n, heads, H // heads).sum(-1))
        rounding = HALF[dtype if size in "qkv" else "f32"]
        (part_off, all_off), (part_want, all_want), (part_size, all_size) = (_norms(v, heads, spans) for v in (y - w, w, s))
        assert (err * all_size <= (0.15 if size == "a" else 0.01) * all_want).all(), f"{name}: the bound is {(err * all_size / all_want).max():.2g} of the gradient"
        worst = max((part_off / (err * part_size + rounding * part_want)).max(), (all_off / (err * all_size + rounding * all_want)).max())
        print(f"{name} {dtype} {n} {dk}x{dv}: {worst:.3f} of the tolerance, {(all_off / all_want).max():.2e} of the gradient")
        assert worst <= 1, name
    y, w = _f64(got[5]), want[5]
    off_by, size = (np.sqrt((v * v).sum((-1, -2))) for v in (y - w, w))
    assert (off_by <= err * math.sqrt(min(dk, dv)) * np.maximum(first, np.sqrt((r["grad_state"] ** 2).sum((-1, -2)))) + U * size).all()

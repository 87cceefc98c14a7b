"""Plain 64-bit implementations of the layer operators (linear attention with decay, group norm with an activation, embeddings),
from their formulas, in numpy: test infrastructure.  Nothing here is shared with the library."""
import math

import numpy as np


# ---- linear attention with a decay for each head, token after token

def _spans(n, offsets):
    return [(0, n)] if offsets is None else list(zip(offsets[:-1], offsets[1:]))


def attention(q, k, v, log_decay, state=None, offsets=None, scale=1.0):
    """q: [tokens, H, dk], k: [tokens, G, dk], v: [tokens, G, dv], state: [sequences, H, dk, dv]; returns (o, final states)."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    n, H, dk = q.shape
    G, dv = v.shape[1:]
    share = np.arange(H) // (H // G)
    gamma = np.exp(np.asarray(log_decay, dtype=np.float64))[:, None, None]
    spans = _spans(n, offsets)
    o = np.zeros((n, H, dv))
    last = np.zeros((len(spans), H, dk, dv))
    for s, (a, b) in enumerate(spans):
        S = np.zeros((H, dk, dv)) if state is None else np.array(state[s], dtype=np.float64)
        for t in range(a, b):
            S = gamma * S + k[t, share][:, :, None] * v[t, share][:, None, :]
            o[t] = scale * np.einsum("hk,hkv->hv", q[t], S)
        last[s] = S
    return o, last


def attention_backward(q, k, v, log_decay, grad_o, state=None, grad_state=None, offsets=None, scale=1.0):
    """Adjoints of the recurrence, walked backwards: returns (grad_q, grad_k, grad_v, grad_state or None)."""
    q, k, v, grad_o = (np.asarray(x, dtype=np.float64) for x in (q, k, v, grad_o))
    n, H, dk = q.shape
    G, dv = v.shape[1:]
    share = np.arange(H) // (H // G)
    gamma = np.exp(np.asarray(log_decay, dtype=np.float64))[:, None, None]
    spans = _spans(n, offsets)
    gq, gk, gv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    gs = np.zeros((len(spans), H, dk, dv))
    for s, (a, b) in enumerate(spans):
        S = np.zeros((H, dk, dv)) if state is None else np.array(state[s], dtype=np.float64)
        states = []
        for t in range(a, b):
            S = gamma * S + k[t, share][:, :, None] * v[t, share][:, None, :]
            states.append(S)
        adj = np.zeros((H, dk, dv)) if grad_state is None else np.array(grad_state[s], dtype=np.float64)
        for t in range(b - 1, a - 1, -1):
            gq[t] = scale * np.einsum("hkv,hv->hk", states[t - a], grad_o[t])
            adj = adj + scale * q[t][:, :, None] * grad_o[t][:, None, :]
            np.add.at(gk[t], share, np.einsum("hkv,hv->hk", adj, v[t, share]))
            np.add.at(gv[t], share, np.einsum("hkv,hk->hv", adj, k[t, share]))
            adj = gamma * adj
        gs[s] = adj
    return gq, gk, gv, gs if state is not None else None


# ---- group norm with an activation, channels last

_erf = np.vectorize(math.erf, otypes=[np.float64])


def activation(z, act):
    """Value and derivative."""
    if act == "silu":
        p = 0.5 * (1 + np.tanh(0.5 * z))
        return z * p, p + z * p * (1 - p)
    if act == "gelu":
        p = 0.5 * (1 + _erf(z / math.sqrt(2)))
        return z * p, p + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return z, np.ones_like(z)


def group_norm(x, groups, weight, bias, eps, act):
    """x: [items, length, channels]; returns (y, mean, rstd)."""
    x = np.asarray(x, dtype=np.float64)
    n, L, C = x.shape
    xg = x.reshape(n, L, groups, C // groups)
    mean = xg.mean(axis=(1, 3))
    var = ((xg - mean[:, None, :, None]) ** 2).mean(axis=(1, 3))
    rstd = 1 / np.sqrt(var + eps)
    z = ((xg - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(n, L, C)
    z = z * (1.0 if weight is None else np.asarray(weight, np.float64)) + (0.0 if bias is None else np.asarray(bias, np.float64))
    return activation(z, act)[0], mean, rstd


def group_norm_backward(x, grad_y, groups, weight, bias, eps, act):
    """Returns (grad_x, grad_weight, grad_bias)."""
    x, grad_y = (np.asarray(t, dtype=np.float64) for t in (x, grad_y))
    n, L, C = x.shape
    _, mean, rstd = group_norm(x, groups, None, None, eps, "none")
    w = np.ones(C) if weight is None else np.asarray(weight, np.float64)
    b = np.zeros(C) if bias is None else np.asarray(bias, np.float64)
    per = lambda t: np.repeat(t, C // groups, axis=1)[:, None, :]  # noqa: E731
    xhat = (x - per(mean)) * per(rstd)
    dz = grad_y * activation(xhat * w + b, act)[1]
    dx = (dz * w).reshape(n, L, groups, -1)
    h = xhat.reshape(dx.shape)
    m1 = dx.mean(axis=(1, 3), keepdims=True)
    m2 = (dx * h).mean(axis=(1, 3), keepdims=True)
    gx = per(rstd) * (dx - m1 - h * m2).reshape(x.shape)
    return gx, (dz * xhat).sum((0, 1)), dz.sum((0, 1))


# ---- embeddings

def embedding(table, tokens, scale=1.0):
    """Rows of the table times scale; a token outside the table has a row of zeros."""
    table, tokens = np.asarray(table, np.float64), np.asarray(tokens)
    out = np.zeros(tokens.shape + table.shape[1:])
    ok = (tokens >= 0) & (tokens < table.shape[0])
    out[ok] = table[tokens[ok]] * scale
    return out


def embedding_backward(tokens, grad, vocab, scale=1.0):
    tokens, grad = np.asarray(tokens).reshape(-1), np.asarray(grad, np.float64)
    grad = grad.reshape(tokens.size, -1)
    out = np.zeros((vocab, grad.shape[1]))
    ok = (tokens >= 0) & (tokens < vocab)
    np.add.at(out, tokens[ok], grad[ok] * scale)
    return out

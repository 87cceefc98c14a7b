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


# ---- the gated delta rule, token after token

def gated_delta(q, k, v, log_decay, beta, state=None, offsets=None, scale=1.0):
    """q, k: [tokens, Q, dk], v: [tokens, H, dv], log_decay, beta: [tokens, H], state: [sequences, H, dk, dv]; returns (o, final states,
    the largest norm of each head's states)."""
    q, k, v, log_decay, beta = (np.asarray(x, dtype=np.float64) for x in (q, k, v, log_decay, beta))
    n, H, dv = v.shape
    share = np.arange(H) // (H // q.shape[1])
    spans = _spans(n, offsets)
    o, last, most = np.zeros((n, H, dv)), np.zeros((len(spans), H, q.shape[2], dv)), np.zeros(H)
    for s, (a, b) in enumerate(spans):
        S = np.zeros(last.shape[1:]) if state is None else np.array(state[s], dtype=np.float64)
        for t in range(a, b):
            most = np.maximum(most, np.sqrt((S * S).sum((1, 2))))
            S = _delta_step(S, k[t, share], v[t], log_decay[t], beta[t])[0]
            o[t] = scale * np.einsum("hk,hkv->hv", q[t, share], S)
        most = np.maximum(most, np.sqrt((S * S).sum((1, 2))))
        last[s] = S
    return o, last, most


def _delta_step(S, k, v, log_decay, beta):
    S = np.exp(log_decay)[:, None, None] * S
    e = v - np.einsum("hk,hkv->hv", k, S)
    return S + k[:, :, None] * (beta[:, None] * e)[:, None, :], e


def gated_delta_backward(q, k, v, log_decay, beta, grad_o, state=None, grad_state=None, offsets=None, scale=1.0):
    """Adjoints of the recurrence, walked backwards: returns (grad_q, grad_k, grad_v, grad_log_decay, grad_beta, grad_state or None, the
    largest norm of each head's adjoints)."""
    q, k, v, log_decay, beta, grad_o = (np.asarray(x, dtype=np.float64) for x in (q, k, v, log_decay, beta, grad_o))
    n, H, dv = v.shape
    share = np.arange(H) // (H // q.shape[1])
    spans = _spans(n, offsets)
    gq, gk, gv, ga, gb = (np.zeros_like(x) for x in (q, k, v, log_decay, beta))
    gs, most = np.zeros((len(spans), H, q.shape[2], dv)), np.zeros(H)
    for s, (a, b) in enumerate(spans):
        S = np.zeros(gs.shape[1:]) if state is None else np.array(state[s], dtype=np.float64)
        before, errors = [], []
        for t in range(a, b):
            before.append(S)
            S, e = _delta_step(S, k[t, share], v[t], log_decay[t], beta[t])
            errors.append(e)
        before.append(S)
        D = np.zeros(gs.shape[1:]) if grad_state is None else np.array(grad_state[s], dtype=np.float64)
        for t in range(b - 1, a - 1, -1):
            old, new, e, decay = before[t - a], before[t - a + 1], errors[t - a], np.exp(log_decay[t])[:, None]
            np.add.at(gq[t], share, scale * np.einsum("hkv,hv->hk", new, grad_o[t]))
            D = D + scale * q[t, share][:, :, None] * grad_o[t][:, None, :]
            most = np.maximum(most, np.sqrt((D * D).sum((1, 2))))
            w = np.einsum("hk,hkv->hv", k[t, share], D)
            gb[t] = (w * e).sum(-1)
            gv[t] = beta[t][:, None] * w
            np.add.at(gk[t], share, np.einsum("hkv,hv->hk", D, beta[t][:, None] * e) - decay * np.einsum("hkv,hv->hk", old, gv[t]))
            D = decay[:, :, None] * (D - k[t, share][:, :, None] * gv[t][:, None, :])
            ga[t] = (D * old).sum((1, 2))
        gs[s] = D
    return gq, gk, gv, ga, gb, gs if state is not None else None, most


# ---- rotary positions

def rotary(x, positions, frequencies, interleaved=False, scale=1.0, back=False):
    """x: [tokens, heads, dim]: pairs as complex numbers, times scale e^(+-i position frequency)."""
    x = np.array(x, dtype=np.float64)
    p = len(frequencies)
    turn = scale * np.exp((-1j if back else 1j) * np.asarray(positions, np.float64)[:, None] * np.asarray(frequencies, np.float64))[:, None, :]
    one, two = (slice(0, 2 * p, 2), slice(1, 2 * p, 2)) if interleaved else (slice(0, p), slice(p, 2 * p))
    z = (x[..., one] + 1j * x[..., two]) * turn
    x[..., one], x[..., two] = z.real, z.imag
    return x


# ---- norms before and after a block

def _groups_norm(x, groups, eps, kind):
    xg = x.reshape(len(x), groups, -1)
    mean = xg.mean(-1) if kind == "layer" else np.zeros(xg.shape[:2])
    rstd = 1 / np.sqrt(((xg - mean[..., None]) ** 2).mean(-1) + eps)
    return ((xg - mean[..., None]) * rstd[..., None]).reshape(x.shape), mean, rstd


def _or(x, otherwise):
    return otherwise if x is None else np.asarray(x, np.float64)


def block_norm(x, groups, weight=None, bias=None, scale=None, gate=None, residual=None, kind="rms", act="silu", eps=1e-5, before=False, rounded=None):
    """x: [tokens, channels]; returns (y, h or None, mean, rstd).  rounded: takes h to the type that it is held in."""
    x = np.asarray(x, np.float64)
    a = 1.0 if gate is None else activation(np.asarray(gate, np.float64), act)[0]
    w, b, s, r = _or(weight, 1.0), _or(bias, 0.0), _or(scale, 1.0), _or(residual, 0.0)
    if before:
        h = r + s * x * a
        if rounded is not None:
            h = rounded(h)
        n, mean, rstd = _groups_norm(h, groups, eps, kind)
        return n * w + b, h, mean, rstd
    n, mean, rstd = _groups_norm(x, groups, eps, kind)
    return r + s * (n * w + b) * a, None, mean, rstd


def block_norm_backward(x, grad_y, groups, weight=None, bias=None, scale=None, gate=None, kind="rms", act="silu", eps=1e-5, h=None, grad_h=None):
    """Returns a dict of the gradients of x, residual, gate, weight, bias, scale; h: what was normalised, before a block."""
    x, gy = np.asarray(x, np.float64), np.asarray(grad_y, np.float64)
    a, slope = (1.0, 0.0) if gate is None else activation(np.asarray(gate, np.float64), act)
    w, b, s = _or(weight, 1.0), _or(bias, 0.0), _or(scale, 1.0)
    before = h is not None
    xhat, _, rstd = _groups_norm(np.asarray(h if before else x, np.float64), groups, eps, kind)
    n = xhat * w + b
    dn = gy if before else gy * s * a
    d = (dn * w).reshape(len(x), groups, -1)
    t = xhat.reshape(d.shape)
    m1 = d.mean(-1, keepdims=True) if kind == "layer" else 0.0
    dx = (rstd[..., None] * (d - m1 - t * (d * t).mean(-1, keepdims=True))).reshape(x.shape)
    if before:
        total = dx + _or(grad_h, 0.0)
        return dict(residual=total, x=total * s * a, gate=total * s * x * slope, weight=(dn * xhat).sum(0), bias=dn.sum(0), scale=(total * x * a).sum(0))
    return dict(residual=gy, x=dx, gate=gy * s * n * slope, weight=(dn * xhat).sum(0), bias=dn.sum(0), scale=(gy * n * a).sum(0))

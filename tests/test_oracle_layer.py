"""The 64-bit implementations that the layer operators are tested against: against definitions written another way, closed forms
and finite differences.  No GPU."""
import numpy as np
import pytest

from oracle import layer_oracle as lo


def _draw(rng, *shapes):
    return [rng.standard_normal(s) for s in shapes]


def test_attention_is_the_sum_over_pairs():
    rng = np.random.default_rng(1)
    n, H, G, dk, dv = 23, 4, 2, 3, 5
    q, k, v = _draw(rng, (n, H, dk), (n, G, dk), (n, G, dv))
    s0, = _draw(rng, (2, H, dk, dv))
    ld = np.array([-0.3, 0.0, -2.0, -np.inf])
    offsets = [0, 9, 23]
    o, last = lo.attention(q, k, v, ld, s0, offsets, 0.7)
    for s, (a, b) in enumerate(zip(offsets, offsets[1:])):
        for h in range(H):
            power = lambda t: 1.0 if t == 0 else np.exp(ld[h] * t)  # noqa: E731
            for i in range(a, b):
                want = sum(power(i - j) * (q[i, h] @ k[j, h // 2]) * v[j, h // 2] for j in range(a, i + 1)) + power(i - a + 1) * q[i, h] @ s0[s, h]
                assert np.allclose(o[i, h], 0.7 * want, rtol=1e-12, atol=1e-12)
            want = sum(power(b - 1 - j) * np.outer(k[j, h // 2], v[j, h // 2]) for j in range(a, b)) + power(b - a) * s0[s, h]
            assert np.allclose(last[s, h], want, rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("H,G", [(2, 2), (4, 2)])
def test_attention_gradients_are_differences(H, G):
    rng = np.random.default_rng(2)
    n, dk, dv = 11, 2, 3
    q, k, v, do = _draw(rng, (n, H, dk), (n, G, dk), (n, G, dv), (n, H, dv))
    s0, ds = _draw(rng, (3, H, dk, dv), (3, H, dk, dv))
    ld = -np.linspace(0.0, 1.0, H)
    offsets = [0, 4, 4, 11]

    def loss(q, k, v, s0):
        o, last = lo.attention(q, k, v, ld, s0, offsets, 1.3)
        return (o * do).sum() + (last * ds).sum()
    grads = lo.attention_backward(q, k, v, ld, do, s0, ds, offsets, 1.3)
    args = [q, k, v, s0]
    for x, g in zip(args, grads):
        for at in [tuple(rng.integers(0, m) for m in x.shape) for _ in range(12)]:
            keep, e = x[at], 1e-5
            x[at] = keep + e
            up = loss(*args)
            x[at] = keep - e
            down = loss(*args)
            x[at] = keep
            assert abs((up - down) / (2 * e) - g[at]) < 1e-7 * (1 + abs(g[at]))


def test_attention_without_decay_on_ones_counts():
    n = 7
    one = np.ones((n, 1, 1))
    o, last = lo.attention(one, one, one, np.zeros(1))
    assert np.array_equal(o[:, 0, 0], np.arange(1, n + 1)) and last[0, 0, 0, 0] == n
    o, _ = lo.attention(one, one, one, np.log([0.5]))
    assert np.allclose(o[:, 0, 0], 2 - 0.5 ** np.arange(n))


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("shape,groups", [((3, 1, 8), 2), ((2, 5, 6), 3)])
def test_group_norm(act, shape, groups):
    rng = np.random.default_rng(3)
    x, gy = _draw(rng, shape, shape)
    w, b = _draw(rng, shape[-1:], shape[-1:])
    y, mean, rstd = lo.group_norm(x, groups, w, b, 1e-3, act)
    cg = shape[-1] // groups
    for n in range(shape[0]):
        for c in range(shape[2]):
            block = x[n, :, c // cg * cg:(c // cg + 1) * cg]
            z = (x[n, :, c] - block.mean()) / np.sqrt(block.var() + 1e-3) * w[c] + b[c]
            assert np.allclose(y[n, :, c], lo.activation(z, act)[0], rtol=1e-12)
            assert np.isclose(mean[n, c // cg], block.mean()) and np.isclose(rstd[n, c // cg], (block.var() + 1e-3) ** -0.5)
    grads = lo.group_norm_backward(x, gy, groups, w, b, 1e-3, act)
    args = [x, w, b]
    loss = lambda: (lo.group_norm(x, groups, w, b, 1e-3, act)[0] * gy).sum()  # noqa: E731
    for t, g in zip(args, grads):
        for at in [tuple(rng.integers(0, m) for m in t.shape) for _ in range(12)]:
            keep, e = t[at], 1e-5
            t[at] = keep + e
            up = loss()
            t[at] = keep - e
            down = loss()
            t[at] = keep
            assert abs((up - down) / (2 * e) - g[at]) < 1e-7 * (1 + abs(g[at]))


def test_activations_at_known_points():
    z = np.array([0.0, 1.0, -1.0, 40.0, -40.0])
    assert np.allclose(lo.activation(z, "silu")[0], [0, 0.7310585786300049, -0.2689414213699951, 40, 0], atol=1e-15)
    assert np.allclose(lo.activation(z, "gelu")[0], [0, 0.8413447460685429, -0.15865525393145707, 40, 0], atol=1e-15)
    assert np.allclose(lo.activation(z, "silu")[1][[0, 3, 4]], [0.5, 1, 0]) and np.allclose(lo.activation(z, "gelu")[1][[0, 3, 4]], [0.5, 1, 0])


def test_embedding_and_its_gradient_are_adjoint():
    rng = np.random.default_rng(4)
    table, grad = _draw(rng, (6, 3), (2, 5, 3))
    tokens = np.array([[0, 5, -1, 2, 2], [6, 2, 0, 100, 1]])
    rows = lo.embedding(table, tokens, 2.0)
    assert np.array_equal(rows[0, 1], 2 * table[5]) and not rows[0, 2].any() and not rows[1, 0].any() and not rows[1, 3].any()
    assert np.isclose((rows * grad).sum(), (lo.embedding_backward(tokens, grad, 6, 2.0) * table).sum())

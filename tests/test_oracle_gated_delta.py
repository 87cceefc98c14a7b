"""The 64-bit gated delta rule that the kernels are held to: its states against the product of its matrices, its gradients against differences."""
import numpy as np
import pytest

from oracle import layer_oracle as lo


def _inputs(n=9, H=4, Q=2, dk=5, dv=3, seqs=3, seed=0):
    rng = np.random.default_rng(seed)
    q, k = rng.standard_normal((2, n, Q, dk))
    return dict(q=q, k=k / np.linalg.norm(k, axis=-1, keepdims=True), v=rng.standard_normal((n, H, dv)), log_decay=-rng.exponential(0.3, (n, H)), beta=rng.uniform(0, 1.5, (n, H)),
                state=rng.standard_normal((seqs, H, dk, dv)))


def test_state_is_the_matrices_product():
    x = _inputs(seqs=1)
    _, last, _ = lo.gated_delta(**x)
    for h in range(4):
        S = x["state"][0, h]
        for t in range(9):
            k = x["k"][t, h // 2]
            S = np.exp(x["log_decay"][t, h]) * (np.eye(5) - x["beta"][t, h] * np.outer(k, k)) @ S + x["beta"][t, h] * np.outer(k, x["v"][t, h])
        assert np.abs(S - last[0, h]).max() < 1e-13


def test_without_beta_it_is_decay_alone_and_keys_without_decay_are_replaced():
    x = _inputs(seqs=1)
    x["beta"][:] = 0
    _, last, _ = lo.gated_delta(**x)
    assert np.allclose(last[0], np.exp(x["log_decay"].sum(0))[:, None, None] * x["state"][0], rtol=1e-13)
    x["beta"][:] = 1
    x["log_decay"][:] = 0
    o, last, _ = lo.gated_delta(**{**x, "q": x["k"]})
    assert np.allclose(o, x["v"], atol=1e-13)  # a key just written gives its value back


@pytest.mark.parametrize("offsets", [[0, 9], [0, 4, 4, 9], [1, 5, 6, 8]])
def test_gradients_against_differences(offsets):
    seqs = len(offsets) - 1
    x = _inputs(seqs=seqs, seed=seqs)
    rng = np.random.default_rng(7)
    go, gs = rng.standard_normal((9, 4, 3)), rng.standard_normal(x["state"].shape)

    def loss(**kw):
        o, last, _ = lo.gated_delta(**{**x, **kw}, offsets=offsets, scale=0.7)
        return (o * go).sum() + (last * gs).sum()
    *grads, _ = lo.gated_delta_backward(x["q"], x["k"], x["v"], x["log_decay"], x["beta"], go, x["state"], gs, offsets, 0.7)
    for name, g in zip(("q", "k", "v", "log_decay", "beta", "state"), grads):
        d = rng.standard_normal(x[name].shape)
        h = 1e-5
        diff = (loss(**{name: x[name] + h * d}) - loss(**{name: x[name] - h * d})) / (2 * h)
        # a third derivative of some thousands (thirty factors of order one) times h^2, and 1e-15 / h of a loss of some hundred
        assert abs(diff - (g * d).sum()) < 1e-6, name

"""The 64-bit rotary positions and block norms that the kernels are held to: gradients against differences, and the frequencies' rules."""
import math

import numpy as np
import pytest

from oracle import layer_oracle as lo


@pytest.mark.parametrize("before", [False, True])
@pytest.mark.parametrize("kind,act", [("rms", "silu"), ("layer", "gelu"), ("layer", "none")])
@pytest.mark.parametrize("gated", [False, True])
def test_block_norm_gradients_against_differences(before, kind, act, gated):
    rng = np.random.default_rng(3)
    n, C, G = 4, 12, 3
    x = dict(x=rng.standard_normal((n, C)), weight=rng.standard_normal(C), bias=rng.standard_normal(C), scale=rng.standard_normal(C), residual=rng.standard_normal((n, C)),
             gate=rng.standard_normal((n, C)) if gated else None)
    gy, gh = rng.standard_normal((2, n, C))

    def loss(**kw):
        v = {**x, **kw}
        y, h, _, _ = lo.block_norm(v.pop("x"), G, **v, kind=kind, act=act, before=before)
        return (y * gy).sum() + ((h * gh).sum() if before else 0.0)
    h = lo.block_norm(x["x"], G, x["weight"], x["bias"], x["scale"], x["gate"], x["residual"], kind, act, before=before)[1]
    grads = lo.block_norm_backward(x["x"], gy, G, x["weight"], x["bias"], x["scale"], x["gate"], kind, act, h=h, grad_h=gh if before else None)
    for name, v in x.items():
        if v is None:
            continue
        d, e = rng.standard_normal(v.shape), 1e-6
        diff = (loss(**{name: v + e * d}) - loss(**{name: v - e * d})) / (2 * e)
        # third derivatives of some hundreds times e^2, and 1e-14 / e of the sums' roundings
        assert abs(diff - (grads[name] * d).sum()) < 1e-6 * (1 + abs(diff)), name


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_keeps_products_of_distances(interleaved):
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 1, 10))
    f = [1.0, 0.3, 0.01]
    dot = lambda a, b: (lo.rotary(q, [a], f, interleaved) * lo.rotary(k, [b], f, interleaved)).sum()  # noqa: E731
    assert abs(dot(5, 3) - dot(105, 103)) < 1e-12 and abs(dot(5, 3) - dot(5, 4)) > 1e-3
    back = lo.rotary(lo.rotary(q, [7], f, interleaved, 2.0), [7], f, interleaved, 0.5, back=True)
    assert np.abs(back - q).max() < 1e-14 and np.array_equal(lo.rotary(q, [7], f, interleaved)[..., 6:], q[..., 6:])


def test_frequencies():
    from paper_2510_03426_amd import rotary_frequencies
    f, s = rotary_frequencies(4, base=16.0)
    assert f.tolist() == [1.0, 0.5, 0.25, 0.125] and s == 1.0
    f2, s = rotary_frequencies(4, base=16.0, factor=2.0, method="linear")
    assert f2.tolist() == [0.5, 0.25, 0.125, 0.0625] and s == 1.0
    f3, _ = rotary_frequencies(4, base=16.0, factor=8.0, method="base")
    assert f3[0] == 1.0 and abs(float(f3[3]) - 0.125 / 8) < 1e-8
    f4, s = rotary_frequencies(32, factor=4.0, method="parts", trained=4096)
    plain, _ = rotary_frequencies(32)
    turns = 4096 * plain.double() / (2 * math.pi)
    assert bool((f4[turns >= 32] == plain[turns >= 32]).all()) and bool(((f4 * 4 - plain).abs() < 1e-6 * plain)[turns <= 1].all()) and abs(s - (0.1 * math.log(4) + 1)) < 1e-15
    assert bool(((f4 <= plain) & (f4 >= plain / 4 * (1 - 1e-6))).all())
    for kw in (dict(pairs=0), dict(pairs=4, base=1.0), dict(pairs=4, factor=0.5), dict(pairs=4, method="other"), dict(pairs=4, method="parts"), dict(pairs=4, method="parts", trained=9, low=2, high=2)):
        with pytest.raises(ValueError):
            rotary_frequencies(**kw)

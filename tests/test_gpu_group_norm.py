"""Group norm with an activation, channels last, against its formulas in 64 bits.

Tolerances, u = 2^-24, n the elements of a group, X its largest |x|.  Statistics: sums of floats in some order, at most
(16 + n / 64) u relative to the sum of magnitudes on the paths taken (a lane adds up to 32 elements, six shuffles; the long
kernels sum in doubles): mean within 40 u X, and with it every x - mean; rstd within 40 u + twice the error of x - mean times
rstd.  So xhat is off by at most e = 100 u (X rstd + |xhat| + 1), z by e |weight| + 4 u, and y by 1.13 times that (the largest
slope of the activations) and 8 u |y| of the functions' own.  Gradients: dz is off by |grad_y| times the slope's change (at most
0.8 times z's error) and 16 u; what is summed over a group enters grad_x once more.  Stored results are rounded to their type."""
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


def _within(got, want, tol, dtype, what):
    got = got.double().cpu().numpy()
    tol = tol + ROUND[dtype] * np.abs(want) + (2.0 ** -25 if dtype == "f16" else 1e-37)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.max(np.abs(got - want) / tol):.3g} of the tolerance, first at {np.argwhere(bad)[0]}"


def _check(g, dtype, items, length, channels, groups, act, wtype="f32", seed=0, offset=0.5, spread=1.0, plain=False, eps=1e-5):
    import torch
    from oracle import layer_oracle as lo
    types = _types()
    rng = np.random.default_rng(seed)
    put = lambda a, t: torch.from_numpy(np.asarray(a, dtype=np.float32)).to(types[t])  # noqa: E731
    x = put(rng.standard_normal((items, length, channels)) * spread + offset, dtype)
    gy = put(rng.standard_normal((items, length, channels)), dtype)
    w, b = (None, None) if plain else (put(1 + 0.3 * rng.standard_normal(channels), wtype), put(0.3 * rng.standard_normal(channels), wtype))
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    f64 = lambda t: None if t is None else t.double().numpy()  # noqa: E731
    y, mean, rstd = g.group_norm(dev(x), groups, dev(w), dev(b), eps=eps, activation=act, want_stats=True)
    want, wm, wr = lo.group_norm(f64(x), groups, f64(w), f64(b), eps, act)
    n = length * channels // groups
    top = np.abs(f64(x)).reshape(items, length, groups, -1).max(axis=(1, 3))
    _within(mean, wm, 40 * U * top, "f32", "mean")
    _within(rstd, wr, wr * (40 * U + 2 * 40 * U * top * wr), "f32", "rstd")
    per = lambda t: np.repeat(t, channels // groups, axis=1)[:, None, :]  # noqa: E731
    xhat = (f64(x) - per(wm)) * per(wr)
    e = 100 * U * (per(top * wr) + np.abs(xhat) + 1)
    aw = 1.0 if plain else np.abs(f64(w))
    ez = e * aw + 4 * U
    _within(y, want, 1.13 * ez + 8 * U * np.abs(want), dtype, "y")
    # the backward pass gets the library's own statistics
    gx, gw, gb = g.group_norm_backward(dev(x), dev(gy), mean, rstd, groups, dev(w), dev(b), activation=act)
    wx, ww, wb = lo.group_norm_backward(f64(x), f64(gy), groups, f64(w), f64(b), eps, act)
    edz = np.abs(f64(gy)) * (0.8 * ez + 16 * U)
    adz = 1.13 * np.abs(f64(gy))
    grp = lambda t: np.repeat(np.broadcast_to(t, xhat.shape).reshape(items, length, groups, -1).mean(axis=(1, 3)), channels // groups, axis=1)[:, None, :]  # noqa: E731
    a1, a2 = grp(adz * aw), grp(adz * aw * np.abs(xhat))
    ex = per(wr) * (edz * aw + grp(edz * aw) + np.abs(xhat) * grp(edz * aw * np.abs(xhat) + adz * aw * e) + e * a2 + (40 + n / 64) * U * (a1 + np.abs(xhat) * a2)
                    + 60 * U * (adz * aw + a1 + np.abs(xhat) * a2) * (1 + per(top * wr)))
    _within(gx, wx, ex, dtype, "grad_x")
    sums = 128 + 64  # positions a thread adds up at most, and the joins
    t = wtype if not plain else "f32"
    _within(gw, ww, (edz * np.abs(xhat) + adz * e + sums * U * adz * np.abs(xhat)).sum((0, 1)), t, "grad_weight")
    _within(gb, wb, (edz + sums * U * adz).sum((0, 1)), t, "grad_bias")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("items,length,channels,groups", [(1, 1, 2, 1), (3, 1, 64, 4), (17, 1, 53, 1), (5, 1, 1744, 16), (2, 1, 2048, 16), (9, 3, 24, 8), (7, 5, 105, 7), (4, 40, 90, 10), (300, 1, 128, 32)])
def test_short_groups(g, dtype, act, items, length, channels, groups):
    _check(g, dtype, items, length, channels, groups, act, seed=channels)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("items,length,channels,groups", [(2, 100, 4100, 4), (3, 700, 36, 6), (2, 500, 320, 32), (1, 1, 5000, 1), (1, 70, 2600, 1), (3, 257, 9, 3), (2, 33, 1024, 2), (1, 4000, 8, 8), (40, 65, 96, 2)])
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_long_groups(g, dtype, items, length, channels, groups, act):
    _check(g, dtype, items, length, channels, groups, act, seed=length)


@pytest.mark.parametrize("wtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("items,length", [(40, 1), (2, 400)])
def test_parameter_types(g, wtype, items, length):
    _check(g, "bf16", items, length, 96, 12, "silu", wtype=wtype)
    _check(g, "f32", items, length, 96, 12, "silu", plain=True)


@pytest.mark.parametrize("length", [1, 600])
def test_means_far_from_zero(g, length):
    """A mean of a thousand spreads: no cancellation between the mean square and the squared mean."""
    _check(g, "f32", 3, length, 64, 2, "none", offset=1000.0, spread=1.0)


@pytest.mark.parametrize("length", [1, 700])
def test_constant_groups(g, length):
    """A variance of zero: rstd = eps^-1/2 and y = bias."""
    import torch
    x = torch.full((3, length, 32), 0.75, device="cuda")
    w, b = torch.full((32,), 2.0, device="cuda"), torch.linspace(-1, 1, 32, device="cuda")
    y, mean, rstd = g.group_norm(x, 4, w, b, eps=1e-4, want_stats=True)
    assert torch.equal(mean, torch.full((3, 4), 0.75, device="cuda")) and torch.allclose(rstd, torch.full((3, 4), 100.0, device="cuda"), rtol=1e-6)
    assert torch.equal(y, b.expand_as(y))


@pytest.mark.parametrize("items,length,channels,groups", [(5000, 1, 256, 16), (3, 900, 80, 8)])
def test_runs_repeat_bit_by_bit(g, items, length, channels, groups):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, gy = (torch.randn(items, length, channels, device="cuda", generator=gen).bfloat16() for _ in range(2))
    w, b = torch.rand(channels, device="cuda", generator=gen), torch.rand(channels, device="cuda", generator=gen)

    def run():
        y, mean, rstd = g.group_norm(x, groups, w, b, activation="silu", want_stats=True)
        return (y, mean, rstd) + g.group_norm_backward(x, gy, mean, rstd, groups, w, b, activation="silu")
    for s, t in zip(run(), run()):
        assert torch.equal(s, t)


def test_a_nan_stays_in_its_group_and_addresses_may_be_odd(g):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(2)
    for length in (1, 300):
        flat = torch.randn(4 * length * 64 + 1, device="cuda", generator=gen)
        x = flat[1:].view(4, length, 64)  # 4-byte aligned only
        y, mean, rstd = g.group_norm(x, 4, activation="silu", want_stats=True)
        z, m, r = g.group_norm(x.clone(), 4, activation="silu", want_stats=True)
        assert torch.allclose(y, z, rtol=1e-5, atol=1e-6) and torch.allclose(mean, m, atol=1e-6) and torch.allclose(rstd, r, rtol=1e-5)
        x[2, 0, 17] = float("nan")
        bad = g.group_norm(x, 4, activation="silu")
        keep = torch.ones_like(y, dtype=torch.bool)
        keep[2, :, 16:32] = False
        assert torch.equal(bad[keep], y[keep]) and bad[~keep].isnan().all()


def test_empty(g):
    import torch
    x = torch.empty(0, 3, 8, device="cuda")
    y, mean, rstd = g.group_norm(x, 2, want_stats=True)
    gx, gw, gb = g.group_norm_backward(x, x, mean, rstd, 2)
    assert y.numel() == 0 and gx.numel() == 0 and torch.equal(gw, torch.zeros(8, device="cuda")) and torch.equal(gb, gw)

"""Norms before and after a block, through the library, against the formulas in 64 bits.

Tolerances, u = 2^-24.  A group's sums of up to N squares and products pass at most 16 + 10 + 16 additions (a lane's entries, lanes, waves), so a factor rstd is off by
some 24 u, the means by 48 u of the mean magnitude; with the handful of products around them every term of an output is off by at most 64 u of
its own size, SiLU by |z| u more (|z| < 6 here) and GELU by 1.5e-7 + 8 u of |z|: 128 u of the sum of the terms' magnitudes.  Parameters' gradients are sums over T
tokens, added in chains of at most T / 8 + 64.  The stored result is rounded once more, eps / 2 of it; a stream that is held in 16 bits is compared before the
norm within that, and the norm is held to what was stored."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": U, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def _types():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def g():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2510_03426_amd import Goom
    g = Goom(0)
    yield g
    g.close()


def _f64(x):
    return None if x is None else x.double().cpu().numpy()


def _near(got, want, size, dtype, what, units=128.0):
    tol = HALF[dtype] * np.abs(want) + units * U * size + (2.0 ** -25 if dtype == "f16" else 0) + 1e-37
    bad = ~(np.abs(_f64(got) - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(_f64(got) - want) / tol):.3g} of the tolerance, first at {np.argwhere(bad)[0]}"


def _check(g, dtype, tokens, channels, groups, kind="rms", act="silu", gate=True, residual=True, scale=True, ptype="f32", params=True, lead=None, mean=0.5):
    import torch
    from oracle import layer_oracle as lo
    rng = np.random.default_rng(tokens + channels)
    t, pt = _types()[dtype], _types()[ptype]
    draw = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32))  # noqa: E731
    x = (draw(tokens, channels) + mean).to(t)
    z = draw(tokens, channels).clamp(-6, 6).to(t) if gate else None
    r = draw(tokens, channels).to(t) if residual else None
    w = (1 + 0.2 * draw(channels)).to(pt) if params else None
    b = (0.2 * draw(channels)).to(pt) if params else None
    s = (0.6 + 0.2 * draw(channels)).to(pt) if scale else None
    gy, gh = draw(tokens, channels).to(t), draw(tokens, channels).to(t)
    X, Z, R, W, B, S, GY, GH = (_f64(v) for v in (x, z, r, w, b, s, gy, gh))
    shape = (lambda v: None if v is None else v.cuda().reshape(lead + (channels,))) if lead else (lambda v: None if v is None else v.cuda())
    dev = lambda v: None if v is None else v.cuda()  # noqa: E731
    flat = lambda v: v.reshape(tokens, -1)  # noqa: E731
    kw = dict(groups=groups, weight=dev(w), bias=dev(b), scale=dev(s), gate=shape(z), kind=kind, activation=act)
    ab = lambda v, o: o if v is None else np.abs(v)  # noqa: E731
    per = lambda v: np.repeat(v, channels // groups, axis=1)  # noqa: E731
    dx, dgy, dgh = shape(x), shape(gy), shape(gh)
    A = 1.0 if z is None else np.abs(Z)  # at least the activation
    # after
    y, m, q = g.norm_after(dx, residual=shape(r), want_stats=True, **kw)
    want, _, wm, wq = lo.block_norm(X, groups, W, B, S, Z, R, kind, act)
    big = (np.abs(X) + per(np.abs(X).reshape(tokens, groups, -1).mean(-1))) * per(wq)  # an xhat's terms
    n_size = big * ab(W, 1.0) + ab(B, 0.0)
    _near(flat(y), want, ab(S, 1.0) * n_size * A + ab(R, 0.0), dtype, "after: y")
    _near(flat(q), wq, wq, "f32", "after: rstd")
    assert (m is None) == (kind == "rms")
    if m is not None:
        _near(flat(m), wm, np.abs(X).reshape(tokens, groups, -1).mean(-1), "f32", "after: mean")
    grads = g.norm_after_backward(dx, dgy, m, q, **kw)
    want = lo.block_norm_backward(X, GY, groups, W, B, S, Z, kind, act)
    slope = 0.0 if z is None else 1.2 + 0 * A
    d = np.abs(GY) * ab(S, 1.0) * (A if z is not None else 1.0)
    over = lambda v: per(v.reshape(tokens, groups, -1).mean(-1))  # noqa: E731
    gx_size = per(wq) * (d * ab(W, 1.0) + over(d * ab(W, 1.0)) + big * over(d * ab(W, 1.0) * big))
    sizes = dict(x=gx_size, gate=np.abs(GY) * ab(S, 1.0) * n_size * slope, weight=(d * big).sum(0), bias=d.sum(0), scale=(np.abs(GY) * n_size * A).sum(0))
    _grads(("x", "gate", "weight", "bias", "scale"), grads, want, sizes, dtype, ptype, "after", tokens, channels)
    # before
    y, h, m, q = g.norm_before(dx, residual=shape(r), want_stats=True, **kw)
    plain = lo.block_norm(X, groups, W, B, S, Z, R, kind, act, before=True)[1]
    _near(flat(h), plain, ab(S, 1.0) * np.abs(X) * A + ab(R, 0.0), dtype, "before: h")
    held = _f64(flat(h))
    want, _, wm, wq = lo.block_norm(held, groups, W, B, None, None, None, kind, act, before=True)
    big = (np.abs(held) + over(np.abs(held))) * per(wq)
    _near(flat(y), want, big * ab(W, 1.0) + ab(B, 0.0), dtype, "before: y")
    grads = g.norm_before_backward(dx, h, dgy, m, q, grad_h=dgh, **kw)
    want = lo.block_norm_backward(X, GY, groups, W, B, S, Z, kind, act, h=held, grad_h=GH)
    d = np.abs(GY) * ab(W, 1.0)
    total = per(wq) * (d + over(d) + big * over(d * big)) + np.abs(GH)
    sizes = dict(residual=total, x=total * ab(S, 1.0) * A, gate=total * ab(S, 1.0) * np.abs(X) * slope, weight=(np.abs(GY) * big).sum(0), bias=np.abs(GY).sum(0),
                 scale=(total * np.abs(X) * A).sum(0))
    _grads(("residual", "x", "gate", "weight", "bias", "scale"), grads, want, sizes, dtype, ptype, "before", tokens, channels)
    if z is None and s is None:
        assert grads[0] is grads[1]
    again = g.norm_before_backward(dx, h, dgy, m, q, grad_h=dgh, **kw)
    assert all(a is None or torch.equal(a, b) for a, b in zip(again, grads))


def _grads(names, grads, want, sizes, dtype, ptype, what, tokens, channels):
    for name, got in zip(names, grads):
        if got is None:
            continue
        param = name in ("weight", "bias", "scale")
        _near(got.reshape(-1) if param else got.reshape(tokens, channels), want[name], sizes[name], ptype if param else dtype, f"{what}: gradient of {name}",
              192.0 + tokens / 8 if param else 192.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32", "f16"])
@pytest.mark.parametrize("tokens,channels,groups", [(1, 1, 1), (3, 7, 1), (1, 2048, 16), (130, 96, 8), (70, 1712, 16), (9, 642, 2), (300, 64, 32), (5, 4096, 1), (6, 5003, 1), (2, 12288 + 7, 1), (2050, 40, 5), (40, 1100, 4)])
def test_sizes(g, dtype, tokens, channels, groups):
    _check(g, dtype, tokens, channels, groups)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("gate,residual,scale,params", [(True, False, False, True), (False, True, True, False), (False, False, False, True), (True, True, True, True)])
def test_what_there_is(g, kind, act, gate, residual, scale, params):
    _check(g, "f32", 20, 192, 3, kind, act, gate, residual, scale, "f32", params)
    _check(g, "bf16", 20, 192, 1, kind, act, gate, residual, scale, "bf16", params, lead=(4, 5))


def test_means_far_from_zero(g):
    _check(g, "f32", 10, 256, 2, "layer", mean=300.0)


def test_streams_graphs_and_refusals(g):
    import torch
    from paper_2510_03426_amd import Goom, GoomError
    x, z, r = torch.randn(3, 50, 256, device="cuda").bfloat16()
    w = torch.rand(256, device="cuda")
    kw = dict(groups=4, weight=w, gate=z)
    run = lambda c: c.norm_after(x, residual=r, want_stats=True, **kw)[::2] + c.norm_before(x, residual=r, **kw)  # noqa: E731
    back = lambda c, q: c.norm_after_backward(x, r, None, q, **kw)[:3]  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = Goom(0, side)
        back(c, run(c)[1])
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = run(c)
            out += back(c, out[1])
    torch.cuda.synchronize()
    for i in range(3):
        x.mul_(1 + 0.25 * i)
        graph.replay()
        want = run(g)
        want += back(g, want[1])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i
    c.close()
    none = torch.zeros(0, 256, device="cuda", dtype=torch.bfloat16)
    assert g.norm_after(none, weight=w).shape == (0, 256)
    gx, _, gw, _, _ = g.norm_after_backward(none, none, None, torch.zeros(0, 1, device="cuda"), weight=w)
    assert gx.shape == (0, 256) and (gw == 0).all()
    for k2 in (dict(kind="other"), dict(activation="relu"), dict(weight=w[:10]), dict(gate=z[:, :10]), dict(gate=z.float()), dict(residual=r[:1])):
        with pytest.raises(ValueError):
            g.norm_after(x, **k2)
    with pytest.raises(TypeError):
        g.norm_after(x, weight=w, bias=w.bfloat16())
    with pytest.raises(GoomError):
        g.norm_after(x, groups=7)
    with pytest.raises(ValueError):
        g.norm_before_backward(x, x, x, None, None, weight=w)

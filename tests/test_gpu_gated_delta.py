"""The gated delta rule, through the library, against the token-by-token recurrence in 64 bits.

Tolerances.  Keys are of length one (rounded) and beta between 0 and 1.5, so that the recurrence's matrices a (I - beta k k^T) have norms
of at most one and carry an error on without growth.  Each token adds roundings of sums of dk products and of the triangular solve of its
chunk (2 C terms, C = 64): with the largest norm of a head's states A, of its keys, queries and betas at most B = 1.5, and u = 2^-24, every token moves the
state by at most r u A sqrt(dk + 2 C + 8), r a random number of order one.  Roundings being independent in good measure, n tokens move it
by r u A sqrt(n (dk + 2 C + 8)); twelve of that is what is allowed.  Outputs are the state times q: times |scale| |q|.  Gradients are products of two such
quantities, the states (A) and their adjoints (D), with rows whose norms stand with them below: twice the roundings.
The stored result is rounded once more: 2^-9 (bfloat16), 2^-12 (half, and 2^-25 below its normal range) of itself and of its neighbour: eps / 2."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": U, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def _torch():
    import torch
    return torch, {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def g():
    torch, _ = _torch()
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2510_03426_amd import Goom
    g = Goom(0)
    yield g
    g.close()


def _inputs(dtype, n, H, Q, dk, dv, seqs, seed):
    torch, types = _torch()
    rng = np.random.default_rng(seed)
    q, k = rng.standard_normal((2, n, Q, dk))
    unit = lambda x: x / np.linalg.norm(x, axis=-1, keepdims=True)  # noqa: E731
    to = lambda x: torch.from_numpy(np.asarray(x, np.float32)).to(types[dtype])  # noqa: E731
    x = dict(q=to(unit(q)), k=to(unit(k)), v=to(rng.standard_normal((n, H, dv))))
    rate = np.exp2(-np.linspace(1, 9, H))
    x["log_decay"] = torch.from_numpy((-rate * np.log1p(np.exp(rng.standard_normal((n, H))))).astype(np.float32))
    x["beta"] = torch.from_numpy((1 / (1 + np.exp(-rng.standard_normal((n, H))))).astype(np.float32))
    x["state"], x["grad_state"] = (torch.from_numpy(rng.standard_normal((seqs, H, dk, dv)).astype(np.float32)) for _ in range(2))
    x["grad_o"] = to(rng.standard_normal((n, H, dv)))
    return x


def _f64(x):
    return None if x is None else x.double().cpu().numpy()


def _near(got, want, bound, dtype, what, mask=None):
    got = _f64(got)
    tol = HALF[dtype] * np.abs(want) + bound + (2.0 ** -25 if dtype == "f16" else 0) + 1e-37
    bad = ~(np.abs(got - want) <= tol)
    if mask is not None:
        bad &= mask
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(got - want) / tol):.3g} of the tolerance, first at {np.argwhere(bad)[0]}"


def _check(g, dtype, n, H, Q, dk, dv, offsets=None, batch=None, with_state=True, scale=1.0, seed=0, change=None, backward=True):
    torch, _ = _torch()
    from oracle import layer_oracle as lo
    seqs = batch if batch else len(offsets) - 1 if offsets else 1
    x = _inputs(dtype, n, H, Q, dk, dv, seqs, seed)
    if change:
        change(x)
    if not with_state:
        x["state"] = x["grad_state"] = None
    spans = offsets or [i * (n // seqs) for i in range(seqs + 1)]
    r = {name: _f64(t) for name, t in x.items()}
    ins = [r[name] for name in ("q", "k", "v", "log_decay", "beta")]
    lead = (lambda t: t.reshape((batch, n // batch) + t.shape[1:])) if batch else (lambda t: t)
    dev = {name: None if t is None else t.cuda() if "state" in name else lead(t.cuda()) for name, t in x.items()}
    off = torch.tensor(offsets, dtype=torch.int64).cuda() if offsets else None
    args = [dev[name] for name in ("q", "k", "v", "log_decay", "beta")]
    here = np.zeros(n, dtype=bool)
    for a, b in zip(spans[:-1], spans[1:]):
        here[a:b] = True
    longest = max(b - a for a, b in zip(spans[:-1], spans[1:]))
    err = 12 * U * math.sqrt(max(1, longest) * (dk + 136.0))

    o, last = g.gated_delta(*args, state=dev["state"], offsets=off, scale=scale, want_state=True)
    assert o.dtype == x["q"].dtype and o.shape == dev["v"].shape
    want, wl, A = lo.gated_delta(*ins, r["state"], spans, scale)
    A = np.maximum(A, np.abs(r["v"]).max(initial=0) * math.sqrt(dv))
    per = lambda t: t.reshape((n,) + t.shape[-2:])  # noqa: E731
    qn = np.linalg.norm(r["q"], axis=-1).max(initial=0)
    _near(per(o), want, abs(scale) * qn * err * A[:, None], dtype, "o", here[:, None, None])
    _near(last, wl, err * A[:, None, None], "f32", "final state")
    if not backward:
        return dev, args, off, (o, last)
    grads = g.gated_delta_backward(*args, dev["grad_o"], state=dev["state"], grad_state=dev["grad_state"], offsets=off, scale=scale)
    *wants, D = lo.gated_delta_backward(*ins, r["grad_o"], r["state"], r["grad_state"], spans, scale)
    gn = np.linalg.norm(r["grad_o"], axis=-1).max(initial=0)
    D = np.maximum(D, abs(scale) * qn * gn)
    share = H // Q
    top = lambda z: z.reshape(Q, share).sum(1)[:, None]  # noqa: E731
    bounds = [2 * err * abs(scale) * gn * top(A), 4 * err * 1.5 * top(A * D), 2 * err * 1.5 * D[:, None], 4 * err * A * D, 4 * err * A * D, 2 * err * D[:, None, None]]
    names = ("grad_q", "grad_k", "grad_v", "grad_log_decay", "grad_beta", "grad_state")
    for name, got, w, bound, t in zip(names, grads, wants, bounds, (dtype, dtype, dtype, "f32", "f32", "f32")):
        if w is None:
            assert got is None
            continue
        flat = got if name == "grad_state" else got.reshape((n,) + w.shape[1:])
        mask = None if name == "grad_state" else here.reshape((n,) + (1,) * (w.ndim - 1))
        _near(flat, w, bound, t, name, mask)
    return dev, args, off, (o, last)


@pytest.mark.parametrize("dtype", ["bf16", "f32", "f16"])
@pytest.mark.parametrize("dk,dv", [(32, 32), (64, 64), (128, 128), (1, 1), (7, 19), (50, 72), (100, 33), (33, 128), (128, 20)])
def test_heads(g, dtype, dk, dv):
    _check(g, dtype, 2 * 70, 4, 2, dk, dv, batch=2, scale=dk ** -0.5, seed=dk + dv)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 129])
def test_lengths(g, dtype, n):
    _check(g, dtype, n, 2, 2, 40, 48, seed=n, with_state=n % 2 == 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32", "f16"])
def test_segments(g, dtype):
    """Few heads: sequences are cut into segments, whose maps are chained."""
    _check(g, dtype, 1500, 1, 1, 64, 40, seed=3)
    _check(g, dtype, 1300, 2, 1, 100, 100, offsets=[0, 700, 700, 705, 1300], seed=4)


@pytest.mark.parametrize("dtype,offsets", [("bf16", [0, 1, 1, 64, 130, 200]), ("f32", [0, 0, 33, 200]), ("f16", [0, 100, 200, 200]), ("bf16", [0, 200])])
def test_packed(g, dtype, offsets):
    _check(g, dtype, 200, 6, 2, 48, 64, offsets=offsets, seed=len(offsets), scale=0.3)


def _forget(x):
    torch, _ = _torch()
    x["log_decay"][::7] = -math.inf
    x["log_decay"][3::11] = -40.0
    x["beta"][5::9] = 0.0
    x["beta"][6::9] = 1.0
    x["log_decay"][10:14] = 0.0
    x["log_decay"][50:] = -3e38


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decays_and_betas_of_zero(g, dtype):
    dev, args, off, _ = _check(g, dtype, 150, 3, 3, 32, 40, batch=1, seed=11, change=_forget)
    ga = g.gated_delta_backward(*args, dev["grad_o"])[3]
    assert (ga[args[3] < -110] == 0).all()  # (where nothing is left, exactly)


def test_equal_keys(g):
    """Every key the same, written whole: each token replaces the last one's value, and the triangular systems are as full as they get."""
    def same(x):
        x["k"][:] = x["k"][0, 0]
        x["beta"][:] = 1.0
    _check(g, "bf16", 130, 2, 2, 64, 64, seed=5, change=same)
    _check(g, "f32", 130, 2, 2, 20, 64, seed=6, change=same)


def test_growing_states(g):
    """Decays above one, over 80 tokens: e^2."""
    def grow(x):
        x["log_decay"][:] = 0.025
    # (errors grow with the states, by e^2 at most after they are made: within twelve random roundings' allowance of the largest state)
    _check(g, "f32", 80, 2, 2, 32, 32, seed=8, change=grow, backward=False)


def test_tokens_outside_the_sequences_are_left(g):
    torch, _ = _torch()
    x = _inputs("bf16", 100, 2, 1, 32, 32, 2, 1)
    off = torch.tensor([10, 40, 90], dtype=torch.int64).cuda()
    args = [x[name].cuda() for name in ("q", "k", "v", "log_decay", "beta")]
    for t in args:  # what lies outside is not looked at either
        t[:10] = math.nan
        t[90:] = math.nan
    empty = torch.empty

    def marked(*a, **kw):
        return empty(*a, **kw).fill_(7.0) if kw.get("dtype") != torch.uint8 else empty(*a, **kw)
    torch.empty = marked
    try:
        o = g.gated_delta(*args, offsets=off)
        grads = g.gated_delta_backward(*args, x["grad_o"].cuda(), offsets=off)
    finally:
        torch.empty = empty
    assert (o[:10] == 7).all() and (o[90:] == 7).all() and torch.isfinite(o[10:90].float()).all()
    for t in grads[1:5]:
        assert (t[:10] == 7).all() and (t[90:] == 7).all() and torch.isfinite(t[10:90].float()).all()


def test_slices_of_a_projection_and_no_tokens(g):
    torch, _ = _torch()
    gen = torch.Generator(device="cuda").manual_seed(1)
    H, d = 4, 32
    fused = torch.randn(2, 70, 3 * H * d, device="cuda", generator=gen).bfloat16()
    q, k, v = (t.unflatten(-1, (H, d)) for t in fused.split(H * d, dim=-1))
    k = (k.float() / k.float().norm(dim=-1, keepdim=True)).bfloat16()
    a, b = -torch.rand(2, 70, H, device="cuda", generator=gen), torch.rand(2, 70, H, device="cuda", generator=gen)
    one = g.gated_delta(q, k, v, a, b, want_state=True)
    two = g.gated_delta(q.contiguous(), k, v.contiguous(), a, b, want_state=True)
    assert all(torch.equal(s, t) for s, t in zip(one, two))
    state = torch.randn(3, H, d, d, device="cuda", generator=gen)
    none = torch.zeros(0, H, d, device="cuda", dtype=torch.bfloat16)
    off = torch.zeros(4, dtype=torch.int64, device="cuda")
    o, last = g.gated_delta(none, none, none, none[..., 0].float(), none[..., 0].float(), state=state, offsets=off, want_state=True)
    assert o.shape == (0, H, d) and torch.equal(last, state)
    grads = g.gated_delta_backward(none, none, none, none[..., 0].float(), none[..., 0].float(), none, state=state, grad_state=2 * state, offsets=off)
    assert torch.equal(grads[5], 2 * state)


@pytest.mark.parametrize("dtype", ["bf16", "f32", "f16"])
@pytest.mark.parametrize("dk,dv,H,Q,n", [(64, 64, 4, 2, 5), (128, 128, 2, 2, 3), (1, 1, 1, 1, 1), (50, 71, 6, 2, 4), (129 - 30, 33, 2, 1, 9)])
def test_step(g, dtype, dk, dv, H, Q, n):
    """Single tokens: the recurrence's next state, in place and into another array, and the chunked form of a sequence of one."""
    torch, _ = _torch()
    from oracle import layer_oracle as lo
    x = _inputs(dtype, n, H, Q, dk, dv, n, seed=dk + n)
    args = [x[name].cuda() for name in ("q", "k", "v", "log_decay", "beta")]
    spans = list(range(n + 1))
    want, wl, A = lo.gated_delta(*[_f64(x[name]) for name in ("q", "k", "v", "log_decay", "beta", "state")], spans, 0.4)
    # sums of dk products each, and a few more roundings
    err = (dk + 8) * U
    state = x["state"].cuda()
    keep, out = state.clone(), torch.empty_like(state)
    o = g.gated_delta_step(*args, state, scale=0.4, out_state=out)
    A = np.maximum(A, np.abs(_f64(x["v"])).max() * math.sqrt(dv))
    assert torch.equal(state, keep)
    _near(out, wl, err * 2 * A[:, None, None], "f32", "state")
    _near(o, want, err * 4 * A[:, None], dtype, "o")
    o2 = g.gated_delta_step(*args, state, scale=0.4)
    assert torch.equal(o, o2) and torch.equal(state, out)
    long = [t.unsqueeze(1) for t in args]
    o3, last = g.gated_delta(*long, state=keep, scale=0.4, want_state=True)
    _near(last, wl, 12 * U * math.sqrt(dk + 136.0) * A[:, None, None], "f32", "a sequence of one: state")
    _near(o3[:, 0], want, 12 * U * math.sqrt(dk + 136.0) * A[:, None], dtype, "a sequence of one: o")


def test_parts_make_the_whole(g):
    """A sequence in two calls, the second from the first's state, written over it."""
    torch, _ = _torch()
    x = _inputs("f32", 190, 2, 2, 32, 32, 1, 2)
    args = [x[name].cuda().unsqueeze(0) for name in ("q", "k", "v", "log_decay", "beta")]
    whole, last = g.gated_delta(*args, want_state=True)
    first, state = g.gated_delta(*[t[:, :77].contiguous() for t in args], want_state=True)
    second, end = g.gated_delta(*[t[:, 77:].contiguous() for t in args], state=state, want_state=True)
    both = torch.cat([first, second], 1)
    err = 24 * U * math.sqrt(190 * 168.0) * max(1.0, float(last.norm()))
    assert (both - whole).abs().max() < err and (end - last).abs().max() < err


def test_graph_and_stream(g):
    """Captured and replayed on new inputs, with eager calls between, and on another stream: the same bits."""
    torch, _ = _torch()
    from paper_2510_03426_amd import Goom
    x = _inputs("bf16", 300, 4, 4, 64, 64, 2, 3)
    args = [x[name].cuda().reshape((2, 150) + x[name].shape[1:]) for name in ("q", "k", "v", "log_decay", "beta")]
    go = x["grad_o"].cuda().reshape(2, 150, 4, 64)
    state = x["state"].cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        h = Goom(0, side)
        run = lambda c: c.gated_delta(*args, state=state, want_state=True) + c.gated_delta_backward(*args, go, state=state, grad_state=state)  # noqa: E731
        run(h)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = run(h)
    torch.cuda.current_stream().wait_stream(side)
    for i in range(3):
        args[2].mul_(-1.0 if i else 1.0).add_(0.125 * i)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = run(g)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i
    h.close()


def test_refuses(g):
    torch, _ = _torch()
    z = lambda *s, t=torch.bfloat16: torch.zeros(s, device="cuda", dtype=t)  # noqa: E731
    f = torch.float32
    ok = dict(q=z(2, 8, 2, 16), k=z(2, 8, 2, 16), v=z(2, 8, 4, 24), log_decay=z(2, 8, 4, t=f), beta=z(2, 8, 4, t=f))
    g.gated_delta(**ok)
    for kw, error in ((dict(k=z(2, 8, 2, 15)), ValueError), (dict(k=z(2, 8, 2, 16, t=f)), TypeError), (dict(log_decay=z(2, 8, 4)), TypeError), (dict(beta=z(2, 8, 2, t=f)), ValueError),
                      (dict(v=z(2, 7, 4, 24)), ValueError), (dict(state=z(2, 4, 24, 16, t=f)), ValueError), (dict(state=z(2, 4, 16, 24)), ValueError),
                      (dict(offsets=torch.zeros(3, dtype=torch.int64, device="cuda")), ValueError), (dict(q=z(2, 8, 1, 16).expand(2, 8, 2, 16)), ValueError)):
        with pytest.raises(error):
            g.gated_delta(**{**ok, **kw})
    with pytest.raises(ValueError):
        g.gated_delta_step(**ok, state=z(2, 4, 16, 24, t=f))
    with pytest.raises(ValueError):
        g.gated_delta_backward(**ok, grad_o=z(2, 8, 4, 16))
    from paper_2510_03426_amd import GoomError
    with pytest.raises(GoomError):
        g.gated_delta(**{**ok, "v": z(2, 8, 3, 24), "log_decay": z(2, 8, 3, t=f), "beta": z(2, 8, 3, t=f)})

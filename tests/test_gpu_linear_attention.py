"""Linear attention with a decay for each head, through the library, against the token-by-token recurrence in 64 bits.

Tolerances.  Every output is a sum of products; with the sum of its terms' magnitudes (the same recurrence on absolute values) as
M, a float evaluation in any order is off by at most about u (terms of the longest sum + weights' roundings) M, u = 2^-24: a
term passes the d products of its inner product, at most 64 of its chunk and one addition a chunk after that, and its decay is
an exponential whose argument, age times log2 of the decay, is rounded (age |log2 decay| u, times the decay itself: at most
u / e over all ages, and 1 / (chunk |log decay|) of it where carried states are multiplied by the same rounded factor again and
again: 16 u here).  Operands in two bf16 parts are off by 2^-16 of themselves, and there are three such operands: the pairs, the
state, and what entered it (states that are returned take three parts, 2^-24).  The stored
output is rounded once more: 2^-8 (bfloat16), 2^-11 (half) of itself."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
ROUND = {"f32": U, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


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


def _inputs(dtype, n, H, G, dk, dv, seqs, seed, decays=None):
    torch, types = _torch()
    rng = np.random.default_rng(seed)
    draw = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(types[dtype])  # noqa: E731
    q, k, v, do = draw(n, H, dk), draw(n, G, dk), draw(n, G, dv), draw(n, H, dv)
    if decays is None:
        decays = np.log1p(-np.exp2(-np.linspace(1, 8, H))) if H > 1 else np.array([-0.05])
    ld = torch.from_numpy(np.asarray(decays, dtype=np.float32))
    s0, ds = (torch.from_numpy(rng.standard_normal((seqs, H, dk, dv)).astype(np.float32)) for _ in range(2))
    return q, k, v, do, ld, s0, ds


def _f64(x):
    return None if x is None else x.double().cpu().numpy()


def _near(got, want, mag, dtype, terms, parts, what):
    got = _f64(got)
    tol = ROUND[dtype] * np.abs(want) + (terms * U + (3 * 2.0 ** -16 if parts else 0)) * mag + (2.0 ** -25 if dtype == "f16" else 0) + 1e-37
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.max(np.abs(got - want) / tol):.3g} of the tolerance, first at {np.argwhere(bad)[0]}"


def _check(g, dtype, n, H, G, dk, dv, offsets=None, batch=None, with_state=True, scale=1.0, seed=0, decays=None, backward=True):
    torch, _ = _torch()
    from oracle import layer_oracle as lo
    seqs = batch if batch else len(offsets) - 1 if offsets else 1
    q, k, v, do, ld, s0, ds = _inputs(dtype, n, H, G, dk, dv, seqs, seed, decays)
    if not with_state:
        s0 = ds = None
    spans = offsets or [i * (n // seqs) for i in range(seqs + 1)]
    args = [_f64(x) for x in (q, k, v)]
    mags = [np.abs(x) for x in args]
    st, dst = _f64(s0), _f64(ds)
    ab = lambda x: None if x is None else np.abs(x)  # noqa: E731
    terms = max(dk, dv) + 64 + n // 64 + 32
    dev = lambda x: None if x is None else x.cuda()  # noqa: E731
    lead = (lambda x: x.reshape((batch, n // batch) + x.shape[1:])) if batch else (lambda x: x)
    flat = lambda x: x.reshape((n,) + x.shape[-2:])  # noqa: E731
    off = torch.tensor(offsets, dtype=torch.int64).cuda() if offsets else None
    dq, dk_, dv_ = (lead(dev(x)) for x in (q, k, v))
    o, last = g.linear_attention(dq, dk_, dv_, dev(ld), state=dev(s0), offsets=off, scale=scale, want_state=True)
    assert o.dtype == q.dtype and o.shape == dq.shape[:-1] + (dv,)
    want, wl = lo.attention(*args, _f64(ld), st, spans, scale)
    mo, ml = lo.attention(*mags, _f64(ld), ab(st), spans, abs(scale))
    parts = dtype != "f32"
    _near(flat(o), want, mo, dtype, terms, parts, "o")
    _near(last, wl, ml, "f32", terms, False, "final state")
    if not backward:
        return
    grads = g.linear_attention_backward(dq, dk_, dv_, dev(ld), lead(dev(do)), state=dev(s0), grad_state=dev(ds), offsets=off, scale=scale)
    want = lo.attention_backward(*args, _f64(ld), _f64(do), st, dst, spans, scale)
    mag = lo.attention_backward(*mags, _f64(ld), np.abs(_f64(do)), ab(st), ab(dst), spans, abs(scale))
    for name, a, b, m, t in zip(("grad_q", "grad_k", "grad_v", "grad_state"), grads, want, mag, (dtype, dtype, dtype, "f32")):
        if b is None:
            assert a is None
            continue
        _near(flat(a) if name != "grad_state" else a, b, m, t, terms + H // G, parts and name != "grad_state", name)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 127, 130])
def test_lengths(g, dtype, n):
    _check(g, dtype, n, 2, 2, 32, 32, seed=n)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dk,dv", [(1, 1), (3, 5), (8, 32), (16, 64), (32, 128), (33, 31), (40, 64), (64, 64), (64, 24), (64, 128), (80, 96), (96, 65), (90, 20), (128, 90), (100, 7), (128, 32), (128, 64), (127, 128), (128, 128)])
def test_head_sizes(g, dtype, dk, dv):
    _check(g, dtype, 150, 3, 3, dk, dv, seed=dk * 200 + dv)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("H,G", [(4, 1), (4, 2), (6, 3), (1, 1)])
@pytest.mark.parametrize("with_state", [True, False])
def test_shared_heads(g, dtype, H, G, with_state):
    _check(g, dtype, 2 * 90, H, G, 24, 48, batch=2, with_state=with_state, scale=-0.25, seed=H * 10 + G)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offsets", [[0, 0], [0, 0, 0, 5], [0, 64, 64, 65, 193, 200], [0, 1, 2, 3, 4], [0, 300, 1000, 1000], [0, 700] + list(range(701, 790))])
def test_packed_sequences(g, dtype, offsets):
    _check(g, dtype, offsets[-1], 2, 1, 20, 36, offsets=offsets, seed=len(offsets))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dk,dv", [(32, 32), (64, 64), (48, 96), (90, 70), (128, 128)])
def test_segments(g, dtype, dk, dv):
    """Few long sequences, which are cut: dense, and packed with one that ends inside a segment."""
    _check(g, dtype, 1500, 1, 1, dk, dv, seed=dk + dv)
    _check(g, dtype, 1500, 1, 1, dk, dv, offsets=[0, 0, 900, 901, 1500], seed=dk + dv + 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decays(g, dtype):
    """No decay, a full one (log-magnitude of zero), ones that underflow within a chunk, and a growing one."""
    _check(g, dtype, 700, 6, 6, 32, 32, seed=5, decays=[0.0, -np.inf, -200.0, -5.0, -1e-4, 0.01])


def test_slices_of_a_projection(g):
    """q, k, v as slices of one tensor; odd offsets, which the vector accesses cannot take, give the same."""
    torch, _ = _torch()
    for H, G, dk, dv, pad, dtype in ((4, 2, 32, 64, 0, torch.bfloat16), (3, 3, 17, 9, 5, torch.float32), (2, 1, 64, 64, 3, torch.bfloat16)):
        gen = torch.Generator(device="cuda").manual_seed(H)
        x = torch.randn(2, 200, pad + H * dk + G * (dk + dv), device="cuda", generator=gen).to(dtype)
        q, k, v = x[..., pad:].split([H * dk, G * dk, G * dv], dim=-1)
        q, k, v = q.unflatten(-1, (H, dk)), k.unflatten(-1, (G, dk)), v.unflatten(-1, (G, dv))
        ld = torch.linspace(-0.5, -0.01, H, device="cuda")
        do = torch.randn(2, 200, H, dv, device="cuda", generator=gen).to(dtype)
        a = g.linear_attention(q, k, v, ld), *g.linear_attention_backward(q, k, v, ld, do)[:3]
        b = g.linear_attention(q.contiguous(), k.contiguous(), v.contiguous(), ld), *g.linear_attention_backward(q.contiguous(), k.contiguous(), v.contiguous(), ld, do)[:3]
        for s, t in zip(a, b):
            assert torch.equal(s, t)


def test_sequences_and_heads_do_not_reach_each_other(g):
    """A NaN stays in its head and sequence; runs are bitwise repeatable."""
    torch, _ = _torch()
    gen = torch.Generator(device="cuda").manual_seed(3)
    offsets = torch.tensor([0, 100, 230, 400], device="cuda")
    q, k, v, do = (torch.randn(400, 4, 32, device="cuda", generator=gen).bfloat16() for _ in range(4))
    ld = torch.full((4,), -0.1, device="cuda")
    run = lambda: (g.linear_attention(q, k, v, ld, offsets=offsets), *g.linear_attention_backward(q, k, v, ld, do, offsets=offsets)[:3])  # noqa: E731
    clean = run()
    for a, b in zip(clean, run()):
        assert torch.equal(a, b)
    v[150, 2] = float("nan")
    for a, b in zip(clean, run()):
        same = torch.ones(400, 4, dtype=torch.bool, device="cuda")
        same[100:230, 2] = False
        assert torch.equal(a[same], b[same])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("batch,H,G,dk,dv", [(1, 1, 1, 1, 1), (3, 4, 2, 33, 30), (2, 2, 2, 128, 128), (5, 3, 1, 64, 36), (2, 2, 1, 100, 37)])
def test_single_tokens(g, dtype, batch, H, G, dk, dv):
    """One token after another, in place, against the recurrence, and against the same tokens at once."""
    torch, _ = _torch()
    from oracle import layer_oracle as lo
    T = 5
    q, k, v, _, ld, s0, _ = _inputs(dtype, batch * T, H, G, dk, dv, batch, batch + dk)
    seq = lambda x: x.reshape((batch, T) + x.shape[1:]).cuda()  # noqa: E731
    q5, k5, v5 = seq(q), seq(k), seq(v)
    state = s0.cuda()
    other = torch.full_like(state, 7.0)
    first = g.linear_attention_step(q5[:, 0], k5[:, 0], v5[:, 0], ld.cuda(), state, out_state=other, scale=0.5)
    assert torch.equal(state, s0.cuda())
    outs = [g.linear_attention_step(q5[:, t], k5[:, t], v5[:, t], ld.cuda(), state, scale=0.5) for t in range(T)]
    assert torch.equal(outs[0], first)
    spans = [i * T for i in range(batch + 1)]
    args = [_f64(x) for x in (q, k, v)]
    want, wl = lo.attention(*args, _f64(ld), _f64(s0), spans, 0.5)
    mo, ml = lo.attention(*[np.abs(x) for x in args], _f64(ld), np.abs(_f64(s0)), spans, 0.5)
    terms = dk + 4 * T + 16
    _near(torch.stack(outs, 1).reshape(batch * T, H, dv), want, mo, dtype, terms, False, "o")
    _near(state, wl, ml, "f32", terms, False, "state")
    full, last = g.linear_attention(q5, k5, v5, ld.cuda(), state=s0.cuda(), scale=0.5, want_state=True)
    _near(full.reshape(batch * T, H, dv), want, mo, dtype, dk + 64 + 32, dtype == "bf16", "o at once")
    _near(last, wl, ml, "f32", dk + 64 + 32, False, "state at once")


def test_final_state_may_replace_the_first(g):
    torch, _ = _torch()
    import ctypes as C
    q, k, v, _, ld, s0, _ = (x.cuda() for x in _inputs("bf16", 1500, 2, 2, 64, 64, 1, 9))
    o, last = g.linear_attention(q[None], k[None], v[None], ld, state=s0, want_state=True)
    shape, pq, pk, pv = g._attention(q[None], k[None], v[None], ld, None, 1.0)
    need = g.lib.goom_linear_attention_workspace_bytes(C.byref(shape), 0)
    assert need > 0  # one sequence of two heads is cut into segments
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    o2, state = torch.empty_like(o), s0.clone()
    p = lambda t: C.c_void_p(t.data_ptr())  # noqa: E731
    assert g.lib.goom_linear_attention(g._ctx, C.byref(shape), pq, pk, pv, p(ld), None, p(state), p(o2), p(state), p(ws), need) == 0
    assert torch.equal(o2, o) and torch.equal(state, last)


@pytest.mark.parametrize("offsets", [[100, 700, 1400], [700, 200, 1100], [1500, 1500, -3], [5, 5000, 9]])
def test_offsets_that_are_none(g, offsets):
    """Offsets that reach outside 0 .. tokens are cut off there; what they name is computed.  Offsets that fall promise no results, but
    nothing outside the sequences they name is touched either."""
    torch, _ = _torch()
    from oracle import layer_oracle as lo
    import ctypes as C
    q, k, v, do, ld, s0, _ = (x.cuda() for x in _inputs("f32", 1500, 1, 1, 32, 32, 2, 3))
    off = torch.tensor(offsets, device="cuda")
    cut = [(min(max(a, 0), 1500), min(max(b, min(max(a, 0), 1500)), 1500)) for a, b in zip(offsets, offsets[1:])]
    shape, pq, pk, pv = g._attention(q, k, v, ld, off, 1.0)
    need = g.lib.goom_linear_attention_workspace_bytes(C.byref(shape), 1)
    ws = torch.full((need + 4096,), 9, dtype=torch.uint8, device="cuda")
    held, last = torch.full((1500 + 128, 1, 32), 7.0, device="cuda"), torch.empty(2, 1, 32, 32, device="cuda")
    o = held[64:-64]
    p = lambda t: C.c_void_p(t.data_ptr())  # noqa: E731
    assert g.lib.goom_linear_attention(g._ctx, C.byref(shape), pq, pk, pv, p(ld), p(off), p(s0), p(o), p(last), p(ws), need) == 0
    inside = torch.zeros(1500, dtype=torch.bool)
    rising = all(a <= b for a, b in zip([a for a, _ in cut], [a for a, _ in cut][1:]))
    for s, (a, b) in enumerate(cut):
        inside[a:b] = True
        if not rising:
            continue
        want, wl = lo.attention(_f64(q)[a:b], _f64(k)[a:b], _f64(v)[a:b], _f64(ld), _f64(s0)[s:s + 1])
        mag, ml = lo.attention(*(np.abs(_f64(x)[a:b]) for x in (q, k, v)), _f64(ld), np.abs(_f64(s0)[s:s + 1]))
        _near(last[s:s + 1], wl, ml, "f32", 160, False, "state")
        _near(o[a:b], want, mag, "f32", 160, False, "o")
    assert (o.cpu()[~inside] == 7).all() and (held[:64] == 7).all() and (held[-64:] == 7).all() and (ws[need:] == 9).all()


def test_another_stream_and_graph(g):
    """Work follows the context's stream; a captured call, replayed on new inputs, gives what an eager one gives."""
    torch, _ = _torch()
    q, k, v, do, ld, s0, ds = (x.cuda() for x in _inputs("bf16", 1200, 2, 1, 64, 32, 1, 4))
    call = lambda: (g.linear_attention(q, k, v, ld, state=s0), *g.linear_attention_backward(q, k, v, ld, do, state=s0, grad_state=ds))  # noqa: E731
    want = call()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    old = g._stream
    try:
        with torch.cuda.stream(stream):
            g.set_stream(stream)
            stream.wait_stream(old)
            got = call()
            for a, b in zip(got, want):
                assert torch.equal(a, b)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                held = call()
            for seed in (5, 6, 7):
                for x, y in zip((q, k, v, do), _inputs("bf16", 1200, 2, 1, 64, 32, 1, seed)):
                    x.copy_(y)
                graph.replay()
                kept = [x.clone() for x in held]
                torch.cuda.synchronize()
                for a, b in zip(kept, call()):
                    assert torch.equal(a, b)
    finally:
        torch.cuda.synchronize()
        g.set_stream(old)

"""Linear attention as training and serving programs call it, beside the forms that test_gpu_linear_attention.py takes: without a
final state, without an initial one's gradient.  References and tolerances are those of that file (the recurrence in 64 bits)."""
import pytest

from test_gpu_linear_attention import _check, _f64, _inputs, _near, g  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,H,G,dk,dv,with_state", [(1, 2, 1, 16, 16, True), (200, 3, 3, 40, 64, False), (1500, 1, 1, 64, 64, False), (1500, 2, 1, 128, 128, True), (700, 2, 2, 50, 100, False)])
def test_outputs_without_a_final_state(g, dtype, n, H, G, dk, dv, with_state):  # noqa: F811
    """The ordinary training call: outputs as the recurrence has them, and the bits of a call that asks for the state."""
    import torch
    import numpy as np
    from oracle import layer_oracle as lo
    q, k, v, _, ld, s0, _ = _inputs(dtype, n, H, G, dk, dv, 1, n + dk)
    args = [x.cuda()[None] for x in (q, k, v)] + [ld.cuda()]
    s = s0.cuda() if with_state else None
    o = g.linear_attention(*args, state=s)
    both, _ = g.linear_attention(*args, state=s, want_state=True)
    assert torch.equal(o, both)
    st = _f64(s0) if with_state else None
    want, _ = lo.attention(*[_f64(x) for x in (q, k, v)], _f64(ld), st)
    mag, _ = lo.attention(*[np.abs(_f64(x)) for x in (q, k, v)], _f64(ld), None if st is None else np.abs(st))
    _near(o[0], want, mag, dtype, max(dk, dv) + 64 + n // 64 + 32, dtype != "f32", "o")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_gradients_without_a_state(g, dtype):  # noqa: F811
    """grad_k and grad_v do not depend on whether the initial state's gradient is formed beside them."""
    import torch
    q, k, v, do, ld, _, _ = (x.cuda() for x in _inputs(dtype, 1500, 2, 1, 64, 64, 1, 21))
    args = [x[None] for x in (q, k, v)] + [ld, do[None]]
    a = g.linear_attention_backward(*args)
    b = g.linear_attention_backward(*args, state=torch.zeros(1, 2, 64, 64, device="cuda"), grad_state=torch.zeros(1, 2, 64, 64, device="cuda"))
    for x, y in zip(a[:3], b[:3]):
        assert torch.equal(x, y)


def _neighbours(got, want):
    """Share of the entries that are not the exact value rounded to their type."""
    import torch
    return float((got != torch.from_numpy(want).cuda().to(got.dtype)).double().mean())


@pytest.mark.parametrize("shape", [(700, 2, 2, 128, 128), (1500, 2, 1, 64, 64)])
def test_bfloat16_outputs_are_sums_of_floats(g, shape):  # noqa: F811
    """Operands that are computed on the way lose no bits that a float holds.  An output whose float sum is off by e = c u s (s: the
    spread of the outputs, u = 2^-24, c some 4 where rounding errors add up at random) is rounded to a neighbour with probability 2 e
    over the spacing of bfloat16 there (2^-8 |y| to 2^-7 |y|, 2^-7.5 taken): 8 u s / (2^-7.5 |y|) = 2^-13.5 s / |y|, whose mean over
    normal y, cut off where it reaches one, is some 7 times 2^-13.5 = 0.06 %.  0.1 % is
    allowed.  With operands of 16 bits, off by up to 2^-17 of themselves, e is some 2^-18 s, 16 times as much."""
    from oracle import layer_oracle as lo
    n, H, G, dk, dv = shape
    q, k, v, do, ld, _, _ = _inputs("bf16", n, H, G, dk, dv, 1, 31)
    args = [x.cuda()[None] for x in (q, k, v)] + [ld.cuda()]
    ref = [_f64(x) for x in (q, k, v)]
    want, _ = lo.attention(*ref, _f64(ld))
    assert _neighbours(g.linear_attention(*args)[0], want) <= 1e-3
    grads = g.linear_attention_backward(*args, do.cuda()[None])
    for got, want in zip(grads[:3], lo.attention_backward(*ref, _f64(ld), _f64(do))):
        assert _neighbours(got[0], want) <= 1e-3


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,G,dk,dv", [(4, 2, 32, 64), (4, 4, 32, 64), (3, 1, 20, 33)])
@pytest.mark.parametrize("offsets", [[100, 700, 1400], [0, 700, 700, 1463], [37, 37], [1500, 1500, -3], [5, 5000, 9]])
def test_gradients_of_tokens_without_a_sequence(g, dtype, H, G, dk, dv, offsets):  # noqa: F811
    """Tokens before the first and after the last sequence (padding of a packed batch): their gradients are not written, whatever the
    workspace holds."""
    import ctypes as C
    import torch
    import numpy as np
    from oracle import layer_oracle as lo
    n, seqs = 1500, len(offsets) - 1
    q, k, v, do, ld, s0, ds = (x.cuda() for x in _inputs(dtype, n, H, G, dk, dv, seqs, 7))
    off = torch.tensor(offsets, device="cuda")
    shape, pq, pk, pv = g._attention(q, k, v, ld, off, 1.0)
    need = g.lib.goom_linear_attention_backward_workspace_bytes(C.byref(shape), 1)
    ws = torch.full((need // 4 + 1024,), float("nan"), device="cuda")
    grads = [torch.full_like(x, 7.0) for x in (q, k, v)]
    gs = torch.empty_like(s0)
    p = lambda t: C.c_void_p(t.data_ptr())  # noqa: E731
    assert g.lib.goom_linear_attention_backward(g._ctx, C.byref(shape), pq, pk, pv, p(ld), p(off), p(s0), p(do), p(ds), p(grads[0]), p(grads[1]), p(grads[2]), p(gs),
                                                p(ws), need) == 0
    assert ws[need // 4:].isnan().all()
    cut = [min(max(a, 0), n) for a in offsets]
    inside = torch.zeros(n, dtype=torch.bool)
    for s, (a, b) in enumerate(zip(cut, cut[1:])):
        inside[a:b] = True
        if b < a:
            continue
        args = [_f64(x[a:b]) for x in (q, k, v)]
        st, dst = _f64(s0[s:s + 1]), _f64(ds[s:s + 1])
        want = lo.attention_backward(*args, _f64(ld), _f64(do[a:b]), st, dst)
        mag = lo.attention_backward(*[np.abs(x) for x in args], _f64(ld), np.abs(_f64(do[a:b])), np.abs(st), np.abs(dst))
        terms = max(dk, dv) + 64 + n // 64 + 32 + H // G
        for name, got, w, m in zip(("grad_q", "grad_k", "grad_v"), grads, want, mag):
            _near(got[a:b], w, m, dtype, terms, False, name)
        _near(gs[s:s + 1], want[3], mag[3], "f32", terms, False, "grad_state")
    for got in grads:
        assert (got[~inside.cuda()] == 7).all()


@pytest.mark.parametrize("dtype,decay,offsets", [("bf16", 1.5, [0, 40]), ("bf16", 1.5, [0, 1, 30, 70]), ("f32", 3.0, [0, 20]), ("f32", 2.9, [0, 7, 7, 24]), ("bf16", 0.75, [0, 100]),
                                                 ("bf16", 0.7, [0, 65, 100, 190])])
def test_growing_decays(g, dtype, decay, offsets):  # noqa: F811
    """Decays above one, within the range of floats over the sequences' lengths but not over those of whole chunks: the chunks' missing
    rows count for nothing.  The exponent of a power, age times log2 of the decay, is rounded three times: 3 u of itself, age |log decay|
    times the power, beside what test_gpu_linear_attention.py allows."""
    import torch
    import numpy as np
    from oracle import layer_oracle as lo
    n, seqs, dk, dv = offsets[-1], len(offsets) - 1, 32, 40
    q, k, v, do, ld, s0, ds = _inputs(dtype, n, 2, 1, dk, dv, seqs, 17, decays=[decay, -0.1])
    args, st, dst = [_f64(x) for x in (q, k, v)], _f64(s0), _f64(ds)
    mags = [np.abs(x) for x in args]
    terms = dv + 64 + 32 + 2 + int(3 * decay * n)
    off = torch.tensor(offsets).cuda()
    dev = [x.cuda() for x in (q, k, v, ld)]
    o, last = g.linear_attention(*dev, state=s0.cuda(), offsets=off, want_state=True)
    for name, got, want, mag, t in zip(("o", "state"), (o, last), lo.attention(*args, _f64(ld), st, offsets), lo.attention(*mags, _f64(ld), np.abs(st), offsets), (dtype, "f32")):
        _near(got, want, mag, t, terms, False, name)
    grads = g.linear_attention_backward(*dev, do.cuda(), state=s0.cuda(), grad_state=ds.cuda(), offsets=off)
    want = lo.attention_backward(*args, _f64(ld), _f64(do), st, dst, offsets)
    mag = lo.attention_backward(*mags, _f64(ld), np.abs(_f64(do)), np.abs(st), np.abs(dst), offsets)
    for name, got, w, m, t in zip(("grad_q", "grad_k", "grad_v", "grad_state"), grads, want, mag, (dtype, dtype, dtype, "f32")):
        _near(got, w, m, t, terms, False, name)

"""Calls of the block operators that a program makes now and then: nothing to do, a NaN somewhere, many short sequences, widths that only the largest
workgroups hold, inputs given twice.  What is compared is computed twice by the library (in parts, or again), so that it has to be the same to the bit, except
parameters' gradients, whose tokens are summed in other groups: 2 sums of n floats, some n^(1/2) u of the terms' size sqrt(n) apart: n u = 1e-4 for n = 1100, 1e-3 is allowed."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def g():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2510_03426_amd import Goom
    g = Goom(0)
    yield g
    g.close()


def _delta(n, H, Q, d, dtype, seed=1):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    q, k = (torch.nn.functional.normalize(new(n, Q, d), dim=-1).to(dtype) for _ in range(2))
    return [q, k, new(n, H, d).to(dtype), -new(n, H).abs() / 4, torch.sigmoid(new(n, H)), new(n, H, d).to(dtype)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_a_nan_stays_in_its_head_and_sequence(g, dtype):
    import torch
    for heads, n in ((4, 200), (1, 1800)):  # whole sequences, and segments of them
        *x, go = _delta(n, heads, heads, 40, getattr(torch, dtype))
        off = torch.tensor([0, n // 4, n // 2, n], device="cuda")
        run = lambda: g.gated_delta(*x, offsets=off, want_state=True) + g.gated_delta_backward(*x, go, offsets=off)[:5]  # noqa: E731
        before, again = run(), run()
        assert all(torch.equal(a, b) for a, b in zip(before, again))
        at = n // 4 + 30
        for i, index in ((2, (at, 0, 7)), (1, (at, 0, 3)), (3, (at, 0)), (4, (at, 0))):
            keep = x[i][index].clone()
            x[i][index] = math.nan
            after = run()
            x[i][index] = keep
            assert after[0][at:n // 2, 0].isnan().any() and after[1][1, 0].isnan().any()
            for j, (a, b) in enumerate(zip(before, after)):
                a, b = a.clone(), b.clone()
                for t in (a, b):
                    if j == 1:
                        t[1, 0] = 0
                    else:
                        t[n // 4:n // 2, 0] = 0
                assert torch.equal(a, b), (i, j)


def test_many_short_sequences(g):
    import torch
    lengths = torch.tensor([0, 1, 3, 2, 0, 5], device="cuda").repeat(500)
    off = torch.cat([lengths.new_zeros(1), lengths.cumsum(0)])
    n = int(off[-1])
    *x, go = _delta(n, 4, 2, 32, torch.bfloat16)
    state = torch.randn(3000, 4, 32, 32, device="cuda")
    o, last = g.gated_delta(*x, state=state, offsets=off, want_state=True)
    grads = g.gated_delta_backward(*x, go, state=state, grad_state=state, offsets=off)
    assert torch.equal(last[0::6], state[0::6]) and torch.equal(grads[5][4::6], state[4::6])
    for s in (1, 2, 3, 5, 2999):
        part = slice(int(off[s]), int(off[s + 1]))
        one = [t[part][None].contiguous() for t in x]
        o1, last1 = g.gated_delta(*one, state=state[s:s + 1], want_state=True)
        assert torch.equal(o1[0], o[part]) and torch.equal(last1[0], last[s])
        for a, b in zip(g.gated_delta_backward(*one, go[part][None].contiguous(), state=state[s:s + 1], grad_state=state[s:s + 1]), grads):
            assert torch.equal(a[0], b[s] if a.dim() == 4 and a.shape[-2:] == (32, 32) and a.shape[1] == 4 and b.shape[0] == 3000 else b[part]), s


def test_nothing_to_do(g):
    import torch
    b, f = torch.bfloat16, torch.float32
    z = lambda *s, t=b: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
    assert g.gated_delta_step(z(0, 2, 16), z(0, 2, 16), z(0, 4, 24), z(0, 4, t=f), z(0, 4, t=f), z(0, 4, 16, 24, t=f)).shape == (0, 4, 24)
    for lead in ((0, 7), (3, 0)):
        args = z(*lead, 2, 16), z(*lead, 2, 16), z(*lead, 4, 24), z(*lead, 4, t=f), z(*lead, 4, t=f)
        o, last = g.gated_delta(*args, want_state=True)
        assert o.shape == lead + (4, 24) and last.shape == (lead[0], 4, 16, 24) and not last.any()
        assert [t.shape for t in g.gated_delta_backward(*args, o)[:5]] == [t.shape for t in args]
    for call in (g.norm_after, g.norm_before):
        call(z(0, 32), gate=z(0, 32), residual=z(0, 32), kind="layer", want_stats=True)
    q, k = g.rotary(z(2, 0, 4, 16), z(2, 0, 1, 16), torch.zeros(2, 0, dtype=torch.int64, device="cuda"), torch.ones(8, device="cuda"))
    assert q.shape == (2, 0, 4, 16) and k.shape == (2, 0, 1, 16)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("channels", [4096, 6000, 8200, 16384])
def test_wide_norms_of_many_tokens(g, dtype, channels):
    """More tokens than workgroups: each goes on from token to token."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(channels)
    x, z, r = (torch.randn(1100, channels, device="cuda", generator=gen).to(getattr(torch, dtype)) for _ in range(3))
    w, b, s = (1 + 0.1 * torch.randn(channels, device="cuda", generator=gen) for _ in range(3))
    kw = dict(weight=w, bias=b, scale=s, kind="layer", activation="gelu")

    def both(i):
        p, t, q = x[i], z[i], r[i]
        y, m, rs = g.norm_after(p, gate=t, residual=q, want_stats=True, **kw)
        out = [y] + list(g.norm_after_backward(p, q, m, rs, gate=t, **kw))
        y, h, m, rs = g.norm_before(p, gate=t, residual=q, want_stats=True, **kw)
        return out + [y, h] + list(g.norm_before_backward(p, h, q, m, rs, grad_h=p, gate=t, **kw))
    whole, parts = both(slice(0, 1100)), [both(slice(i, i + 100)) for i in range(0, 1100, 100)]
    for j, a in enumerate(whole):
        if a.dim() == 2:
            assert torch.equal(a, torch.cat([p[j] for p in parts])), j
        else:
            total = sum(p[j].double() for p in parts)
            assert (a.double() - total).abs().max() < 1e-3 * total.abs().max(), j


def test_one_tensor_as_two_inputs(g):
    import torch
    x = torch.randn(40, 256, device="cuda")
    a, b = g.norm_before(x, residual=x), g.norm_before(x, residual=x.clone())
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert torch.equal(g.norm_after(x, gate=x, residual=x), g.norm_after(x, gate=x.clone(), residual=x.clone()))
    q = torch.nn.functional.normalize(torch.randn(2, 70, 4, 32, device="cuda"), dim=-1)
    ld, beta = -torch.rand(2, 70, 4, device="cuda"), torch.rand(2, 70, 4, device="cuda")
    one, two = g.gated_delta(q, q, q, ld, beta), g.gated_delta(q, q.clone(), q.clone(), ld, beta)
    assert torch.equal(one, two)
    for s, t in zip(g.gated_delta_backward(q, q, q, ld, beta, q)[:5], g.gated_delta_backward(q, q.clone(), q.clone(), ld, beta, q.clone())):
        assert torch.equal(s, t)
    at, f = torch.arange(70, device="cuda").repeat(2, 1), torch.rand(16, device="cuda")
    s, t = g.rotary(q, q, at, f)
    assert torch.equal(s, t)


@pytest.mark.parametrize("seqs", [600, 5000])
def test_the_order_of_sequences_changes_nothing(g, seqs):
    """Few long sequences among many short ones, then all of them the other way round: the same bits for each."""
    import torch
    lengths = torch.randint(0, 40, (seqs,), generator=torch.Generator().manual_seed(seqs))
    lengths[7], lengths[seqs // 2], lengths[-1] = 70000, 5000, 66000
    n = int(lengths.sum())
    ends = torch.cat([lengths.new_zeros(1), lengths.cumsum(0)])
    turned = torch.cat([torch.arange(int(ends[s]), int(ends[s + 1])) for s in range(seqs - 1, -1, -1)]).cuda()
    off, off2 = ends.cuda(), torch.cat([lengths.new_zeros(1), lengths.flip(0).cumsum(0)]).cuda()
    *x, go = _delta(n, 1, 1, 16, torch.bfloat16)
    state = torch.randn(seqs, 1, 16, 16, device="cuda")
    o, last = g.gated_delta(*x, state=state, offsets=off, want_state=True)
    grads = g.gated_delta_backward(*x, go, state=state, offsets=off)
    y, go2, state2 = [t[turned] for t in x], go[turned], state.flip(0).contiguous()
    o2, last2 = g.gated_delta(*y, state=state2, offsets=off2, want_state=True)
    grads2 = g.gated_delta_backward(*y, go2, state=state2, offsets=off2)
    assert torch.equal(o[turned], o2) and torch.equal(last.flip(0), last2) and torch.equal(grads[5].flip(0), grads2[5])
    assert all(torch.equal(a[turned], b) for a, b in zip(grads[:5], grads2[:5]))
    assert all(bool(t.float().isfinite().all()) for t in (o, last) + grads)

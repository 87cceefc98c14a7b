"""Norms around a block where a parameter or an entry is no number: what stands outside a group does not reach it."""
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


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("dtype,channels,groups", [("float32", 48, 4), ("float32", 9, 3), ("bfloat16", 120, 5), ("float32", 2 * 1036, 2), ("bfloat16", 2 * 5000, 2), ("float16", 2 * 9000, 2)])
def test_a_scale_that_is_no_number_stays_in_its_group(g, kind, bad, dtype, channels, groups):
    """The lanes of a team that have no channels count for nothing, whatever parameters they read."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(channels)
    t = getattr(torch, dtype)
    x, r, z, gy = (torch.randn(7, channels, device="cuda", generator=gen).to(t) for _ in range(4))
    w, b = (1 + 0.1 * torch.randn(channels, device="cuda", generator=gen) for _ in range(2))
    s = torch.rand(channels, device="cuda", generator=gen) + 0.5
    spoilt = s.clone()
    spoilt[0] = bad
    cg = channels // groups
    for gate in (None, z):
        kw = dict(groups=groups, weight=w, bias=b, gate=gate, kind=kind)
        for after in (False, True):
            run = g.norm_after if after else g.norm_before
            got, want = (run(x, scale=p, residual=r, want_stats=True, **kw) for p in (spoilt, s))
            outs = 1 if after else 2
            assert all(torch.equal(a[:, cg:], c[:, cg:]) for a, c in zip(got[:outs], want[:outs]))
            assert all(torch.equal(a[:, 1:], c[:, 1:]) for a, c in zip(got[outs:], want[outs:]) if a is not None)
            assert not torch.isfinite(got[0][:, 0].float()).any()
            stats = want[outs:]  # the way back, from statistics that are numbers
            back = (lambda p: g.norm_after_backward(x, gy, *stats, scale=p, **kw)) if after else (lambda p: g.norm_before_backward(x, want[1], gy, *stats, scale=p, **kw))
            for a, c in zip(back(spoilt), back(s)):
                if a is not None:
                    assert torch.equal(a[..., cg:], c[..., cg:])

"""The gated delta rule's chunks, one by one: the same tokens give the same bits wherever and whenever they are worked on."""
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


@pytest.mark.parametrize("dtype,n", [("bfloat16", 64), ("bfloat16", 51), ("float32", 32), ("float32", 19), ("float16", 32)])
def test_equal_chunks_give_equal_bits(g, dtype, n):
    """30,000 chunks of the same tokens: what the lanes of a wave hand one another through LDS is there in all of them."""
    import torch
    seqs, H, d = 30000 // 4, 4, 32
    t = getattr(torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(n)
    k = torch.nn.functional.normalize(torch.randn(1, n, 1, d, device="cuda", generator=gen) + 0.5, dim=-1)  # (keys that are much alike: full systems)
    q, v, go = (torch.randn(1, n, 1, d, device="cuda", generator=gen) for _ in range(3))
    ld, beta = -0.05 * torch.rand(1, n, 1, device="cuda", generator=gen), torch.rand(1, n, 1, device="cuda", generator=gen)
    all_of = lambda x: x.expand(seqs, n, H, *x.shape[3:]).contiguous()  # noqa: E731
    q, k, v, go = (all_of(x).to(t) for x in (q, k, v, go))
    ld, beta = all_of(ld), all_of(beta)
    for turn in range(3):
        o, last = g.gated_delta(q, k, v, ld, beta, want_state=True)
        assert bool(o.float().isfinite().all())
        assert torch.equal(o, o[:1, :, :1].expand_as(o)) and torch.equal(last, last[:1, :1].expand_as(last)), turn
        for x in g.gated_delta_backward(q, k, v, ld, beta, go)[:5]:
            assert torch.equal(x, x[:1, :, :1].expand_as(x)), turn

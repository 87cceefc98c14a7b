"""A context's workspace where its stream is not torch's current one: memory that it lets go is not handed to the current stream's next tensor, eagerly or in a
capture whose branches run side by side."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture()
def side():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2510_03426_amd import Goom
    stream = torch.cuda.Stream()
    h = Goom(0, stream)
    yield stream, h
    torch.cuda.synchronize()
    h.close()


BYTES = 40 << 20  # (a block of its own in torch's allocator)


def _used_again(at):
    """Tensors of the workspace's size on the current stream: does one of them take its place?"""
    import torch
    mine = [torch.empty(BYTES, dtype=torch.uint8, device="cuda") for _ in range(4)]
    return any(t.data_ptr() == at for t in mine)


def test_what_is_let_go_stays_with_its_stream(side):
    import torch
    stream, h = side
    at = h.workspace(BYTES)[0].data_ptr()
    h.workspace(BYTES + (4 << 20))  # more: the first is let go
    assert not _used_again(at)
    torch.cuda.synchronize()


def test_captured_branches(side):
    """A branch on the context's stream, and one on the capture's own that fills tensors of the same sizes meanwhile."""
    import torch
    stream, h = side
    gen = torch.Generator(device="cuda").manual_seed(1)
    n, H, d = 3000, 4, 64
    q, k, v, go = (torch.randn(2, n, H, d, device="cuda", generator=gen).bfloat16() for _ in range(4))
    k = torch.nn.functional.normalize(k.float(), dim=-1).bfloat16()
    ld, beta = -torch.rand(2, n, H, device="cuda", generator=gen), torch.rand(2, n, H, device="cuda", generator=gen)
    run = lambda: h.gated_delta_backward(q, k, v, ld, beta, go)[:5]  # noqa: E731
    stream.wait_stream(torch.cuda.current_stream())
    want = run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        stream.wait_stream(torch.cuda.current_stream())
        at = h.workspace(BYTES)[0].data_ptr()
        reused = _used_again(at)
        got = run()
        others = [torch.full((size,), 0x7F, dtype=torch.uint8, device="cuda") for size in (BYTES, 100 << 20, 300 << 20)]
        torch.cuda.current_stream().wait_stream(stream)
    assert not reused
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(bool((t == 0x7F).all()) for t in others)
        q.mul_(-1)
        stream.wait_stream(torch.cuda.current_stream())
        want = run()
        torch.cuda.synchronize()

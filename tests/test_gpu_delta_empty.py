"""The gated delta rule over packed sequences that are empty, all of them or nearly all: states and their gradients pass through, bit for bit, whatever
the workspace held before."""
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


def _fill(g, what, nbytes=1 << 22):
    """The handle's workspace as another call may have left it."""
    import torch
    ws = g.workspace(nbytes)[0]
    if what == "7f":
        ws.fill_(0x7F)
    else:  # whole numbers that are sequences, each many times
        ws[:ws.numel() // 4 * 4].view(torch.int32).copy_(torch.arange(ws.numel() // 4, device="cuda", dtype=torch.int32) % 7)


@pytest.mark.parametrize("what", ["7f", "small"])
@pytest.mark.parametrize("seqs,H,dtype", [(32, 16, "bfloat16"), (300, 16, "bfloat16"), (300, 1, "float32"), (17, 16, "float16"), (5000, 2, "float32")])
def test_all_empty(g, what, seqs, H, dtype):
    import torch
    t = getattr(torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(seqs)
    dk, dv = 24, 40
    state, grad = (torch.randn(seqs, H, dk, dv, device="cuda", generator=gen) for _ in range(2))
    q, v = torch.zeros(0, H, dk, device="cuda", dtype=t), torch.zeros(0, H, dv, device="cuda", dtype=t)
    ld = torch.zeros(0, H, device="cuda")
    off = torch.zeros(seqs + 1, dtype=torch.int64, device="cuda")
    _fill(g, what)
    o, last = g.gated_delta(q, q, v, ld, ld, state=state, offsets=off, want_state=True)
    assert o.shape == (0, H, dv) and torch.equal(last, state)
    _fill(g, what)
    grads = g.gated_delta_backward(q, q, v, ld, ld, v, state=state, grad_state=grad, offsets=off)
    assert torch.equal(grads[5], grad)
    last = g.gated_delta(q, q, v, ld, ld, offsets=off, want_state=True)[1]
    assert (last == 0).all()


@pytest.mark.parametrize("what", ["7f", "small"])
def test_one_of_many_has_tokens(g, what):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(3)
    seqs, H, d, n, at = 400, 2, 32, 70, 133
    state, grad = (torch.randn(seqs, H, d, d, device="cuda", generator=gen) for _ in range(2))
    q, k, v, go = (torch.randn(n, H, d, device="cuda", generator=gen) * d ** -0.5 for _ in range(4))
    ld, beta = -torch.rand(n, H, device="cuda", generator=gen), torch.rand(n, H, device="cuda", generator=gen)
    off = torch.zeros(seqs + 1, dtype=torch.int64, device="cuda")
    off[at + 1:] = n
    _fill(g, what)
    o, last = g.gated_delta(q, k, v, ld, beta, state=state, offsets=off, want_state=True)
    one, end = g.gated_delta(*(x.unsqueeze(0) for x in (q, k, v, ld, beta)), state=state[at:at + 1], want_state=True)
    others = torch.arange(seqs, device="cuda") != at
    assert torch.equal(o, one[0]) and torch.equal(last[at], end[0]) and torch.equal(last[others], state[others])
    _fill(g, what)
    grads = g.gated_delta_backward(q, k, v, ld, beta, go, state=state, grad_state=grad, offsets=off)
    want = g.gated_delta_backward(*(x.unsqueeze(0) for x in (q, k, v, ld, beta, go)), state=state[at:at + 1], grad_state=grad[at:at + 1])
    assert all(torch.equal(a, b[0]) for a, b in zip(grads[:5], want[:5]))
    assert torch.equal(grads[5][at], want[5][0]) and torch.equal(grads[5][others], grad[others])

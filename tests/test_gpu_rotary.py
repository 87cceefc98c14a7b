"""Rotary positions, through the library, against complex numbers in 64 bits.

Tolerances.  An angle is a product in 64 bits, taken to a fraction of a turn there and rounded to 2^-25 of one: 2 pi 2^-25 < 2^-22.3, times the entries' size.  The
library's sine and cosine of it add two units of 2^-24, the scale's product one, the two products and their sum three more: less than 2^-20 of
|x1| + |x2| in all.  The stored result is rounded once more: eps / 2 of it."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


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


@pytest.mark.parametrize("dtype", ["bf16", "f32", "f16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n,H,G,dim,pairs", [(1, 1, 0, 2, 1), (5, 4, 2, 64, 32), (300, 2, 1, 77, 19), (33, 3, 3, 40, 8), (7, 16, 4, 128, 64), (4, 1, 1, 9, 3), (3, 2, 2, 17, 7), (1100, 20, 4, 100, 50)])
def test_turns(g, dtype, interleaved, n, H, G, dim, pairs):
    import torch
    from oracle import layer_oracle as lo
    rng = np.random.default_rng(n + dim)
    q, k = (torch.from_numpy(rng.standard_normal((n, h, dim)).astype(np.float32)).to(_types()[dtype]) for h in (H, G))
    pos = torch.from_numpy(rng.integers(0, 1 << 20, n))
    pos[0] = (1 << 40) + 12345 if n > 1 else 0
    pos[-1] = -3 if n > 2 else pos[-1]
    f = torch.from_numpy(np.float32(10000.0) ** -(np.arange(pairs, dtype=np.float32) / pairs))
    for scale, run, back in ((1.3, g.rotary, False), (-0.7, g.rotary_backward, True)):
        oq, ok = run(q.cuda(), k.cuda() if G else None, pos.cuda(), f.cuda(), interleaved=interleaved, scale=scale)
        assert (ok is None) == (G == 0)
        for x, o in ((q, oq), (k, ok)):
            if o is None:
                continue
            want = lo.rotary(x.double().numpy(), pos.numpy(), f.numpy(), interleaved, scale, back)
            a = np.abs(x.double().numpy())
            size = lo.rotary(a, np.zeros(n), f.numpy(), interleaved)
            one, two = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if interleaved else (slice(0, pairs), slice(pairs, 2 * pairs))
            size[..., one] = size[..., two] = a[..., one] + a[..., two]
            # (2^40 positions times 2^-53 of an angle: 2^-13 of a turn's part is below the rest where frequencies are below one)
            tol = HALF[dtype] * np.abs(want) + 2.0 ** -20 * abs(scale) * size + (2.0 ** -25 if dtype == "f16" else 0)
            if n > 1:
                tol[0] += 2.0 ** -11 * size[0]
            assert (np.abs(o.double().cpu().numpy() - want) <= tol).all()
            assert torch.equal(o.cpu()[..., 2 * pairs:], x[..., 2 * pairs:])


def test_slices_streams_and_no_tokens(g):
    import torch
    from paper_2510_03426_amd import Goom, rotary_frequencies
    f, scale = rotary_frequencies(16, factor=4.0, method="parts", trained=512, device="cuda")
    fused = torch.randn(2, 9, 3 * 4 * 32, device="cuda").bfloat16()
    q, k, _ = (t.unflatten(-1, (4, 32)) for t in fused.split(128, dim=-1))
    pos = torch.arange(9, device="cuda").repeat(2, 1) + 100
    a = g.rotary(q, k, pos, f, scale=scale)
    b = g.rotary(q.contiguous(), k.contiguous(), pos, f, scale=scale)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        h = Goom(0, side)
        h.rotary(q, k, pos, f, scale=scale)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = h.rotary(q, k, pos, f, scale=scale)
    torch.cuda.synchronize()
    for i in range(3):
        pos.add_(i)
        graph.replay()
        want = g.rotary(q, k, pos, f, scale=scale)
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    h.close()
    none = torch.zeros(0, 4, 32, device="cuda")
    assert g.rotary(none, None, torch.zeros(0, dtype=torch.int64, device="cuda"), f)[0].shape == (0, 4, 32)
    ok = dict(q=q, k=k, positions=pos, frequencies=f)
    for kw in (dict(positions=pos.int()), dict(positions=pos[0]), dict(frequencies=f.double()), dict(k=k.float()), dict(k=k[..., :30]), dict(k=k[:1])):
        with pytest.raises(ValueError):
            g.rotary(**{**ok, **kw})
    from paper_2510_03426_amd import GoomError
    with pytest.raises(GoomError):
        g.rotary(**{**ok, "frequencies": torch.ones(17, device="cuda")})

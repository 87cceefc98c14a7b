"""Rotary positions up to 2^53, against angles from whole numbers.  A position times a float frequency is a whole number times a power of two; its part of a
turn is taken with 1 / 2 pi as a whole number of 2^-400, so nothing is lost before the last rounding to 64 bits.

Tolerances: those of test_gpu_rotary.py for every position: the part of a turn is rounded to 2^-25 of one (2 pi 2^-25 < 2^-22.3), sine and cosine add two units of
2^-24, the scale's product one, the two products and their sum three: less than 2^-20 of |x1| + |x2|; the stored result half a unit of its type."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
BITS = 400


def _pi(bits):
    """pi 2^bits by Machin's formula, 16 atan(1/5) - 4 atan(1/239)."""
    one = 1 << (bits + 32)

    def atan(n):
        total, term, k = 0, one // n, 1
        while term:
            total += term // k if k % 4 == 1 else -(term // k)
            term //= n * n
            k += 2
        return total
    return (16 * atan(5) - 4 * atan(239)) >> 32


TURNS = (1 << (2 * BITS)) // (2 * _pi(BITS))  # 2^BITS / 2 pi


def _angles(positions, frequencies):
    """Angles in -pi .. pi."""
    out = np.empty((len(positions), len(frequencies)))
    for j, f in enumerate(frequencies):
        num, den = float(f).as_integer_ratio()
        for i, p in enumerate(positions):
            part = (int(p) * num * TURNS // den) % (1 << BITS)
            if part >> (BITS - 1):
                part -= 1 << BITS
            out[i, j] = 2 * math.pi * (part / (1 << BITS))
    return out


def test_pi():
    assert _pi(60) == 3622009729038561421  # 3.14159265358979323846.. 2^60, rounded down


@pytest.fixture(scope="module")
def g():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2510_03426_amd import Goom
    g = Goom(0)
    yield g
    g.close()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,pairs", [(2, 1), (64, 32), (77, 19), (24, 3), (600, 130), (200, 1)])
def test_positions_up_to_2_53(g, dtype, interleaved, dim, pairs):
    import torch
    t = getattr(torch, dtype)
    rng = np.random.default_rng(dim + pairs)
    at = [0, 1, -1, 7, 100003] + [int(s * (2 ** e - o)) for e in (20, 30, 31, 32, 40, 45, 50, 52, 53) for s, o in ((1, 1), (-1, 12345))] + [2 ** 53]
    n, H = len(at), 3
    x = torch.from_numpy(rng.standard_normal((n, H, dim)).astype(np.float32)).to(t)
    f = np.float32(10000.0) ** -(np.arange(pairs, dtype=np.float32) / np.float32(pairs))
    f[-1] = 0.75
    if pairs > 2:
        f[1:3] = 37.125, 1e6
    angle = _angles(at, f)[:, None, :]
    X = x.double().numpy()
    one, two = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if interleaved else (slice(0, pairs), slice(pairs, 2 * pairs))
    for scale, run, sign in ((1.3, g.rotary, 1), (-0.7, g.rotary_backward, -1)):
        got = run(x.cuda(), None, torch.tensor(at).cuda(), torch.from_numpy(f).cuda(), interleaved=interleaved, scale=scale)[0].cpu()
        c, s = scale * np.cos(angle), sign * scale * np.sin(angle)
        size = 2.0 ** -20 * abs(scale) * (np.abs(X[..., one]) + np.abs(X[..., two])) + (2.0 ** -25 if dtype == "float16" else 0)
        for part, want in ((one, X[..., one] * c - X[..., two] * s), (two, X[..., one] * s + X[..., two] * c)):
            assert (np.abs(got.double().numpy()[..., part] - want) <= HALF[dtype] * np.abs(want) + size).all(), (scale, np.argwhere(np.abs(got.double().numpy()[..., part] - want) > HALF[dtype] * np.abs(want) + size)[:3])
        assert torch.equal(got[..., 2 * pairs:], x[..., 2 * pairs:])

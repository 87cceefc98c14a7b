"""Sizes that no launch takes are refused before anything is enqueued, through the C ABI and without a GPU: with a null context, what
is in order ends in GOOM_EINVAL for the context."""
import ctypes as C

import pytest

from test_abi_layer_host import EINVAL, EUNSUP, P, attention, err, lib  # noqa: F401


def norm(**kw):
    from paper_2510_03426_amd.binding import NormShape
    f = dict(items=4, length=1000, channels=64, groups=8, type=16, param_type=16, activation=1, flags=0, eps=1e-5)
    f.update(kw)
    return NormShape(**f)


@pytest.mark.parametrize("kw", [dict(items=1 << 24, length=600, channels=8), dict(items=1 << 30, length=3, channels=2048, groups=1), dict(items=1 << 25, length=2100, channels=1, groups=1)])
def test_group_norm(lib, kw):  # noqa: F811
    """Long groups: a workgroup an item at least, of 192 threads or more."""
    many = norm(**kw)
    few = norm(**{**kw, "items": 1 << 20})
    forward = lambda s: lib.goom_group_norm(None, C.byref(s), P, None, None, P, None, None, P, 1 << 60)  # noqa: E731
    back = lambda s: lib.goom_group_norm_backward(None, C.byref(s), *[P] * 9, P, 1 << 60)  # noqa: E731
    for call in (forward, back):
        assert call(many) == EUNSUP and "too many" in err(lib)
        assert call(few) == EINVAL and "context" in err(lib)


def test_linear_attention_step(lib):  # noqa: F811
    """256 threads for every head of every sequence: fewer than 2^24 of them."""
    step = lambda n, heads: lib.goom_linear_attention_step(None, C.byref(attention(seqs=n, tokens=n, heads=heads, kv_heads=heads)), *[P] * 7)  # noqa: E731
    for heads in (1, 16):
        assert step((1 << 24) // heads, heads) == EUNSUP and "too many" in err(lib)
        assert step((1 << 24) // heads - 1, heads) == EINVAL and "context" in err(lib)


def test_scales_that_no_float_holds(lib):  # noqa: F811
    """They would be infinities, or an eps of zero, on the device."""
    for scale in (1e39, -1e300):
        assert lib.goom_linear_attention(None, C.byref(attention(scale=scale)), P, P, P, P, None, None, P, None, P, 1 << 40) == EINVAL and "scale" in err(lib)
        assert lib.goom_embedding(None, P, P, P, 5, 10, 8, 16, scale) == EINVAL and "scale" in err(lib)
        assert lib.goom_embedding_backward(None, P, P, P, 5, 10, 8, 16, 17, scale, P, 1 << 40) == EINVAL and "scale" in err(lib)
    for eps in (1e39, 1e-60):
        assert lib.goom_group_norm(None, C.byref(norm(eps=eps)), P, None, None, P, None, None, P, 1 << 40) == EINVAL and "eps" in err(lib)
    assert lib.goom_group_norm(None, C.byref(norm(eps=0.0)), P, None, None, P, None, None, P, 1 << 40) == EINVAL and "context" in err(lib)

"""What the layer operators refuse, and their workspace queries, through the C ABI.  Arguments are checked before the device is
touched, so no GPU is needed."""
import ctypes as C

import pytest

EINVAL, EUNSUP, EWS = -1, -2, -3
P = C.c_void_p(0x1000)  # a plausible, aligned address that is never read


@pytest.fixture(scope="module")
def lib():
    from paper_2510_03426_amd import binding, build
    build.build()
    return binding.load_library()


def err(lib):
    return lib.goom_last_error(None).decode()


def attention(**kw):
    from paper_2510_03426_amd.binding import AttentionShape
    f = dict(seqs=2, tokens=256, heads=4, kv_heads=2, dk=32, dv=64, type=17, flags=0, scale=1.0)
    f.update(kw)
    return AttentionShape(**f)


def forward(lib, shape, q=P, k=P, v=P, ld=P, off=None, state=None, o=P, last=None, ws=P, wsn=1 << 40):
    return lib.goom_linear_attention(None, C.byref(shape) if shape is not None else None, q, k, v, ld, off, state, o, last, ws, wsn)


def test_linear_attention_refuses(lib):
    assert forward(lib, attention()) == EINVAL and "context" in err(lib)  # everything else is in order
    for kw, word in ((dict(type=0), "type"), (dict(type=19), "type"), (dict(flags=1), "flags"), (dict(seqs=-1), "negative"), (dict(tokens=-1), "negative"),
                     (dict(kv_heads=3), "divide"), (dict(heads=0), "divide"), (dict(kv_heads=0), "divide"), (dict(dk=0), "positive"), (dict(dv=-4), "positive"),
                     (dict(scale=float("nan")), "finite"), (dict(scale=float("inf")), "finite"), (dict(seqs=0), "sequence"), (dict(seqs=3), "tokens / seqs"),
                     (dict(q_token=16, q_head=32), "strides"), (dict(k_token=64, k_head=0), "strides"), (dict(v_head=-64), "strides")):
        assert forward(lib, attention(**kw)) == EINVAL and word in err(lib), kw
    for kw in (dict(dk=129), dict(dv=200), dict(q_token=1 << 23, q_head=32), dict(seqs=1 << 40, tokens=1 << 40), dict(tokens=1 << 50)):
        assert forward(lib, attention(**kw)) == EUNSUP, kw
    assert forward(lib, None) == EINVAL and "null" in err(lib)
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(ld=None), dict(o=None)):
        assert forward(lib, attention(), **kw) == EINVAL and "null" in err(lib), kw
    odd = C.c_void_p(0x1001)
    for kw in (dict(q=odd), dict(o=odd), dict(ld=C.c_void_p(0x1002)), dict(state=C.c_void_p(0x1002)), dict(off=C.c_void_p(0x1004)), dict(last=C.c_void_p(0x1002))):
        assert forward(lib, attention(), **kw) == EINVAL and "aligned" in err(lib), kw
    few = attention(tokens=8192)  # few long sequences are cut into segments, whose states need room
    need = lib.goom_linear_attention_workspace_bytes(C.byref(few), 0)
    assert need > 0
    assert forward(lib, few, ws=None, wsn=0) == EWS and forward(lib, few, wsn=need - 1) == EWS
    assert forward(lib, few, ws=C.c_void_p(0x1010), wsn=need) == EINVAL and "256" in err(lib)
    # with offsets the tokens need not divide; nothing to do is no error as such
    assert forward(lib, attention(seqs=3), off=P) == EINVAL and "context" in err(lib)
    assert forward(lib, attention(seqs=0, tokens=0)) == EINVAL and "context" in err(lib)


def test_linear_attention_step_and_backward_refuse(lib):
    step = lambda shape, **kw: lib.goom_linear_attention_step(None, C.byref(shape), *[kw.get(x, P) for x in ("q", "k", "v", "ld", "state", "o", "next")])  # noqa: E731
    one = attention(seqs=8, tokens=8)
    assert step(one) == EINVAL and "context" in err(lib)
    assert step(attention(seqs=8, tokens=16)) == EINVAL and "one token" in err(lib)
    assert step(one, next=None) == EINVAL and "null" in err(lib)
    assert step(one, o=C.c_void_p(0x1001)) == EINVAL and "aligned" in err(lib)
    assert step(attention(seqs=8, tokens=8, dk=256)) == EUNSUP
    names = ("q", "k", "v", "ld", "off", "state", "go", "gf", "gq", "gk", "gv", "gs")

    def back(shape, ws=P, wsn=1 << 40, **kw):
        return lib.goom_linear_attention_backward(None, C.byref(shape), *[kw.get(x, None if x in ("off", "state", "gf", "gs") else P) for x in names], ws, wsn)
    assert back(attention()) == EINVAL and "context" in err(lib)
    for x in ("q", "go", "gq", "gk", "gv", "ld"):
        assert back(attention(), **{x: None}) == EINVAL and "null" in err(lib), x
    assert back(attention(), gk=C.c_void_p(0x1001)) == EINVAL and "aligned" in err(lib)
    need = lib.goom_linear_attention_backward_workspace_bytes(C.byref(attention()), 0)
    assert need >= 4 * 256 * 4 * (32 + 64)  # floats of 256 tokens' 4 heads, to be summed where they share keys and values
    assert back(attention(), wsn=need - 1) == EWS
    assert lib.goom_linear_attention_workspace_bytes(C.byref(attention(dk=0)), 0) == 0


def test_group_norm_refuses(lib):
    from paper_2510_03426_amd.binding import NormShape

    def shape(**kw):
        f = dict(items=4, length=1000, channels=64, groups=8, type=16, param_type=16, activation=1, flags=0, eps=1e-5)
        f.update(kw)
        return NormShape(**f)

    def call(s, x=P, w=None, b=None, y=P, mean=None, rstd=None, ws=P, wsn=1 << 40):
        return lib.goom_group_norm(None, C.byref(s), x, w, b, y, mean, rstd, ws, wsn)
    assert call(shape()) == EINVAL and "context" in err(lib)
    for kw, word in ((dict(type=1), "type"), (dict(param_type=0), "type"), (dict(flags=2), "flags"), (dict(items=-1), "items"), (dict(length=0), "length"),
                     (dict(channels=0), "channels"), (dict(groups=0), "groups"), (dict(groups=7), "groups"), (dict(activation=3), "activation"), (dict(activation=-1), "activation"),
                     (dict(eps=-1e-9), "eps"), (dict(eps=float("nan")), "eps")):
        assert call(shape(**kw)) == EINVAL and word in err(lib), kw
    assert call(shape(channels=1 << 21, groups=1)) == EUNSUP
    assert call(shape(), x=None) == EINVAL and call(shape(), y=None) == EINVAL
    assert call(shape(), x=C.c_void_p(0x1002)) == EINVAL and "aligned" in err(lib)
    assert call(shape(), mean=C.c_void_p(0x1002)) == EINVAL
    need = lib.goom_group_norm_workspace_bytes(C.byref(shape()))
    assert need > 0 and call(shape(), wsn=need - 1) == EWS
    assert lib.goom_group_norm_workspace_bytes(C.byref(shape(length=1))) == 0
    back = lambda s, ws=P, wsn=1 << 40, **kw: lib.goom_group_norm_backward(  # noqa: E731
        None, C.byref(s), *[kw.get(x, P) for x in ("x", "gy", "mean", "rstd", "w", "b", "gx", "gw", "gb")], ws, wsn)
    assert back(shape()) == EINVAL and "context" in err(lib)
    for x in ("x", "gy", "mean", "rstd", "gx"):
        assert back(shape(), **{x: None}) == EINVAL and "null" in err(lib), x
    need = lib.goom_group_norm_backward_workspace_bytes(C.byref(shape()))
    assert need > 0 and back(shape(), wsn=need - 1) == EWS


def test_embedding_refuses(lib):
    call = lambda table=P, tokens=P, rows=P, n=5, vocab=10, width=8, type=16, scale=1.0: lib.goom_embedding(None, table, tokens, rows, n, vocab, width, type, scale)  # noqa: E731
    assert call() == EINVAL and "context" in err(lib)
    for kw, word in ((dict(type=0), "type"), (dict(n=-1), "n must"), (dict(vocab=0), "vocab"), (dict(width=0), "width"), (dict(scale=float("inf")), "finite"), (dict(table=None), "null"),
                     (dict(tokens=None), "null"), (dict(rows=None), "null"), (dict(tokens=C.c_void_p(0x1004)), "aligned"), (dict(table=C.c_void_p(0x1001)), "aligned")):
        assert call(**kw) == EINVAL and word in err(lib), kw
    assert call(n=1 << 31) == EUNSUP and call(vocab=1 << 31) == EUNSUP
    back = lambda tokens=P, grad=P, out=P, n=5, vocab=10, width=8, type=16, ttype=17, scale=1.0, ws=P, wsn=1 << 40: lib.goom_embedding_backward(  # noqa: E731
        None, tokens, grad, out, n, vocab, width, type, ttype, scale, ws, wsn)
    assert back() == EINVAL and "context" in err(lib)
    for kw, word in ((dict(type=0), "type"), (dict(ttype=3), "type"), (dict(grad=None), "null"), (dict(out=None), "null"), (dict(out=C.c_void_p(0x1001)), "aligned")):
        assert back(**kw) == EINVAL and word in err(lib), kw
    need = lib.goom_embedding_backward_workspace_bytes(5, 10, 8)
    assert need > 0 and back(wsn=need - 1) == EWS and back(ws=None) == EWS
    assert lib.goom_embedding_backward_workspace_bytes(-1, 10, 8) == 0

"""What the gated delta rule, rotary positions and block norms refuse, and their workspace queries, through the C ABI.  Arguments are checked
before the device is touched, so no GPU is needed: with a null context, what is in order ends in GOOM_EINVAL for the context."""
import ctypes as C

import pytest

from test_abi_layer_host import EINVAL, EUNSUP, EWS, P, err, lib  # noqa: F401

ODD, HALF = C.c_void_p(0x1001), C.c_void_p(0x1002)


def delta(**kw):
    from paper_2510_03426_amd.binding import DeltaShape
    f = dict(seqs=2, tokens=256, heads=4, qk_heads=2, dk=32, dv=64, type=17, flags=0, scale=1.0)
    f.update(kw)
    return DeltaShape(**f)


def forward(lib, shape, ws=P, wsn=1 << 60, **kw):  # noqa: F811
    names = ("q", "k", "v", "ld", "beta", "off", "state", "o", "last")
    return lib.goom_gated_delta(None, C.byref(shape) if shape is not None else None, *[kw.get(x, None if x in ("off", "state", "last") else P) for x in names], ws, wsn)


def test_gated_delta_refuses(lib):  # noqa: F811
    assert forward(lib, delta()) == EINVAL and "context" in err(lib)
    for kw, word in ((dict(type=0), "type"), (dict(flags=1), "flags"), (dict(seqs=-1), "negative"), (dict(tokens=-1), "negative"), (dict(qk_heads=3), "divide"),
                     (dict(heads=0), "divide"), (dict(qk_heads=0), "divide"), (dict(dk=0), "positive"), (dict(dv=-4), "positive"), (dict(scale=float("nan")), "finite"),
                     (dict(scale=1e39), "finite"), (dict(seqs=0), "sequence"), (dict(seqs=3), "tokens / seqs"), (dict(q_token=16, q_head=32), "strides"),
                     (dict(k_token=64, k_head=0), "strides"), (dict(v_head=-64), "strides")):
        assert forward(lib, delta(**kw)) == EINVAL and word in err(lib), kw
    for kw in (dict(dk=129), dict(dv=200), dict(q_token=1 << 23, q_head=32), dict(seqs=1 << 40, tokens=1 << 40), dict(tokens=1 << 50)):
        assert forward(lib, delta(**kw)) == EUNSUP, kw
    assert forward(lib, None) == EINVAL and "null" in err(lib)
    for x in ("q", "k", "v", "ld", "beta", "o"):
        assert forward(lib, delta(), **{x: None}) == EINVAL and "null" in err(lib), x
    for kw in (dict(q=ODD), dict(o=ODD), dict(ld=HALF), dict(beta=HALF), dict(state=HALF), dict(last=HALF), dict(off=C.c_void_p(0x1004))):
        assert forward(lib, delta(), **kw) == EINVAL and "aligned" in err(lib), kw
    need = lib.goom_gated_delta_workspace_bytes(C.byref(delta()), 0)
    assert need >= 256 // 64 * 4 * 12288  # a chunk's matrix for every head
    assert forward(lib, delta(), wsn=need - 1) == EWS and forward(lib, delta(), ws=None) == EWS
    assert forward(lib, delta(), ws=C.c_void_p(0x1010), wsn=need) == EINVAL and "256" in err(lib)
    assert forward(lib, delta(seqs=3), off=P) == EINVAL and "context" in err(lib)
    assert forward(lib, delta(seqs=0, tokens=0)) == EINVAL and "context" in err(lib)
    assert lib.goom_gated_delta_workspace_bytes(C.byref(delta(dk=0)), 0) == 0
    # few long sequences are cut into segments, whose maps need room too
    few, many = (lib.goom_gated_delta_workspace_bytes(C.byref(delta(seqs=s, tokens=65536, heads=1, qk_heads=1)), 0) for s in (1, 256))
    assert few > many > 0


def test_gated_delta_step_and_backward_refuse(lib):  # noqa: F811
    step = lambda shape, **kw: lib.goom_gated_delta_step(None, C.byref(shape), *[kw.get(x, P) for x in ("q", "k", "v", "ld", "beta", "state", "o", "next")])  # noqa: E731
    one = delta(seqs=8, tokens=8)
    assert step(one) == EINVAL and "context" in err(lib) and step(one, state=None) == EINVAL and "context" in err(lib)
    assert step(delta(seqs=8, tokens=16)) == EINVAL and "one token" in err(lib)
    for x in ("q", "beta", "next"):
        assert step(one, **{x: None}) == EINVAL and "null" in err(lib)
    assert step(one, o=ODD) == EINVAL and "aligned" in err(lib)
    assert step(delta(seqs=1 << 22, tokens=1 << 22)) == EUNSUP and "too many" in err(lib)
    names = ("q", "k", "v", "ld", "beta", "off", "state", "go", "gf", "gq", "gk", "gv", "ga", "gb", "gs")

    def back(shape, ws=P, wsn=1 << 60, **kw):
        return lib.goom_gated_delta_backward(None, C.byref(shape), *[kw.get(x, None if x in ("off", "state", "gf", "gs") else P) for x in names], ws, wsn)
    assert back(delta()) == EINVAL and "context" in err(lib)
    for x in ("q", "beta", "go", "gq", "gk", "gv", "ga", "gb"):
        assert back(delta(), **{x: None}) == EINVAL and "null" in err(lib), x
    for kw in (dict(gk=ODD), dict(ga=HALF), dict(gs=HALF), dict(gf=HALF)):
        assert back(delta(), **kw) == EINVAL and "aligned" in err(lib), kw
    need = lib.goom_gated_delta_backward_workspace_bytes(C.byref(delta()), 0)
    assert need >= 2 * (256 // 64) * 4 * (32 * 64 + 64 * 64) * 4  # states, adjoints and rows of every chunk
    assert back(delta(), wsn=need - 1) == EWS


def test_rotary_refuses(lib):  # noqa: F811
    from paper_2510_03426_amd.binding import RotaryShape

    def call(x=None, **kw):
        f = dict(tokens=7, heads=4, kv_heads=2, dim=64, pairs=32, type=16, flags=0, scale=1.0)
        given = {k: kw.pop(k) for k in ("q", "k", "pos", "freq", "oq", "ok") if k in kw}
        f.update(kw)
        return lib.goom_rotary(None, C.byref(RotaryShape(**f)), *[given.get(k, P) for k in ("q", "k", "pos", "freq", "oq", "ok")])
    assert call() == EINVAL and "context" in err(lib)
    assert call(kv_heads=0, k=None, ok=None) == EINVAL and "context" in err(lib)
    for kw, word in ((dict(type=1), "type"), (dict(flags=4), "flags"), (dict(tokens=-1), "negative"), (dict(heads=0), "heads"), (dict(kv_heads=-1), "heads"), (dict(pairs=0), "pairs"),
                     (dict(pairs=33), "pairs"), (dict(dim=1, pairs=1), "pairs"), (dict(scale=float("inf")), "finite"), (dict(q_token=10, q_head=64), "strides"), (dict(q=None), "null"),
                     (dict(k=None), "null"), (dict(pos=None), "null"), (dict(freq=None), "null"), (dict(ok=None), "null"), (dict(pos=C.c_void_p(0x1004)), "aligned"), (dict(oq=HALF), "aligned")):
        assert call(**kw) == EINVAL and word in err(lib), kw
    assert call(heads=1 << 21) == EUNSUP and call(tokens=1 << 38) == EUNSUP


@pytest.mark.parametrize("before", [False, True])
def test_block_norm_refuses(lib, before):  # noqa: F811
    from paper_2510_03426_amd.binding import BlockNormShape

    def shape(**kw):
        f = dict(tokens=9, channels=64, groups=4, type=17, param_type=16, activation=1, flags=1, eps=1e-5)
        f.update(kw)
        return BlockNormShape(**f)

    names = ("x", "gate", "res", "w", "b", "s") + (("h",) if before else ()) + ("y", "mean", "rstd")
    fn = lib.goom_norm_before if before else lib.goom_norm_after
    call = lambda sh, **kw: fn(None, C.byref(sh) if sh is not None else None, *[kw.get(x, P) for x in names])  # noqa: E731
    assert call(shape()) == EINVAL and "context" in err(lib)
    assert call(shape(), **{x: None for x in names if x not in ("x", "y")}) == EINVAL and "context" in err(lib)
    assert call(None) == EINVAL and "null" in err(lib)
    for kw, word in ((dict(type=1), "type"), (dict(param_type=0), "type"), (dict(flags=2), "flags"), (dict(tokens=-1), "tokens"), (dict(channels=0), "channels"), (dict(groups=0), "groups"),
                     (dict(groups=7), "groups"), (dict(activation=3), "activation"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(eps=1e-60), "eps")):
        assert call(shape(**kw)) == EINVAL and word in err(lib), kw
    assert call(shape(channels=16385, groups=1)) == EUNSUP and call(shape(tokens=1 << 40)) == EUNSUP
    for x in ("x", "y"):
        assert call(shape(), **{x: None}) == EINVAL and "null" in err(lib)
    for kw in (dict(x=ODD), dict(gate=ODD), dict(w=HALF), dict(mean=HALF)):
        assert call(shape(), **kw) == EINVAL and "aligned" in err(lib), kw
    names = ("x", "gate", "h", "gy", "gh", "mean", "rstd", "w", "s", "gres", "gx", "ggate", "gw", "gb", "gs") if before else \
        ("x", "gate", "gy", "mean", "rstd", "w", "b", "s", "gx", "ggate", "gw", "gb", "gs")
    fb = lib.goom_norm_before_backward if before else lib.goom_norm_after_backward
    back = lambda sh, ws=P, wsn=1 << 40, **kw: fb(None, C.byref(sh), *[kw.get(x, P) for x in names], ws, wsn)  # noqa: E731
    assert back(shape()) == EINVAL and "context" in err(lib)
    for x in ("gy", "mean", "rstd", "ggate") + (("h", "gres", "gx", "x") if before else ("x", "gx")):
        assert back(shape(), **{x: None}) == EINVAL and "null" in err(lib), x
    assert back(shape(flags=0), mean=None) == EINVAL and "context" in err(lib)
    need = lib.goom_block_norm_backward_workspace_bytes(C.byref(shape()))
    assert need >= 3 * 64 * 4 and back(shape(), wsn=need - 1) == EWS and back(shape(), ws=None) == EWS
    none = {x: None for x in ("gw", "gb", "gs")}
    assert back(shape(), ws=None, **none) == EINVAL and "context" in err(lib)  # without parameters' gradients no workspace
    if before:  # x and its gradient stand apart from the stream only behind a gate or a scale
        alone = dict(gate=None, s=None, x=None, gx=None, ggate=None, gs=None)
        assert back(shape(), **alone) == EINVAL and "context" in err(lib)
        assert back(shape(), **{**alone, "gs": P, "x": P}) == EINVAL and "scale" in err(lib)

"""What the gated delta rule's workspace queries answer where sequences are empty, through the C ABI; no GPU is needed."""
import ctypes as C

import pytest

from test_abi_block_host import delta
from test_abi_layer_host import EINVAL, P, err, lib  # noqa: F401


@pytest.mark.parametrize("seqs,heads", [(1, 1), (3, 4), (17, 16), (300, 1), (300, 16), (4096, 16), (5000, 16)])
@pytest.mark.parametrize("packed", [0, 1])
def test_empty_sequences_need_no_room(lib, seqs, heads, packed):  # noqa: F811
    """Without tokens no kernel writes the workspace, so none may read it: the queries ask for nothing, and the calls take none."""
    shape = delta(seqs=seqs, tokens=0, heads=heads, qk_heads=heads)
    assert lib.goom_gated_delta_workspace_bytes(C.byref(shape), packed) == 0
    assert lib.goom_gated_delta_backward_workspace_bytes(C.byref(shape), packed) == 0
    off = P if packed else None
    none = [None] * 5
    assert lib.goom_gated_delta(None, C.byref(shape), *none, off, P, None, P, None, 0) == EINVAL and "context" in err(lib)
    assert lib.goom_gated_delta_backward(None, C.byref(shape), *none, off, P, None, P, *none, P, None, 0) == EINVAL and "context" in err(lib)


def test_one_token_among_empty_sequences(lib):  # noqa: F811
    """The ordering is there again with the first token."""
    for n in (300, 4096):
        one, none = (lib.goom_gated_delta_workspace_bytes(C.byref(delta(seqs=n, tokens=t, heads=16, qk_heads=16)), 1) for t in (1, 0))
        assert none == 0 and one >= 4 * n


@pytest.mark.parametrize("kind", [16, 17, 18])  # float, bfloat16, half
@pytest.mark.parametrize("seqs,tokens,heads,qk_heads,dk,dv,packed", [(8, 8 * 4096, 16, 16, 128, 128, 0), (4096, 4096, 16, 16, 128, 128, 1), (300, 5000, 16, 4, 50, 72, 1), (700, 700 * 33, 1, 1, 20, 20, 1)])
def test_sizes_are_what_the_header_says(lib, kind, seqs, tokens, heads, qk_heads, dk, dv, packed):  # noqa: F811
    """Records of chunks, two states and two chunks of rows, shared heads' sums; each part ends at a multiple of 256 bytes.  (No segments: 256 walks and more.)"""
    ch = 64 if kind == 17 else 32
    chunks = tokens // ch + seqs if packed else seqs * -(-(tokens // seqs) // ch)
    rows, cols = next(x for x in (32, 64, 128) if x >= dk), 32 if dv <= 32 else -(-dv // 64) * 64
    record = 13632 if ch == 64 else 4800
    shape = delta(seqs=seqs, tokens=tokens, heads=heads, qk_heads=qk_heads, dk=dk, dv=dv, type=kind)
    forward = lib.goom_gated_delta_workspace_bytes(C.byref(shape), packed)
    backward = lib.goom_gated_delta_backward_workspace_bytes(C.byref(shape), packed)
    order = 4 * seqs if packed else 0
    want = chunks * heads * record
    assert want <= forward <= want + order + 3 * 256
    want += chunks * heads * 2 * 4 * cols * (rows + ch) + (8 * dk * tokens * heads if heads != qk_heads else 0)
    assert want <= backward <= want + order + 9 * 256

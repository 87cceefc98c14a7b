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

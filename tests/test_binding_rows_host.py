"""Which tensors the binding passes on as rows of tokens and heads, without a GPU: only sizes and strides matter, so a stand-in has them."""
import pytest
import torch

from paper_2510_03426_amd.binding import _rows


class OnDevice:
    """A tensor's shape and strides, said to be on the device."""
    is_cuda = True

    def __init__(self, t):
        self.t, self.shape = t, t.shape

    def __getattr__(self, name):
        return getattr(self.t, name)


def rows(t):
    return _rows(OnDevice(t), "k")[1:]


def test_slices_of_a_projection():
    x = torch.empty(2, 7, 5 + 3 * 4)
    assert rows(x[..., 5:].unflatten(-1, (3, 4))) == (17, 4)
    assert rows(torch.empty(2, 7, 3, 4)) == (0, 0)
    assert rows(torch.empty(2, 7, 3, 8)[..., :4]) == (24, 8)
    assert rows(torch.empty(7, 3, 4)[:, :1]) == (12, 4)
    assert rows(torch.empty(1, 3, 8)[..., 4:]) == (24, 8)
    assert rows(torch.empty(1, 3, 7, 4).transpose(1, 2)) == (4, 28)
    assert rows(torch.empty(1, 5, 4).transpose(0, 1)[2:3]) == (0, 0)  # one row


@pytest.mark.parametrize("shape,base", [((2, 7, 3, 4), (4,)), ((7, 3, 4), (4,)), ((7, 3, 4), (1, 1, 4)), ((1, 3, 4), (1, 1, 4)), ((5, 1, 3, 4), (1, 1, 1, 4)), ((7, 1, 4), (1, 1, 4)),
                                        ((2, 7, 3, 4), (2, 7, 1, 4)), ((2, 7, 3, 4), (1, 1, 3, 4)), ((2, 7, 3, 4), (2, 1, 3, 4)), ((2, 7, 1, 4), (1, 7, 1, 4))])
def test_expanded_axes_are_refused(shape, base):
    """Rows that share memory: strides of 0 would be read as those of contiguous rows, beyond the storage."""
    with pytest.raises(ValueError, match="k: "):
        rows(torch.empty(base).expand(shape))


def test_overlapping_rows_are_refused():
    with pytest.raises(ValueError, match="k: "):
        rows(torch.empty(40).as_strided((7, 2, 4), (3, 4, 1)))
    with pytest.raises(ValueError, match="k: "):
        rows(torch.empty(60).as_strided((7, 2, 4), (8, 3, 1)))
    with pytest.raises(ValueError, match="k: "):
        rows(torch.empty(7, 3, 8)[..., ::2])
    with pytest.raises(ValueError, match="k: "):
        rows(torch.empty(2, 3, 7, 4).transpose(1, 2))

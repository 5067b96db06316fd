"""Which strides the binding takes for rows of heads (no GPU: only addresses and strides are formed)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2607_17154_amd import ordermoe as om  # noqa: E402


class _OnDevice(torch.Tensor):
    is_cuda = True


def _rows(t, *shape):
    return om._rows(t.as_subclass(_OnDevice), torch.float32, *shape)


def test_tokens_may_lie_apart():
    x = torch.zeros((5, 6, 64))
    assert _rows(x, 5, 6, 64) == (x.data_ptr(), 384)
    assert _rows(x[:, 4:], 5, 2, 64) == (x.data_ptr() + 4 * 64 * 4, 384)
    assert _rows(x[:1, 1:3], 1, 2, 64)[1] == 128               # one token: the stride says nothing
    assert _rows(x[:0], 0, 6, 64)[1] == 384


def test_the_stride_of_a_single_head_says_nothing():
    x = torch.zeros((1, 5, 64))                                 # one head's tokens, side by side
    t = x.transpose(0, 1)
    assert t.stride(1) == 320 and t.is_contiguous()
    assert _rows(t, 5, 1, 64) == (x.data_ptr(), 64)


@pytest.mark.parametrize("make", [lambda: torch.zeros((5, 64, 2)).transpose(1, 2), lambda: torch.zeros((2, 5, 64)).transpose(0, 1),
                                  lambda: torch.zeros((5, 2, 128))[..., :64], lambda: torch.zeros((5, 2, 128))[..., ::2]])
def test_heads_apart_are_refused(make):
    with pytest.raises(ValueError):
        _rows(make(), 5, 2, 64)


def test_other_types_and_shapes_are_refused():
    for t, shape in ((torch.zeros((5, 2, 64)), (4, 2, 64)), (torch.zeros((5, 2, 64), dtype=torch.bfloat16), (5, 2, 64)),
                     (torch.zeros((10, 64)), (5, 2, 64))):
        with pytest.raises(ValueError):
            _rows(t, *shape)
    with pytest.raises(ValueError):
        om._rows(torch.zeros((5, 2, 64)), torch.float32, 5, 2, 64)

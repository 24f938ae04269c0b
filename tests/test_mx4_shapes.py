"""mx4: what becomes of a tensor's strides before a call, without a GPU."""
import pytest
import torch

import paper_2508_00806_amd as adacc
from paper_2508_00806_amd import mx4

SMALL = torch.zeros(4, dtype=torch.uint8)


def accepted(x):
    """The library takes the strides: what it refuses is the blob."""
    with pytest.raises(adacc.AdaccError) as e:
        adacc.mx4_compress(x, SMALL, stream=0)
    return e.value.code == adacc.ESIZE


@pytest.mark.parametrize("x", [torch.ones(1, 1).expand(300, 1), torch.ones(()).expand(300, 1), torch.ones(3, 1, 1).expand(3, 100, 1),
                               torch.ones(()).expand(3, 100, 1), torch.ones(5, 1).t().expand(300, 5)[:, 2:3], torch.ones(4).expand(300, 4),
                               torch.ones(300, 6)[:, :1], torch.ones(1, 300).t(), torch.ones(300, 1)],
                         ids=lambda x: f"{tuple(x.shape)}-{x.stride()}")
def test_rows_that_share_memory_become_rows_of_their_own(x):
    """A broadcast column's rows are no distance apart, which the library refuses."""
    flat = mx4._flat(x)
    assert accepted(flat) and torch.equal(flat, x.reshape(300, -1))


@pytest.mark.parametrize("x", [torch.ones(2, 1, 1).expand(2, 150, 1), torch.ones(()).expand(2, 150, 1), torch.ones(1, 150, 1).expand(2, 150, 1),
                               torch.ones(1, 1, 7).expand(2, 150, 7), torch.ones(2, 150, 9)[:, :, 3:4]],
                         ids=lambda x: f"{tuple(x.shape)}-{x.stride()}")
def test_stacks_of_such_rows(x):
    stack = mx4._stack(x)
    assert accepted(stack) and torch.equal(stack, x)


def test_rows_that_lie_well_are_not_copied():
    for x in (torch.zeros(30, 6)[:, 1:4], torch.zeros(30, 6)[:, 2:3], torch.zeros(1, 9).expand(1, 9), torch.zeros(6, 30).t()[:, :1]):
        assert mx4._flat(x).data_ptr() == x.data_ptr()
    x = torch.zeros(2, 30, 8)[:, ::2, :5]
    assert mx4._stack(x).data_ptr() == x.data_ptr()


@pytest.mark.parametrize("shape", [(2, 3, 0), (0, 3, 0), (4, 0), (2, 0, 5), (1, 1, 1, 0), (0,), (7,)])
def test_empty_dimensions_are_counted(shape):
    flat = mx4._flat(torch.zeros(shape))
    rows = 1
    for d in shape[:-1]:
        rows *= d
    assert flat.shape == (rows, shape[-1])


@pytest.mark.parametrize("shape", [(3, 4, 0), (0, 4, 0), (3, 0, 8), (3, 0)])
def test_an_empty_stack_is_restored(shape, monkeypatch):
    """By the library itself, which touches nothing."""
    monkeypatch.setattr(mx4, "_stream_of", lambda t: 0)
    monkeypatch.setattr(mx4, "_on_gpu", lambda t: None)
    m = mx4.Mx4Matrix(torch.zeros(0, dtype=torch.uint8), shape)
    assert m.restore(torch.float32).shape == shape

"""mx4 layers whose matrices have one column, or none."""
import numpy as np
import pytest
import torch

from mx4_reference import assert_product, f64, matrix, rounded
from paper_2508_00806_amd import mx4

pytestmark = pytest.mark.gpu


def sums(k):
    return 2 * (-(-k // 64)) + 10


@pytest.mark.parametrize("lead", [(40,), (5, 8), (300,)])
def test_one_column_of_results_and_the_gradient_of_their_sum(lead):
    """The gradient of a sum is one value for all rows, no distance apart."""
    print(f"[mx4 shapes] one column {lead}", flush=True)
    k, m = 96, int(np.prod(lead))
    x, w = matrix(m, k, torch.bfloat16, 1, 0.5), matrix(1, k, torch.bfloat16, 2, 0.5)
    xg, wg = x.cuda().view(*lead, k).requires_grad_(), w.cuda().requires_grad_()
    y = mx4.linear(xg, wg, out_dtype=torch.float32)
    y.sum().backward()
    ones = np.ones((m, 1))
    assert_product(y.view(m, 1), rounded(f64(x)), rounded(f64(w)), torch.float32, sums(k))
    assert_product(xg.grad.view(m, k), rounded(ones), rounded(f64(w).T), torch.bfloat16, sums(1))
    assert_product(wg.grad, rounded(ones.T), rounded(f64(x).T), torch.bfloat16, sums(m))


def test_one_broadcast_column_of_rows():
    print("[mx4 shapes] broadcast column", flush=True)
    m, n = 70, 33
    x, w = torch.full((1, 1), 1.5), matrix(n, 1, torch.float32, 3, 0.5)
    wide = x.cuda().expand(m, 1)
    for got in (mx4.linear(wide, w.cuda()), mx4.linear(wide, mx4.compress(w.cuda()))):
        assert_product(got, rounded(f64(x)).repeat(m, 0), rounded(f64(w)), torch.float32, sums(1))
    stack = mx4.compress(x.cuda().expand(2, m, 1))
    assert (stack.restore(torch.float32) == 1.5).all() and stack.shape == (2, m, 1)


@pytest.mark.parametrize("lead,n,k", [((2, 3), 5, 0), ((6,), 5, 0), ((2, 3), 0, 8), ((0, 3), 5, 8), ((2, 0), 0, 0)])
def test_empty_dimensions(lead, n, k):
    """A contraction of length zero gives zeros; gradients have their shapes."""
    print(f"[mx4 shapes] empty {lead} {n} {k}", flush=True)
    x, w = torch.ones(*lead, k, device="cuda", requires_grad=True), torch.ones(n, k, device="cuda", requires_grad=True)
    held = mx4.compress(w.detach())
    assert held.restore(torch.float32).shape == (n, k)
    with torch.no_grad():
        served = mx4.linear(x, held)
    y = mx4.linear(x, w)
    assert served.shape == y.shape == (*lead, n) and torch.equal(served, y.detach())
    if k == 0:
        assert (y == 0).all()
    y.sum().backward()
    assert x.grad.shape == x.shape and w.grad.shape == w.shape and (w.grad == 0).all()


def test_an_empty_stack():
    for shape in ((3, 4, 0), (3, 0, 8), (0, 4, 8)):
        along, across = mx4.compress_both(torch.empty(shape, device="cuda"))
        assert along.restore().shape == shape and across.restore().shape == (shape[0], shape[2], shape[1])


def test_restored_into_a_given_tensor():
    m = mx4.compress(matrix(40, 96, torch.bfloat16, 5).cuda())
    with pytest.raises(ValueError, match="out is on cpu"):
        m.restore(out=torch.zeros(40, 96))
    room = torch.full((40, 100), 7.0, device="cuda")
    assert m.restore(out=room[:, :96]) is not None and torch.equal(room[:, :96], m.restore(torch.float32)) and (room[:, 96:] == 7.0).all()


def test_rows_that_a_gradient_is_wanted_for_are_served_alike():
    x, w = matrix(20, 96, torch.bfloat16, 1).cuda(), mx4.compress(matrix(33, 96, torch.bfloat16, 2).cuda())
    want = mx4.linear(x, w)
    xg = x.clone().requires_grad_()
    y = mx4.linear(xg, w)
    assert torch.equal(y, want)
    with pytest.raises(RuntimeError, match="Mx4Matrix has no gradient"):
        y.sum().backward()
    with torch.no_grad():
        assert torch.equal(mx4.linear(xg, w), want)

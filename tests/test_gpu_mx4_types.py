"""mx4 layers with float16 and float32 rows: gradients whose values stay in float16's range, and experts' rows of few and many."""
import numpy as np
import pytest
import torch

import paper_2508_00806_amd as adacc
from mx4_reference import assert_product, f64, matrix, quantise_groups, rounded, values
from paper_2508_00806_amd import mx4

pytestmark = pytest.mark.gpu
MOST = 60000.0


def sums(k):
    return 2 * (-(-k // 64)) + 10


def check(got, a, b, dtype, k):
    assert got.dtype == dtype
    if dtype == torch.float16:  # (what is compared is in range, or the test shows nothing)
        assert np.abs(a @ b.T).max() < MOST
    assert_product(got, a, b, dtype, sums(k))


def small(rows, cols, dtype, seed):
    """A gradient: 2^-6 of the others' size (a power of two: the codes are the same)."""
    return (matrix(rows, cols, torch.float32, seed, 0.5) * 2.0 ** -6).to(dtype)


@pytest.mark.parametrize("dtype,wtype", [(torch.float16, torch.float16), (torch.float16, torch.float32), (torch.float32, torch.float16)])
@pytest.mark.parametrize("m,n,k", [(1, 30, 40), (77, 130, 264), (1000, 515, 300), (2100, 2048, 520)])
def test_gradients(m, n, k, dtype, wtype):
    print(f"[mx4 types] {m} {n} {k} {dtype} {wtype}", flush=True)
    x, w, dy = matrix(m, k, dtype, 1, 0.5), matrix(n, k, wtype, 2, 0.5), small(m, n, dtype, 3)
    xg, wg = x.cuda().requires_grad_(), w.cuda().requires_grad_()
    y = mx4.linear(xg, wg)
    dx, dw = torch.autograd.grad(y, (xg, wg), dy.cuda())
    check(y, rounded(f64(x)), rounded(f64(w)), dtype, k)
    check(dx, rounded(f64(dy)), rounded(f64(w).T), dtype, n)
    check(dw, rounded(f64(dy).T), rounded(f64(x).T), wtype, m)


@pytest.mark.parametrize("dtype,wtype", [(torch.float16, torch.float16), (torch.float16, torch.float32), (torch.float32, torch.float32)])
@pytest.mark.parametrize("offsets", [[0, 5, 5, 40], [0, 0, 300, 301, 700], [0, 128, 1200], list(range(0, 130, 2))], ids=lambda o: f"{len(o) - 1}groups{o[-1]}rows")
@pytest.mark.parametrize("n,k", [(140, 200), (33, 131)])
def test_experts_gradients(offsets, n, k, dtype, wtype):
    print(f"[mx4 types] experts {offsets[:6]} {n} {k} {dtype} {wtype}", flush=True)
    experts, rows = len(offsets) - 1, offsets[-1] + 3
    x, w, dy = matrix(rows, k, dtype, 1, 0.5), matrix(experts * n, k, wtype, 2, 0.5).view(experts, n, k), small(rows, n, dtype, 3)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    xg, wg = x.cuda().requires_grad_(), w.cuda().requires_grad_()
    y = mx4.experts(xg, off, wg)
    dx, dw = torch.autograd.grad(y, (xg, wg), dy.cuda())
    positions = adacc.mx4_grouped_cols(rows, experts)
    xt, dyt = (values(*quantise_groups(f64(t), offsets, positions)) for t in (x, dy))
    at = 0
    for e in range(experts):
        a, b = offsets[e], offsets[e + 1]
        if a == b:
            assert (dw[e] == 0).all()
            continue
        check(y[a:b], rounded(f64(x[a:b])), rounded(f64(w[e])), dtype, k)
        check(dx[a:b], rounded(f64(dy[a:b])), rounded(f64(w[e]).T), dtype, n)
        check(dw[e], dyt[:, at:at + b - a], xt[:, at:at + b - a], wtype, b - a)
        at += -(-(b - a) // 128) * 128
    assert (y[offsets[-1]:] == 0).all() and (dx[offsets[-1]:] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("groups,n", [(5, 64), (16, 387), (64, 262), (3, 2731)])  # 16, 32, 64 and 64 columns a workgroup
@pytest.mark.parametrize("each,k", [(1, 200), (11, 200), (16, 4096), (1, 77), (20, 200), (100, 136)])
def test_experts_rows(groups, n, each, k, dtype):
    """Few rows compressed on the way (16 and fewer, k a multiple of 8), from the workspace, and many."""
    print(f"[mx4 types] {groups} of {each} rows n={n} k={k} {dtype}", flush=True)
    rows = groups * each
    x, w = matrix(rows, k, dtype, 31), matrix(groups * n, k, torch.bfloat16, 32).view(groups, n, k)
    off = torch.arange(0, rows + 1, each, dtype=torch.int32, device="cuda")
    y = mx4.experts(x.cuda(), off, mx4.compress(w.cuda()), out_dtype=torch.float32)
    for g in {0, groups // 2, groups - 1}:
        part = slice(g * each, (g + 1) * each)
        check(y[part], rounded(f64(x[part])), rounded(f64(w[g])), torch.float32, k)

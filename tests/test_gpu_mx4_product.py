"""Products of microscaled 4-bit matrices against binary64: dense, by groups of rows, and the gradient of the groups' matrices."""
import numpy as np
import pytest
import torch

import paper_2508_00806_amd as adacc
from mx4_reference import TYPES, assert_product, f64, grouped_positions, matrix, quantise, quantise_groups, rounded, values
from paper_2508_00806_amd import mx4

pytestmark = pytest.mark.gpu


def sums(k):
    """binary32 additions that a result can depend on, generously: two for every 64 columns, and the joining of eight partial sums"""
    return 2 * (-(-k // 64)) + 10


def blob_of(x):
    return mx4.compress(x.cuda()).blob


def run(m, n, k, dtype=torch.bfloat16, seed=0, out_pad=0):
    a, b = matrix(m, k, torch.bfloat16, seed), matrix(n, k, torch.bfloat16, seed + 1)
    room = torch.full((m, n + out_pad), 7.0, dtype=dtype, device="cuda")
    adacc.mx4_product(blob_of(a), blob_of(b), k, room[:, :n])
    torch.cuda.synchronize()
    assert (room[:, n:] == 7.0).all()
    if dtype == torch.float16:  # (values beyond its range become infinite)
        want = rounded(f64(a)) @ rounded(f64(b)).T
        keep = np.abs(want) < 60000
        got = f64(room[:, :n])
        assert np.isfinite(got[keep]).all()
        room = room[:, :n].float().cpu()
        room[torch.from_numpy(~keep)] = torch.from_numpy(want).float()[torch.from_numpy(~keep)]
        return assert_product(room, rounded(f64(a)), rounded(f64(b)), torch.float16, sums(k))
    assert_product(room[:, :n], rounded(f64(a)), rounded(f64(b)), dtype, sums(k))


FEW = [(1, 1, 1), (1, 16, 128), (1, 1003, 2040), (2, 33, 4096), (15, 64, 256), (16, 130, 700), (17, 48, 33), (32, 4100, 1000), (33, 515, 129), (64, 200, 2048),
       (50, 9000, 160), (3, 17000, 384), (16, 33000, 31)]
TILES = [(65, 64, 128), (65, 1, 1), (100, 130, 1), (129, 257, 2040), (777, 1003, 520), (128, 128, 4096), (1000, 513, 384), (2048, 1100, 640), (4096, 2050, 256),
         (4097, 4099, 130), (66, 70000, 96)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", FEW + TILES)
def test_products(shape, dtype):
    print(f"[mx4 product] {shape} {dtype}", flush=True)
    run(*shape, dtype=dtype, seed=sum(shape))


@pytest.mark.parametrize("shape", [(5, 30, 300), (100, 30, 300), (300, 515, 200), (2000, 2047, 256)])
@pytest.mark.parametrize("pad", [1, 2, 4])
def test_rows_of_the_result_apart(shape, pad):
    print(f"[mx4 product] {shape} pad={pad}", flush=True)
    run(*shape, seed=9, out_pad=pad)


def test_every_tile_size_is_met():
    """The same product in the kernels of few rows and in tiles of 64, 128 and 256: m decides."""
    k, n = 384, 4096
    b = matrix(n, k, torch.bfloat16, 1)
    for m in (16, 64, 80, 512, 1100, 5000):
        print(f"[mx4 product] m={m}", flush=True)
        a = matrix(m, k, torch.bfloat16, 2)
        out = torch.empty(m, n, device="cuda")
        adacc.mx4_product(blob_of(a), blob_of(b), k, out)
        assert_product(out, rounded(f64(a)), rounded(f64(b)), torch.float32, sums(k))


@pytest.mark.parametrize("m", [3, 64, 300, 4200])
def test_what_is_not_finite_reaches_its_row_and_column_only(m):
    print(f"[mx4 product] not finite, m={m}", flush=True)
    k, n = 300, 4100
    a, b = matrix(m, k, torch.bfloat16, 3), matrix(n, k, torch.bfloat16, 4)
    a[1, 299] = float("inf")
    a[2, 0] = float("nan")
    b[0, 150] = float("-inf")
    b[n - 1, 33] = float("nan")
    out = torch.empty(m, n, device="cuda")
    adacc.mx4_product(blob_of(a), blob_of(b), k, out)
    want = np.zeros((m, n), bool)
    want[[1, 2]] = True
    want[:, [0, n - 1]] = True
    assert np.array_equal(np.isnan(f64(out)), want)
    assert_product(out, rounded(f64(a)), rounded(f64(b)), torch.float32, sums(k))


def test_sizes_of_zero():
    b = mx4.compress(torch.randn(8, 64, device="cuda"))
    assert mx4.linear(torch.empty(0, 64, device="cuda"), b).shape == (0, 8)
    out = torch.full((3, 8), 5.0, device="cuda")
    adacc.mx4_product(torch.empty(0, dtype=torch.uint8, device="cuda"), torch.empty(0, dtype=torch.uint8, device="cuda"), 0, out)
    assert (out == 0).all()
    out = torch.full((300, 8), 5.0, device="cuda")
    adacc.mx4_product(torch.empty(0, dtype=torch.uint8, device="cuda"), torch.empty(0, dtype=torch.uint8, device="cuda"), 0, out)
    assert (out == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(1, 4096, 2048), (7, 1003, 520), (16, 40, 40), (16, 515, 1000), (5, 64, 37), (20, 300, 256), (200, 300, 256), (1500, 2048, 264)])
def test_linear(m, n, k, dtype):
    """Rows that are compressed on the way, and in a workspace; rows that start anywhere."""
    print(f"[mx4 linear] {m} {n} {k} {dtype}", flush=True)
    big, w = matrix(m, k + 5, dtype, 6), matrix(n, k, dtype, 7)
    for x in (big[:, :k].contiguous(), big[:, 3:3 + k]):
        got = mx4.linear(x.cuda() if x.is_contiguous() else big.cuda()[:, 3:3 + k], mx4.compress(w.cuda()), out_dtype=torch.float32)
        assert_product(got, rounded(f64(x)), rounded(f64(w)), torch.float32, sums(k))


def test_linear_by_the_other_rule_and_not_finite():
    k, n = 256, 100
    w = matrix(n, k, torch.bfloat16, 7)
    for m in (4, 90):
        x = matrix(m, k, torch.bfloat16, 6)
        x[2, 40] = float("nan")
        out = torch.empty(m, n, device="cuda")
        need = adacc.mx4_linear_workspace_bytes(m, n, k)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        adacc.mx4_linear(x.cuda(), blob_of(w), out, workspace=ws, scale_rule=adacc.MX4_SCALE_FULLRANGE)
        assert_product(out, rounded(f64(x), 1), rounded(f64(w)), torch.float32, sums(k))
        assert np.isnan(f64(out)[2]).all()


GROUPS = [[0, 1], [0, 0, 1, 1], [0, 3, 3, 20, 64], [0, 40, 41, 41, 300], [0, 130, 259, 259, 1000, 1001], [0, 700, 2400], [0, 0, 0, 0],
          [0, 1500, 3001, 3001, 4500], list(range(0, 201)), [0] * 70 + [5] * 30 + [90], [0, 2, 4, 4, 4, 6, 1030]]


@pytest.mark.parametrize("offsets", GROUPS, ids=lambda o: f"{len(o) - 1}groups{o[-1]}rows")
@pytest.mark.parametrize("n,k", [(64, 128), (131, 300), (515, 96)])
@pytest.mark.parametrize("tail", [0, 7])
def test_rows_by_group(offsets, n, k, tail):
    """Groups of any size, none included; rows of no group give zeros."""
    print(f"[mx4 groups] {offsets[:8]} n={n} k={k} tail={tail}", flush=True)
    groups, rows = len(offsets) - 1, offsets[-1] + tail
    if rows == 0:
        rows = 2
    x, w = matrix(rows, k, torch.bfloat16, 11), matrix(groups * n, k, torch.bfloat16, 12).view(groups, n, k)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    xr = rounded(f64(x))
    wc = w.cuda()
    got = {"few or tiles": mx4.experts(x.cuda(), off, mx4.compress(wc), out_dtype=torch.float32)}
    out = torch.full((rows, n), 5.0, device="cuda")
    adacc.mx4_product(blob_of(x), mx4.compress(wc).blob, k, out, offsets=off)
    got["compressed rows"] = out
    for name, y in got.items():
        for g in range(groups):
            a, b = offsets[g], offsets[g + 1]
            if b > a:
                assert_product(y[a:b], xr[a:b], rounded(f64(w[g])), torch.float32, sums(k))
        assert (y[offsets[-1]:] == 0).all(), name


@pytest.mark.parametrize("groups,n", [(16, 1091), (64, 262), (48, 217), (16, 387), (48, 333), (5, 1003), (3, 2730), (2, 5003), (16, 67), (8, 1030)])
@pytest.mark.parametrize("each", [1, 11, 40, 150])
def test_the_last_rows_of_a_stack_whose_matrices_begin_anywhere(groups, n, each):
    """Matrices of n rows begin between the words of four scale bytes; the last one ends where the block columns do, or shortly before."""
    print(f"[mx4 groups] {groups} of {each} rows n={n}", flush=True)
    k, rows = 200, groups * each
    x, w = matrix(rows, k, torch.bfloat16, 21), matrix(groups * n, k, torch.bfloat16, 22).view(groups, n, k)
    off = torch.arange(0, rows + 1, each, dtype=torch.int32, device="cuda")
    stack = mx4.compress(w.cuda())
    out = torch.full((rows, n), 5.0, device="cuda")
    adacc.mx4_product(blob_of(x), stack.blob, k, out, offsets=off)
    for y in (mx4.experts(x.cuda(), off, stack, out_dtype=torch.float32), out):
        for g in {0, groups // 2, groups - 2, groups - 1}:
            assert_product(y[g * each:(g + 1) * each], rounded(f64(x))[g * each:(g + 1) * each], rounded(f64(w[g])), torch.float32, sums(k))


@pytest.mark.parametrize("offsets", GROUPS, ids=lambda o: f"{len(o) - 1}groups{o[-1]}rows")
@pytest.mark.parametrize("m,n", [(64, 128), (131, 67), (260, 515)])
def test_gradient_of_the_groups(offsets, m, n):
    print(f"[mx4 gradient] {offsets[:8]} m={m} n={n}", flush=True)
    groups, rows = len(offsets) - 1, max(offsets[-1] + 3, 2)
    a, b = matrix(rows, m, torch.bfloat16, 13), matrix(rows, n, torch.float32, 14)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    positions = adacc.mx4_grouped_cols(rows, groups)
    blobs = []
    for x in (a, b):
        blob = adacc.alloc_mx4(x.shape[1], positions)[0].fill_(0xFF)  # what is not written is NaN, if it were read
        adacc.mx4_compress(x.cuda(), None, blob, offsets=off)
        blobs.append(blob)
    out = torch.full((groups, m, n), 5.0, device="cuda")
    adacc.mx4_gradient(*blobs, rows, out, offsets=off)
    av, bv = (values(*quantise_groups(f64(x), offsets, positions)) for x in (a, b))
    first, _ = grouped_positions(offsets)
    for g in range(groups):
        p, size = first[g], offsets[g + 1] - offsets[g]
        if size == 0:
            assert (out[g] == 0).all()
        else:
            assert_product(out[g], av[:, p:p + size], bv[:, p:p + size], torch.float32, sums(size))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,m,n", [(1, 40, 33), (100, 64, 200), (1000, 700, 500), (333, 2048, 2050)])
def test_gradient_without_groups(rows, m, n, dtype):
    print(f"[mx4 gradient] rows={rows} m={m} n={n} {dtype}", flush=True)
    a, b = matrix(rows, m, torch.bfloat16, 15, 0.5), matrix(rows, n, torch.bfloat16, 16, 0.5)
    at, bt = (mx4.compress_both(x.cuda())[1].blob for x in (a, b))
    out = torch.empty(m, n, dtype=dtype, device="cuda")
    adacc.mx4_gradient(at, bt, rows, out)
    av, bv = (values(*quantise(f64(x).T)) for x in (a, b))
    assert_product(out, av, bv, dtype, sums(rows))


def test_the_order_of_a_sum_does_not_change():
    a, b = matrix(300, 5000, torch.bfloat16, 17), matrix(700, 5000, torch.bfloat16, 18)
    for m in (8, 50, 300):
        first = None
        for _ in range(5):
            out = torch.empty(m, 700, device="cuda")
            adacc.mx4_product(blob_of(a[:m]), blob_of(b), 5000, out)
            first = out if first is None else first
            assert torch.equal(out, first)

"""adacc_mx4_compress / adacc_mx4_decompress against the format's definition in 64 bits: every byte of a blob, every value restored."""
import numpy as np
import pytest
import torch

import paper_2508_00806_amd as adacc
from mx4_reference import TYPES, blob_parts, f64, matrix, padded, quantise, quantise_groups, values
from paper_2508_00806_amd import mx4

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (1, 31), (2, 33), (3, 7), (5, 8), (9, 3), (2, 127), (33, 128), (31, 129), (128, 512), (130, 515), (257, 1031), (8, 4100), (700, 12), (300, 254)]


def blobs(x, along=True, across=True, offsets=None, rule=0):
    """Blobs full of 0xA5 before the call"""
    mats = x.shape[0] if x.dim() == 3 else 1
    rows, cols = x.shape[-2:]
    positions = rows if offsets is None else adacc.mx4_grouped_cols(rows, offsets.numel() - 1)
    a = adacc.alloc_mx4(mats * rows, cols)[0].fill_(0xA5) if along else None
    t = adacc.alloc_mx4(mats * cols, positions)[0].fill_(0xA5) if across else None
    adacc.mx4_compress(x, a, t, offsets=offsets, scale_rule=rule)
    torch.cuda.synchronize()
    return a, t


def check_blob(blob, codes, bytes_):
    rows, cols = codes.shape
    got_codes, got_bytes = blob_parts(blob, adacc.mx4_layout_of(rows, cols), rows, cols)
    assert np.array_equal(got_codes, padded(codes, got_codes.shape[1])), "codes differ"
    assert np.array_equal(got_bytes, padded(bytes_, got_bytes.shape[1])), "scale bytes differ"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rule", [0, 1])
@pytest.mark.parametrize("shape", SHAPES)
def test_every_byte(shape, rule, dtype):
    print(f"[mx4] {shape} rule={rule} {dtype}", flush=True)
    x = matrix(*shape, dtype, sum(shape) + rule)
    xc = x.cuda()
    along, across = quantise(f64(x), rule), quantise(f64(x).T, rule)
    for want_a, want_t in ((True, False), (False, True), (True, True)):
        a, t = blobs(xc, want_a, want_t, rule=rule)
        if want_a:
            check_blob(a, *along)
        if want_t:
            check_blob(t, *across)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_that_start_anywhere(dtype):
    print(f"[mx4] strides {dtype}", flush=True)
    big = matrix(70, 333, dtype, 3).cuda()
    for c0, c1, r0, step in ((1, 300, 0, 1), (3, 132, 5, 2), (330, 333, 1, 3), (7, 39, 69, 1)):
        x = big[r0::step, c0:c1]
        a, t = blobs(x)
        check_blob(a, *quantise(f64(x)))
        check_blob(t, *quantise(f64(x).T))


@pytest.mark.parametrize("shape", [(3, 40, 72), (2, 129, 33), (5, 1, 256), (4, 37, 5), (1, 64, 64)])
@pytest.mark.parametrize("apart", [False, True])
def test_stacks(shape, apart):
    print(f"[mx4] stack {shape} apart={apart}", flush=True)
    mats, rows, cols = shape
    x = matrix(mats * (rows + 3), cols, torch.bfloat16, 8).cuda().view(mats, rows + 3, cols)
    x = x[:, :rows] if apart else x[:, :rows].contiguous()
    a, t = blobs(x)
    flat = f64(x).reshape(mats * rows, cols)
    check_blob(a, *quantise(flat))
    parts = [quantise(f64(x[i]).T) for i in range(mats)]
    check_blob(t, np.concatenate([p[0] for p in parts]), np.concatenate([p[1] for p in parts]))


@pytest.mark.parametrize("offsets", [[0, 5], [0, 0, 130, 130, 131, 300], [0, 128, 256, 384], [0, 1, 2, 3, 700], [0, 0, 0], [0, 100, 100, 612, 690]])
@pytest.mark.parametrize("cols", [5, 96, 520])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_groups_are_cut(offsets, cols, dtype):
    """Rows behind the last group are compressed along, and have no place across."""
    print(f"[mx4] groups {offsets} cols={cols} {dtype}", flush=True)
    rows = max(offsets[-1] + 9, 3)
    x = matrix(rows, cols, dtype, 5)
    xc = x.cuda()
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    positions = adacc.mx4_grouped_cols(rows, len(offsets) - 1)
    codes, bytes_ = quantise_groups(f64(x), offsets, positions)
    used = sum(-(-(b - a) // 128) * 128 for a, b in zip(offsets, offsets[1:]))
    for both in (True, False):
        a, t = blobs(xc, both, True, offsets=off)
        if both:
            check_blob(a, *quantise(f64(x)))
        got_codes, got_bytes = blob_parts(t, adacc.mx4_layout_of(cols, positions), cols, positions)
        assert np.array_equal(got_codes[:, :used], codes[:, :used]) and np.array_equal(got_bytes[:, :used // 32], bytes_[:, :used // 32])
        assert (got_codes[:, used:] == np.where(np.arange(positions - used) % 2, 0xA, 0x5)).all(), "written behind the last group"


def special(dtype):
    """Blocks whose values lie on and next to every border between codes, at the ends of the type's range, and without anything finite."""
    info = torch.finfo(dtype)
    rows = []
    grid = [0.0, 0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0, 7.0]
    for scale in (1.0, 2.0 ** 9, 2.0 ** -9, 2.0 ** 12):
        v = torch.tensor(grid, dtype=torch.float64) * scale
        near = torch.tensor(grid).to(dtype).double() * (1 - info.eps) * scale
        rows.append(torch.cat((v, -near)))
        rows.append(torch.cat((-v, v * (1 + info.eps)))[torch.randperm(32, generator=torch.Generator().manual_seed(1))])
    tiny = info.smallest_normal
    rows.append(torch.full((32,), tiny * info.eps, dtype=torch.float64))          # the smallest subnormal number
    rows.append(torch.linspace(-1, 1, 32, dtype=torch.float64) * tiny)            # subnormal numbers
    rows.append(torch.linspace(-1, 1, 32, dtype=torch.float64) * info.max)        # up to the largest
    rows.append(torch.full((32,), info.max, dtype=torch.float64))
    rows.append(torch.zeros(32, dtype=torch.float64))
    rows.append(-torch.zeros(32, dtype=torch.float64))
    one = torch.ones(32, dtype=torch.float64)
    for bad in (float("inf"), float("-inf"), float("nan")):
        for at in (0, 17, 31):
            r = one.clone()
            r[at] = bad
            rows.append(r)
    rows.append(torch.full((32,), float("nan"), dtype=torch.float64))
    rows.append(torch.cat((torch.full((1,), 6.0, dtype=torch.float64), torch.full((31,), 6.0 * 2.0 ** -30, dtype=torch.float64))))
    return torch.stack(rows).to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rule", [0, 1])
def test_values_that_need_care(rule, dtype):
    print(f"[mx4] special values rule={rule} {dtype}", flush=True)
    x = special(dtype)
    wide = torch.cat((x, x.flip(0)), 1)  # two blocks a row
    a, _ = blobs(wide.cuda(), across=False, rule=rule)
    check_blob(a, *quantise(f64(wide), rule))
    tall = wide.t().contiguous()
    a, t = blobs(tall.cuda(), rule=rule)
    check_blob(t, *quantise(f64(wide), rule))
    check_blob(a, *quantise(f64(tall), rule))
    for out in TYPES:
        m = mx4.compress(wide.cuda(), scale_rule=("floor", "fullrange")[rule])
        want = torch.from_numpy(values(*quantise(f64(wide), rule))).float().to(out)
        got = m.restore(out).cpu()
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(1.0), want.nan_to_num(1.0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_restored_values(shape, dtype):
    """All codes and scale bytes, drawn; the rows' neighbours in memory stay as they are."""
    print(f"[mx4] restore {shape} {dtype}", flush=True)
    rows, cols = shape
    g = torch.Generator().manual_seed(rows + cols)
    blob, lay = adacc.alloc_mx4(rows, cols)
    blob.copy_(torch.randint(0, 256, (int(lay.total_bytes),), dtype=torch.uint8, generator=g))
    codes, bytes_ = blob_parts(blob, lay, rows, cols)
    want = torch.from_numpy(values(codes[:, :cols], bytes_)).float().to(dtype)
    for before, after in ((0, 0), (3, 2)):
        room = torch.full((rows, before + cols + after), 7.0, dtype=dtype, device="cuda")
        adacc.mx4_decompress(blob, room[:, before:before + cols])
        got = room.cpu()
        assert (got[:, :before] == 7.0).all() and (got[:, before + cols:] == 7.0).all()
        got = got[:, before:before + cols]
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(1.0), want.nan_to_num(1.0))


def test_large_matrix_by_samples():
    """More than 2^31 values: offsets that pass 32 bits."""
    rows, cols = (1 << 17) + 40, 16384 + 64
    print(f"[mx4] {rows} x {cols}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(rows, cols, generator=g, device="cuda", dtype=torch.bfloat16)
    m, t = mx4.compress_both(x)
    back, across = m.restore(), t.restore()
    pick = [0, 1, 65535, 65536, 131071, 131072, rows - 1]
    assert np.array_equal(f64(back[pick]), values(*quantise(f64(x[pick]))))
    cpick = [0, 511, 512, 16383, 16384, cols - 1]
    assert np.array_equal(f64(across[cpick]), values(*quantise(f64(x[:, cpick]).T)))


def test_empty():
    for shape in ((0, 5), (5, 0), (0, 4, 4), (3, 0, 8)):
        m = mx4.compress(torch.empty(shape, device="cuda"))
        assert m.restore(torch.float32).shape == shape

"""Microscaled 4-bit floating point in 64 bits, from the format's definition, and the blob's bytes; shared by the tests of adacc_mx4_*."""
import numpy as np
import torch

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
TYPES = [torch.bfloat16, torch.float16, torch.float32]
# half a step relative to the value
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}  # half a step of the subnormal numbers


def f64(t):
    return t.detach().cpu().double().numpy()


def quantise(x, fullrange=0):
    """x [rows, cols] in binary64 -> (codes [rows, cols], scale bytes [rows, blocks])"""
    rows, cols = x.shape
    blocks = -(-cols // 32)
    codes = np.zeros((rows, cols), np.uint8)
    bytes_ = np.zeros((rows, blocks), np.uint8)
    for b in range(blocks):
        part = x[:, 32 * b:32 * b + 32]
        finite = np.isfinite(part).all(1)
        v = np.where(finite[:, None], part, 0.0)
        top = np.abs(v).max(1)
        e = np.full(rows, -127)
        some = top > 0
        e[some] = np.frexp(top[some])[1] - 1 - 2  # floor(log2) - 2
        if fullrange:
            e[some] += top[some] > 6.0 * np.exp2(e[some].astype(float))
        e = np.maximum(e, -127)
        r = np.abs(v) / np.exp2(e.astype(float))[:, None]
        far = np.abs(r[:, :, None] - GRID)  # (exact: few bits)
        near = far.min(2, keepdims=True)
        is_near = far == near
        even = is_near & (np.arange(8) % 2 == 0)
        code = np.where(is_near.sum(2) > 1, even.argmax(2), is_near.argmax(2))
        code = code + 8 * np.signbit(v)
        codes[:, 32 * b:32 * b + 32] = np.where(finite[:, None], code, 0)
        bytes_[:, b] = np.where(finite, e + 127, 255)
    return codes, bytes_


def values(codes, bytes_):
    """What codes and scale bytes stand for, binary64."""
    v = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    scale = np.where(bytes_ == 255, np.nan, np.exp2(bytes_.astype(float) - 127.0))
    return v * np.repeat(scale, 32, axis=1)[:, :codes.shape[1]]


def rounded(x, fullrange=0):
    return values(*quantise(x, fullrange))


def grouped_positions(offsets):
    """(first position of every group, positions in all): groups start at multiples of 128."""
    at, first = 0, []
    for a, b in zip(offsets, offsets[1:]):
        first.append(at)
        at += -(-(b - a) // 128) * 128
    return first, at


def quantise_groups(x, offsets, positions, fullrange=0):
    """x [rows, cols] -> codes [cols, positions] and bytes [cols, positions / 32] of the transposed matrix, blocks cut at the groups"""
    cols = x.shape[1]
    codes, bytes_ = np.zeros((cols, positions), np.uint8), np.zeros((cols, positions // 32), np.uint8)
    for p, a, b in zip(grouped_positions(offsets)[0], offsets, offsets[1:]):
        if b > a:
            c, s = quantise(x[a:b].T, fullrange)
            codes[:, p:p + b - a] = c
            bytes_[:, p // 32:p // 32 + s.shape[1]] = s
    return codes, bytes_


def blob_parts(blob, layout, rows, cols):
    """(codes [rows, 128 * steps], scale bytes [rows, 4 * steps]) as the blob holds them, padding included"""
    raw = blob.cpu().numpy()
    steps = -(-cols // 128)
    packed = raw[layout.codes_off:layout.codes_off + steps * layout.step_bytes].reshape(steps, rows, 64).transpose(1, 0, 2)
    codes = np.stack((packed & 15, packed >> 4), 3).reshape(rows, 128 * steps)
    s = raw[layout.scales_off:layout.scales_off + 4 * steps * layout.scale_pitch].reshape(4 * steps, layout.scale_pitch)
    return codes, s[:, :rows].T


def padded(a, cols):
    return np.pad(a, ((0, 0), (0, cols - a.shape[1])))


def matrix(rows, cols, dtype, seed, spread=2.0):
    """Rows of very different ranges, with outliers."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-int(4 * spread), int(4 * spread) + 1, (rows, 1), generator=g).float())
    x *= torch.where(torch.rand(rows, cols, generator=g) < 0.01, 20.0, 1.0)
    if dtype == torch.float16:
        x = x.clamp(-60000, 60000)
    return x.to(dtype)


def assert_product(got, a, b, dtype, sums):
    """got against the binary64 product a @ b.T: `sums` binary32 additions in a row, each off by a step of the sum of magnitudes at most,
    and one rounding to dtype."""
    want, size = a @ b.T, np.abs(a) @ np.abs(b).T
    got = f64(got)
    bad = np.isnan(want)
    assert np.array_equal(np.isnan(got), bad)
    exact = size * sums * 2.0 ** -23
    room = exact + (np.abs(want) + exact) * HALF_STEP[dtype] + TINY[dtype]
    off = np.abs(got - want) - room
    off[bad] = -1.0
    assert off.max(initial=-1.0) <= 0, f"{(off > 0).sum()} of {off.size} are off, worst {np.abs(got - want)[off > 0].max()}"

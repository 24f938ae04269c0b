"""mx4.linear and mx4.experts as layers: gradients against the formula and against differences, streams, graphs, views."""
import numpy as np
import pytest
import torch

import paper_2508_00806_amd as adacc
from mx4_reference import HALF_STEP, assert_product, f64, matrix, quantise_groups, rounded, values
from paper_2508_00806_amd import mx4

pytestmark = pytest.mark.gpu


def sums(k):
    return 2 * (-(-k // 64)) + 10


def representable(rows, cols, seed):
    """Values that keep their value in a block along either direction: whole numbers of at most 4 in magnitude, 4 in every block."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randint(-4, 5, (rows, cols), generator=g).float()
    for i in range(32):  # (a permutation's diagonal in every 32 x 32 tile)
        x[i::32, (7 * i + 3) % 32::32] = 4.0
    return x


@pytest.mark.parametrize("shape", [(64, 96, 160), (32, 32, 32), (320, 256, 192)])
def test_gradients_against_differences(shape):
    """Where every value is representable nothing is rounded, and y = x w^T: its gradients, and its differences, are whole numbers."""
    m, n, k = shape
    print(f"[mx4 layer] {shape}", flush=True)
    x, w, c = representable(m, k, 1), representable(n, k, 2), representable(m, n, 3)
    xg, wg = x.cuda().requires_grad_(), w.cuda().requires_grad_()
    y = mx4.linear(xg, wg)
    assert np.array_equal(f64(y), f64(x) @ f64(w).T)
    y.backward(c.cuda())
    assert np.array_equal(f64(xg.grad), f64(c) @ f64(w)) and np.array_equal(f64(wg.grad), f64(c).T @ f64(x))
    # differences of the layer's own output: steps from -2 to 2 stay representable
    loss = lambda a, b: (f64(mx4.linear(a.cuda(), b.cuda())) * f64(c)).sum()
    for t, grad, which in ((x, xg.grad, 0), (w, wg.grad, 1)):
        for i, j in ((0, 0), (5, 9), (t.shape[0] - 1, t.shape[1] - 1)):
            up, down = t.clone(), t.clone()
            if up[i, j].abs() == 4.0:
                j = (j + 1) % t.shape[1]
            up[i, j], down[i, j] = 2.0, -2.0
            diff = (loss(up, w) - loss(down, w)) / 4 if which == 0 else (loss(x, up) - loss(x, down)) / 4
            assert diff == f64(grad)[i, j]


@pytest.mark.parametrize("dtype,wtype", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float16, torch.float16), (torch.float32, torch.float32)])
@pytest.mark.parametrize("m,n,k", [(1, 30, 40), (77, 130, 264), (1000, 515, 300), (2100, 2048, 520)])
def test_gradients_against_the_formula(m, n, k, dtype, wtype):
    print(f"[mx4 layer] {m} {n} {k} {dtype} {wtype}", flush=True)
    x, w, dy = matrix(m, k, dtype, 1, 0.5), matrix(n, k, wtype, 2, 0.5), matrix(m, n, dtype, 3, 0.5)
    xg, wg = x.cuda().requires_grad_(), w.cuda().requires_grad_()
    y = mx4.linear(xg, wg, out_dtype=torch.float32)
    y.backward(dy.cuda().float())
    xt, wt, dyt = (rounded(f64(t).T) for t in (x, w, dy))
    assert_product(y, rounded(f64(x)), rounded(f64(w)), torch.float32, sums(k))
    if dtype != torch.float16:
        assert_product(xg.grad, rounded(f64(dy)), wt, dtype, sums(n))
        assert_product(wg.grad, dyt, xt, wtype, sums(m))
    assert xg.grad.dtype == dtype and wg.grad.dtype == wtype


OFFSETS = [[0, 5, 5, 40], [0, 0, 300, 301, 700], [0, 128, 1200], list(range(0, 130, 2))]


@pytest.mark.parametrize("offsets", OFFSETS, ids=lambda o: f"{len(o) - 1}groups{o[-1]}rows")
@pytest.mark.parametrize("tail", [0, 5])
def test_experts_gradients_against_the_formula(offsets, tail):
    print(f"[mx4 experts] {offsets[:6]} tail={tail}", flush=True)
    n, k, experts, rows = 140, 200, len(offsets) - 1, offsets[-1] + tail
    x, w, dy = matrix(rows, k, torch.bfloat16, 1, 0.5), matrix(experts * n, k, torch.float32, 2, 0.5).view(experts, n, k), matrix(rows, n, torch.bfloat16, 3, 0.5)
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
        assert_product(y[a:b], rounded(f64(x[a:b])), rounded(f64(w[e])), torch.bfloat16, sums(k))
        assert_product(dx[a:b], rounded(f64(dy[a:b])), rounded(f64(w[e]).T), torch.bfloat16, sums(n))
        assert_product(dw[e], dyt[:, at:at + b - a], xt[:, at:at + b - a], torch.float32, sums(b - a))
        at += -(-(b - a) // 128) * 128
    assert (y[offsets[-1]:] == 0).all() and (dx[offsets[-1]:] == 0).all()


def test_only_what_is_asked_for():
    x, w = matrix(80, 64, torch.bfloat16, 1).cuda(), matrix(48, 64, torch.bfloat16, 2).cuda()
    dy = matrix(80, 48, torch.bfloat16, 3).cuda()
    both = torch.autograd.grad(mx4.linear(x.requires_grad_(), w.requires_grad_()), (x, w), dy)
    (dx,) = torch.autograd.grad(mx4.linear(x, w.detach()), (x,), dy)
    (dw,) = torch.autograd.grad(mx4.linear(x.detach(), w), (w,), dy)
    assert torch.equal(dx, both[0]) and torch.equal(dw, both[1])
    with torch.no_grad():
        assert not mx4.linear(x, w).requires_grad


def test_views_broadcast_gradients_and_leading_dimensions():
    x = matrix(60, 70, torch.bfloat16, 1).cuda()
    w = matrix(64, 90, torch.bfloat16, 2).cuda()
    xv, wv = x.t()[:64].t(), w.t()[5:69].t()  # neither has adjacent columns in one piece
    want = f64(mx4.linear(xv.contiguous(), wv.contiguous(), out_dtype=torch.float32))
    assert np.array_equal(f64(mx4.linear(xv, wv, out_dtype=torch.float32)), want)
    x3 = xv.contiguous().view(3, 20, 64).requires_grad_()
    y = mx4.linear(x3, wv)
    assert y.shape == (3, 20, 64) and np.array_equal(f64(y.float()).reshape(60, 64), f64(torch.from_numpy(want).bfloat16()))
    (dx,) = torch.autograd.grad(y.sum(), (x3,))  # a gradient with strides of zero
    (dx2,) = torch.autograd.grad(mx4.linear(x3, wv), (x3,), torch.ones_like(y))
    assert torch.equal(dx, dx2) and dx.shape == x3.shape


def test_on_another_stream():
    x, w = matrix(300, 512, torch.bfloat16, 1).cuda(), matrix(400, 512, torch.bfloat16, 2).cuda()
    want = mx4.linear(x, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        xs = x * 2
        held = mx4.compress(w)
        got = [mx4.linear(xs, w), mx4.linear(xs, held), mx4.linear(xs[:4], held)]
        xg = xs.clone().requires_grad_()
        y = mx4.linear(xg, w)
    torch.cuda.current_stream().wait_stream(side)
    for t, rows in zip(got, (300, 300, 4)):
        assert torch.equal(t, want[:rows] * 2)
    (dx,) = torch.autograd.grad(y, (xg,), y.detach())
    xg2 = (x * 2).requires_grad_()
    y2 = mx4.linear(xg2, w)
    assert torch.equal(dx, torch.autograd.grad(y2, (xg2,), y2.detach())[0])


@pytest.mark.parametrize("rows", [1, 24, 300])
def test_in_a_graph(rows):
    """A serving step: rows and offsets change between the replays."""
    k, n, experts = 256, 384, 6
    w = mx4.compress(matrix(experts * n, k, torch.bfloat16, 1).view(experts, n, k).cuda())
    x = torch.zeros(rows, k, dtype=torch.bfloat16, device="cuda")
    off = torch.zeros(experts + 1, dtype=torch.int32, device="cuda")
    warm = torch.cuda.Stream()
    warm.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(warm):
        mx4.experts(x, off, w)
    torch.cuda.current_stream().wait_stream(warm)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = mx4.experts(x, off, w)
    for turn in range(4):
        x.copy_(matrix(rows, k, torch.bfloat16, 10 + turn))
        cuts = torch.randint(0, rows + 1, (experts - 1,), generator=torch.Generator().manual_seed(turn)).sort().values.tolist()
        off.copy_(torch.tensor([0, *cuts, rows], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        assert torch.equal(got, mx4.experts(x, off, w))
        assert got.abs().max() > 0


def test_the_saved_form_is_small():
    """What the layer keeps for its backward pass: 4.25 bits a value of x and w, not 16."""
    x, w = torch.randn(4096, 1024, device="cuda", dtype=torch.bfloat16), torch.randn(1024, 1024, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    x.requires_grad_()
    kept = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t.numel() * t.element_size()) or t, lambda t: t):
        y = mx4.linear(x, w)
    assert sum(kept) == adacc.mx4_layout_of(1024, 4096).total_bytes + adacc.mx4_layout_of(1024, 1024).total_bytes
    assert sum(kept) <= 1.001 * 4.25 / 16 * 2 * (x.numel() + w.numel())
    y.sum().backward()
    assert x.grad.shape == x.shape and HALF_STEP[x.dtype] > 0


def test_the_example_learns_and_serves():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "mx4_experts.py")
    spec = importlib.util.spec_from_file_location("mx4_experts_example", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, err = example.main(["--steps", "12", "--tokens", "512", "--hidden", "256", "--ffn", "512", "--experts", "4"])
    assert losses[-1] < 0.8 * losses[0]
    assert err <= 2.0 ** -5  # bf16 sums of values up to 8 in another order


@pytest.mark.parametrize("offsets", [[0, 500, 100, -3, 10 ** 9], [7, -1, 2 ** 31 - 1, 0, 64], [0, 300, 300, 299, 300], [300, 300, 300, 300, 300]])
def test_offsets_without_sense_lead_nowhere(offsets):
    """Offsets that do not ascend, or lead beyond the rows, are held between 0 and the number of rows: the results mean nothing, and nothing
    beside them is written."""
    print(f"[mx4 offsets] {offsets}", flush=True)
    n, k, rows, groups = 132, 256, 300, 4
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    x, w = matrix(rows, k, torch.bfloat16, 1).cuda(), mx4.compress(matrix(groups * n, k, torch.bfloat16, 2).view(groups, n, k).cuda())
    for take in (rows, 40):
        room = torch.full((take + 8, n), 7.0, device="cuda")
        out = room[4:4 + take]
        need = adacc.mx4_linear_workspace_bytes(take, n, k, groups)
        adacc.mx4_linear(x[:take], w.blob, out, offsets=off, workspace=torch.empty(max(need, 256), dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        assert (room[:4] == 7.0).all() and (room[4 + take:] == 7.0).all()
    positions = adacc.mx4_grouped_cols(rows, groups)
    size = int(adacc.mx4_layout_of(k, positions).total_bytes)
    blob = torch.full((size + 512,), 0xA5, dtype=torch.uint8, device="cuda")
    adacc.mx4_compress(x, None, blob[256:256 + size], offsets=off)
    grads = torch.full((groups + 2, k, k), 7.0, device="cuda")
    adacc.mx4_gradient(blob[256:256 + size], blob[256:256 + size], rows, grads[1:-1], offsets=off)
    torch.cuda.synchronize()
    assert (blob[:256] == 0xA5).all() and (blob[256 + size:] == 0xA5).all()
    assert (grads[0] == 7.0).all() and (grads[-1] == 7.0).all()


def test_more_elements_than_32_bits_count():
    """A tensor of 4.6e9 elements: both compressions, restorations and products with it, in places on either side of 2^31 and 2^32; results of 4.6e9."""
    rows, cols = 70001, 65544
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    for i in range(0, rows, 10000):
        x[i:i + 10000].normal_(generator=torch.Generator("cuda").manual_seed(i))
    along, across = mx4.compress_both(x)
    print("[mx4 large] compressed", flush=True)
    y = along.restore(torch.float32)
    for i in (0, 32764, 32768, 65532, rows - 9):
        assert np.array_equal(f64(y[i:i + 9]), rounded(f64(x[i:i + 9])))
    del y
    y = across.restore(torch.float32)
    for j in (0, 30677, 30681, 61355, cols - 9):
        assert np.array_equal(f64(y[j:j + 9]), rounded(f64(x[:, j:j + 9].t().contiguous())))
    del y, across
    print("[mx4 large] restored", flush=True)
    for m in (3, 40, 300):
        a = matrix(m, cols, torch.bfloat16, m)
        z = mx4.linear(a.cuda(), along, out_dtype=torch.float32)
        for i in (0, 32764, 65532, rows - 9):
            assert_product(z[:, i:i + 9], rounded(f64(a)), rounded(f64(x[i:i + 9])), torch.float32, sums(cols))
    del x, along, z
    print("[mx4 large] multiplied", flush=True)
    a, b = matrix(rows, 64, torch.bfloat16, 41), matrix(cols, 64, torch.bfloat16, 42)
    z = mx4.linear(a.cuda(), mx4.compress(b.cuda()))
    bv = rounded(f64(b))
    for i in (0, 32760, 65530, rows - 9):
        assert_product(z[i:i + 9], rounded(f64(a[i:i + 9])), bv, torch.bfloat16, sums(64))

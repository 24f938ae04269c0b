"""The layers on the GPU at the ends of their types' ranges and of their sizes, against their plain forms in 64 bits."""
import pytest
import torch

import paper_2508_00806_amd as adacc
from layers_reference import TYPES, act, close, groups, rand

pytestmark = pytest.mark.gpu
layers = pytest.importorskip("paper_2508_00806_amd.layers")
E = 2.0 ** -18
KINDS = ["gelu", "gelu_tanh", "silu"]


# results of one tile of 128, of a contraction that is cut, and of tiles of 256 (216 of them, where those of 128 come in four rounds)
@pytest.mark.parametrize("size", [(40, 60, 96), (500, 300, 4100), (3400, 3900, 1000)])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_kept_pre_activation_stays_in_its_types_range(dtype, kind, size):
    """Columns whose bias takes what the activation is given out of the 16-bit type's range, not out of binary32's: results and gradients are those of the formula, where an infinity would
    have no slope.  An infinity that was one stays one.  Tolerances of sums as for every other product: (k + 8) 2^-24 of the sum of the magnitudes, half a step of dpre."""
    m, n, k = size
    t = TYPES[dtype]
    far = 1e5 if dtype == "f16" else 3.4e38
    x, w = rand((m, k), t, 1), rand((n, k), t, 2, 0.5 / k ** 0.5)
    b = rand((n,), torch.float32, 3)
    low, high, none = [torch.arange(i, n, 7, device="cuda") for i in (1, 3, 5)]
    b[low], b[high] = -far, far
    dy = rand((m, n), t, 4, 0.1)
    leaves = [v.requires_grad_() for v in (x, w, b)]
    y = layers.linear(x, w, b, kind, saved="input")
    kept = [v for v in y.grad_fn.saved_tensors if v is not None][-1]
    most = torch.finfo(t).max
    assert kept.dtype == t and bool((kept[:, low] == -most).all()) and bool((kept[:, high] == most).all()) and bool(torch.isfinite(kept).all())
    assert bool((y.detach()[:, low] == 0).all()) and bool((y.detach()[:, high] == float("inf")).all())
    dx, dw, db = torch.autograd.grad(y, leaves, dy)
    D, X, W = dy.double(), x.detach().double(), w.detach().double()
    back = kept.double().clamp(-1e5, 1e5)  # (every slope there is 0 or 1; the reference's cube would leave the range of 64 bits)
    dpre = D * act(kind, back)[1]
    bend = D.abs() * E * (1 + back.abs().clamp(max=100.0)) + torch.finfo(t).eps / 2 * torch.finfo(t).smallest_normal
    half = torch.finfo(t).eps / 2
    close(dx, dpre @ W, t, (half + (n + 8) * 2.0 ** -24) * (dpre.abs() @ W.abs()) + bend @ W.abs(), "dx")
    close(dw, dpre.t() @ X, t, (half + (m + 8) * 2.0 ** -24) * (dpre.abs().t() @ X.abs()) + bend.t() @ X.abs(), "dw")
    close(db, dpre.sum(0), torch.float32, (m + 8) * 2.0 ** -24 * dpre.abs().sum(0) + bend.sum(0), "db")
    assert not bool(dw[low].any()) and not bool(db[low].any())
    with torch.no_grad():
        b[none] = -float("inf")
    y = layers.linear(x, w, b, kind, saved="input")
    kept = [v for v in y.grad_fn.saved_tensors if v is not None][-1]
    assert bool((kept[:, none] == -float("inf")).all()) and bool((kept[:, low] == -most).all())


# ---------------------------------------------------------------- small results of activations
LOWEST = {"gelu": -13.2, "gelu_tanh": -10.5, "silu": -90.0}


def tail_bound(kind, x, dtype):
    """(relative error of share and of what makes the slope) of activations at negative x, by the steps that lead there.
      gelu, 16 bits: the tail's fit, 1.9e-5 up to 6 and 1.5e-4 beyond, evaluation included, and an exponential
      gelu, binary32: the fit, 3.9e-7, three roundings of an argument of x^2 / 2, an exponential, four products
      silu, gelu_tanh: two and eight roundings of an argument z, an exponential, a sum, a reciprocal, a product"""
    if kind == "gelu":
        return 2.0 ** -20 + x * x * 2.0 ** -23 if dtype == torch.float32 else torch.where(x.abs() <= 6, 2.0 ** -15, 2.0 ** -12).double()
    z = x.abs() if kind == "silu" else 1.5957691216 * x.abs() * (1 + 0.044715 * x * x)
    return 2.0 ** -21 + z * (2.0 ** -23 if kind == "silu" else 2.0 ** -21)


def check_tail(kind, x, y, dx, dtype):
    """Relative to the result, however small it is: half a step of the type and the bound above; shares below 2^-126, and steps below the smallest normal number, count as they are."""
    x = x.detach().double()
    value, slope = act(kind, x)
    z = x.abs() if kind != "gelu_tanh" else 1.5957691216 * x.abs() * (1 + 3 * 0.044715 * x * x)
    f = torch.finfo(dtype)
    least, bound = f.smallest_normal * f.eps / 2, tail_bound(kind, x, dtype)

    def within(got, want, size, floor, what):
        off = (got.detach().double() - want).abs() - f.eps / 2 * want.abs() - bound * size - floor
        at = int(off.argmax())
        assert float(off.max()) <= 0, f"{what} at {float(x.flatten()[at])}: {float(got.flatten()[at])} for {float(want.flatten()[at])}"
    within(y, value, value.abs(), least + 2.0 ** -126 * x.abs(), "y")
    if dx is not None:
        share = value / x
        bound = bound + 2.0 ** -21
        within(dx, slope, share + (share - slope).abs(), least + 2.0 ** -126 * (2 + z), "dx")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
def test_small_results_of_activations_are_as_exact_as_large_ones(dtype, kind):
    t = TYPES[dtype]
    x = torch.linspace(LOWEST[kind], -2.0 ** -6, 97 * 130).view(97, 130).to(t).cuda().requires_grad_()
    y = layers.activation(x, kind, saved="input")
    dx, = torch.autograd.grad(y, x, torch.ones_like(y))
    check_tail(kind, x, y, dx, t)
    # a gate of them: the product's rounding is the only one more
    with torch.no_grad():
        assert torch.equal(layers.gated(x, torch.ones_like(x), kind), y)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("m,n", [(5, 1500), (70, 1500), (3400, 3900)])
def test_small_results_of_products(m, n, dtype, kind):
    """Few rows, tiles of 128 and of 256; sums that are one value of w each."""
    t = TYPES[dtype]
    w = torch.zeros((n, 40), dtype=t, device="cuda")
    w[:, 33] = torch.linspace(LOWEST[kind], -2.0 ** -6, n).to(t)
    x = torch.zeros((m, 40), dtype=t, device="cuda")
    x[:, 33] = 1
    y = layers.linear(x, w, activation=kind)
    assert torch.equal(y, y[:1].expand(m, n))
    check_tail(kind, w[:, 33], y[0], None, t)


# ---------------------------------------------------------------- groups with the largest numbers
def test_groups_with_the_largest_binary32_numbers_restore_to_finite_ones():
    """Half of a scale, and the scale's own rounding 127 times: 0.5001 of it.  (M / 127 rounded up, times 127, would be infinite.)"""
    most = torch.finfo(torch.float32).max
    x = rand((5, 300), torch.float32, 1, 1e36)
    x[0, 7], x[1, 130], x[2, 299] = most, -most, most
    x[3, 0] = torch.nextafter(torch.tensor(most), torch.tensor(0.0)).item()
    x[4] = -most
    back = layers.compress(x).restore(torch.float32)
    assert bool(torch.isfinite(back).all())
    scale = torch.nn.functional.pad(x, (0, 84)).unflatten(-1, (3, 128)).abs().amax(-1).double() / 127
    assert float(((back.double() - x.double()).abs() / scale.repeat_interleave(128, -1)[:, :300]).max()) <= 0.5001
    x.requires_grad_()
    for kind in KINDS:  # masks of the type's lowest value, which no gradient reaches
        dx, = torch.autograd.grad(layers.activation(x, kind), x, torch.ones_like(x))
        assert bool(torch.isfinite(dx).all()) and not bool(dx[4].any()) and float(dx[1, 130]) == 0 and float(dx[0, 7]) == 1


# ---------------------------------------------------------------- sizes near the limits
def test_parameters_of_more_columns_than_one_launch_sums():
    """A row of 2^27 + 72 columns: mean and averages are sums of 16385 values a lane, and ten steps between the lanes: within 2^14.1 2^-24 of the sum of the magnitudes."""
    cols = (1 << 27) + 72
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((1, cols), generator=g, device="cuda", dtype=torch.bfloat16).requires_grad_()
    w = torch.ones(cols, device="cuda", dtype=torch.bfloat16).requires_grad_()
    b = torch.zeros(cols, device="cuda", dtype=torch.bfloat16).requires_grad_()
    dy = torch.randn((1, cols), generator=g, device="cuda", dtype=torch.bfloat16)
    y = layers.layer_norm(x, w, b, saved="input")
    dw, db = torch.autograd.grad(y, (w, b), dy)
    assert torch.equal(db, dy[0])
    off = 2.0 ** -9.8
    for part in (slice(0, 1 << 20), slice(cols - (1 << 20), cols)):
        v, d = x.detach()[0, part].double(), dy[0, part].double()  # mean 0 and deviation 1, within 2^-12 of them
        close(dw[part], d * v, torch.bfloat16, off * d.abs() * (1 + v.abs()), "dw")
        close(y.detach()[0, part], v, torch.bfloat16, off * (1 + v.abs()), "y")


def test_a_bias_of_more_columns_than_one_launch_sums():
    n = (1 << 28) + 72
    dy = torch.randn((1, n), device="cuda", dtype=torch.bfloat16)
    db = torch.empty(n, device="cuda", dtype=torch.bfloat16)
    adacc.linear_columns(dy, dbias=db, workspace=torch.empty(adacc.linear_columns_workspace_bytes(1, n), dtype=torch.uint8, device="cuda"))
    assert torch.equal(db, dy[0])


def test_as_many_rows_as_there_may_be():
    """2^30 rows of one value, which take two launches: what the same values in rows of 2^15 give."""
    rows = 1 << 30
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty((rows, 1), device="cuda", dtype=torch.bfloat16)
    x.view(-1, 1 << 24)[:] = torch.randn((1 << 6, 1 << 24), generator=g, device="cuda", dtype=torch.bfloat16)
    wide = x.view(1 << 15, 1 << 15)
    assert torch.equal(layers.activation(x).view_as(wide), layers.activation(wide))
    grads = []
    for v in (x, wide):
        v = v.detach().requires_grad_()
        grads.append(torch.autograd.grad(layers.activation(v, "silu", saved="input"), v, x.view_as(v))[0])
    assert torch.equal(grads[0].view_as(wide), grads[1])
    del grads
    kept = layers.compress(x)  # (a group of one value: its code is 127, with the value's sign)
    back = kept.restore(torch.bfloat16)
    assert torch.equal(back, x)


@pytest.mark.parametrize("saved", ["codes", "input"])
def test_a_product_of_one_row_longer_than_rows_may_lie_apart(saved):
    """One row by one row of 2^23 + 77 values.  The result: a sum of k products, (k + 8) 2^-24 of the magnitudes at most; dx and dw: one product each, of dpre rounded to its type."""
    k = (1 << 23) + 77
    x, w = rand((1, k), torch.bfloat16, 1), rand((1, k), torch.bfloat16, 2, 2.0 ** -12)
    leaves = [t.requires_grad_() for t in (x, w)]
    y = layers.linear(x, w, activation="silu", saved=saved)
    dy = torch.full((1, 1), 0.5, dtype=torch.bfloat16, device="cuda")
    kept = [t for t in y.grad_fn.saved_tensors if t is not None][-1]
    pre = layers.Rows8(kept, (1, 1)).restore(torch.float32).double() if saved == "codes" else kept.double()
    dx, dw = torch.autograd.grad(y, leaves, dy)
    X, W = x.detach().double(), w.detach().double()
    exact, size = (X * W).sum(), (X * W).abs().sum()
    assert float((pre - exact).abs()) <= float((k + 8) * 2.0 ** -24 * size + exact.abs() * 2.0 ** -7)
    dpre = 0.5 * act("silu", pre)[1]
    near = torch.finfo(torch.bfloat16).eps / 2 + E
    restored = groups(x.detach())[2].bfloat16().double() if saved == "codes" else X
    close(dx, dpre * W, torch.bfloat16, near * (dpre * W).abs() + E * W.abs() * (1 + pre.abs()), "dx")
    close(dw, dpre * restored, torch.bfloat16, near * (dpre * restored).abs() + E * restored.abs() * (1 + pre.abs()), "dw")


def test_one_row_by_as_many_as_there_may_be():
    n = 1 << 30
    w = torch.zeros((n, 8), dtype=torch.bfloat16, device="cuda")
    w[:, 5] = (torch.arange(n, device="cuda") % 251).bfloat16()
    x = torch.tensor([[7.0, 0, 0, 0, 0, 3.0, 0, 1.0]], dtype=torch.bfloat16, device="cuda")
    y = layers.linear(x, w)
    for i in range(0, n, 1 << 28):
        assert torch.equal(y[0, i:i + (1 << 28)], (3.0 * w[i:i + (1 << 28), 5].float()).bfloat16())


# ---------------------------------------------------------------- what no wanted gradient takes is not kept
def kept_by(call):
    """(result, bytes of every tensor that is kept for the backward pass)"""
    kept = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t.nbytes) or t, lambda t: t):
        y = call()
    return y, sorted(kept)


@pytest.mark.parametrize("saved", ["codes", "input"])
@pytest.mark.parametrize("cols", [96, 700, 3001, 17000])
def test_a_norm_whose_bias_alone_is_trained_keeps_nothing_of_its_rows(cols, saved):
    x, w, b, dy = rand((33, cols), torch.bfloat16, 1), rand((cols,), torch.bfloat16, 2) + 1, rand((cols,), torch.bfloat16, 3), rand((33, cols), torch.bfloat16, 4)
    every = [t.clone().requires_grad_() for t in (x, w, b)]
    y = layers.layer_norm(*every, saved=saved)
    want = torch.autograd.grad(y, every, dy)[2]
    got, kept = kept_by(lambda: layers.layer_norm(x, w, b.requires_grad_(), saved=saved))
    assert kept == sorted([33 * 8, w.nbytes]) and torch.equal(got, y)
    assert torch.equal(torch.autograd.grad(got, b, dy)[0], want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("saved", ["codes", "input"])
def test_a_gated_activation_of_which_up_alone_is_trained_keeps_the_gate_alone(saved, dtype):
    t = TYPES[dtype]
    x, u, dy = rand((5, 9, 301), t, 1), rand((5, 9, 301), t, 2), rand((5, 9, 301), t, 3)
    both = [v.clone().requires_grad_() for v in (x, u)]
    y = layers.gated(*both, "gelu", saved=saved)
    want = torch.autograd.grad(y, both, dy)
    got, kept = kept_by(lambda: layers.gated(x, u.requires_grad_(), "gelu", saved=saved))
    assert kept == [layers.compress(x).nbytes if saved == "codes" else x.nbytes] and torch.equal(got, y)
    assert torch.equal(torch.autograd.grad(got, u, dy)[0], want[1])
    got, kept = kept_by(lambda: layers.gated(x.requires_grad_(), u.detach(), "gelu", saved=saved))  # the gate's takes both
    assert len(kept) == 2 and torch.equal(torch.autograd.grad(got, x, dy)[0], want[0])

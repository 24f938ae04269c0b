"""The layers on the GPU at the ends of their types' ranges and of their sizes, against their plain forms in 64 bits."""
import pytest
import torch

from layers_reference import TYPES, act, close, rand

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

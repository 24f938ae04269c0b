"""Matrices in microscaled 4-bit floating point, and layers that compute with them.

`compress` keeps a matrix in 4.25 bits a value (blocks of 32 values, one power of two each); `linear` and `experts` multiply rows of 16 or 32 bits
with weights in that form on the matrix cores.  Given a plain weight, they are differentiable: what is saved for the backward pass is
not the activation but its 4-bit form, compressed along the tokens while it is read for the product (Section 3.2 compresses saved
activations and restores them; here the gradient's product reads the codes as they are).

With MX(.) for the blocks along the rows and MXT(.) for those across them, the gradients go straight through the rounding:

    y = MX(x) MX(w)^T        dx = MX(dy) MXT(w)^T        dw = MXT(dy) MXT(x)^T

Plumbing only: buffers and calls; every step runs in the HIP kernels.
"""
import functools

import torch
from torch import _C
from torch.autograd import forward_ad

from . import (MX4_SCALE_FLOOR, MX4_SCALE_FULLRANGE, mx4_compress, mx4_decompress, mx4_gradient, mx4_grouped_cols, mx4_layout_of, mx4_linear,
               mx4_linear_workspace_bytes, mx4_product)

SCALE_RULES = {"floor": MX4_SCALE_FLOOR, "fullrange": MX4_SCALE_FULLRANGE}


def _rule(name):
    try:
        return SCALE_RULES[name]
    except KeyError:
        raise ValueError(f"scale_rule is one of {', '.join(SCALE_RULES)}, not {name!r}") from None


class Mx4Matrix:
    """A compressed matrix [rows, cols], or a stack [mats, rows, cols] of them, blocks along the rows."""
    __slots__ = ("blob", "shape")

    def __init__(self, blob, shape):
        self.blob, self.shape = blob, tuple(shape)

    @property
    def nbytes(self):
        return self.blob.numel()

    def restore(self, dtype=torch.bfloat16, out=None):
        """The matrix of the values that the codes stand for, in a tensor of its own or in `out`, which is of the matrix's shape, on its device."""
        _on_gpu(self.blob)
        if out is not None and out.device != self.blob.device:
            raise ValueError(f"out is on {out.device}, the matrix on {self.blob.device}")
        if _elsewhere(self.blob):
            with torch.cuda.device(self.blob.get_device()):
                return self.restore(dtype, out)
        out = torch.empty(self.shape, dtype=dtype, device=self.blob.device) if out is None else out
        if out.shape != self.shape:
            raise ValueError(f"out has shape {tuple(out.shape)}, the matrix {self.shape}")
        mx4_decompress(self.blob, out if out.dim() == 2 else out.view(out.shape[:-1].numel(), out.shape[-1]), stream=_stream_of(self.blob))
        return out


def _stream_of(t):
    """The current stream of the tensor's device, as a handle."""
    return _C._cuda_getCurrentRawStream(t.get_device())


def _elsewhere(t):
    """Whether another device than the tensor's is current.  A launch goes to the current one (and the default stream has one handle on all of
    them), so every call makes its tensors' device current; in a backward pass the autograd engine has done so."""
    at = t.get_device()
    return at >= 0 and at != _C._cuda_getDevice()


def _flat(x):
    """[..., cols] as a matrix with adjacent columns (a copy only where the strides ask for one)."""
    if x.dim() != 2:
        x = x.reshape(x.shape[:-1].numel(), x.shape[-1])  # (not -1: the last dimension may be empty)
    stride, step = x.stride()
    rows, cols = x.shape
    return x if (step == 1 or cols <= 1) and (stride >= cols or rows <= 1) else x.contiguous()


def _stack(x):
    if x.dim() == 2:
        return _flat(x)
    if x.dim() != 3:
        raise ValueError(f"a matrix or a stack of matrices is needed, not {x.dim()} dimensions")
    _, rows, cols = x.shape
    plain = (x.stride(2) == 1 or cols <= 1) and (x.stride(1) >= cols or rows <= 1)
    return x if plain else x.contiguous()


@functools.lru_cache(maxsize=4096)
def _blob_bytes(rows, cols):
    return int(mx4_layout_of(rows, cols).total_bytes)


@functools.lru_cache(maxsize=4096)
def _positions(rows, groups):
    return mx4_grouped_cols(rows, groups)


def _buffer(nbytes, device):
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _blobs(x, along, across, rule, offsets=None):
    rows, cols = x.shape[-2:]
    mats = x.shape[0] if x.dim() == 3 else 1
    a = _buffer(_blob_bytes(mats * rows, cols), x.device) if along else None
    t = None
    if across:
        t = _buffer(_blob_bytes(mats * cols, rows if offsets is None else _positions(rows, offsets.shape[0] - 1)), x.device)
    mx4_compress(x, a, t, offsets=offsets, scale_rule=rule, stream=_stream_of(x))
    return a, t


def compress(x, scale_rule="floor"):
    """x: a matrix or a stack of matrices of bfloat16, float16 or float32; blocks along the last dimension.  The result is bytes: no gradient passes."""
    _on_gpu(x)
    if _elsewhere(x):
        with torch.cuda.device(x.get_device()):
            return compress(x, scale_rule)
    x = _stack(x.detach() if x.requires_grad else x)
    return Mx4Matrix(_blobs(x, True, False, _rule(scale_rule))[0], x.shape)


def compress_both(x, scale_rule="floor"):
    """(x, x transposed), both compressed, from one reading of x: blocks along the last dimension, and along the one before it."""
    _on_gpu(x)
    if _elsewhere(x):
        with torch.cuda.device(x.get_device()):
            return compress_both(x, scale_rule)
    x = _stack(x.detach() if x.requires_grad else x)
    along, across = _blobs(x, True, True, _rule(scale_rule))
    return Mx4Matrix(along, x.shape), Mx4Matrix(across, (*x.shape[:-2], x.shape[-1], x.shape[-2]))


def _serve(x, w, offsets, out_dtype):
    rows = _flat(x)
    m, k = rows.shape
    n = w.shape[-2]
    groups = 0 if offsets is None else offsets.numel() - 1
    out = torch.empty((m, n), dtype=out_dtype or x.dtype, device=x.device)
    need = mx4_linear_workspace_bytes(m, n, k, groups)
    ws = _buffer(need, x.device) if need else None
    mx4_linear(rows, w.blob, out, offsets=offsets, workspace=ws, stream=_stream_of(x))
    return out if x.dim() == 2 else out.view(*x.shape[:-1], n)


class _Served(torch.autograd.Function):
    """A product with a kept weight, of rows that a gradient is wanted for.  It has none: the weight's codes have their blocks along the contraction, the
    gradient of the rows needs them across it.  A backward pass that comes here says so; cut off, the rows would be left without a word."""
    @staticmethod
    def forward(ctx, x, w, offsets, out_dtype):
        return _serve(x, w, offsets, out_dtype)

    @staticmethod
    def backward(ctx, dy):
        raise RuntimeError("a product with an Mx4Matrix has no gradient: pass the weight itself to train through it, or detach the rows")


def _served(x, w, offsets, out_dtype):
    if (x.requires_grad and torch.is_grad_enabled()) or forward_ad._current_level >= 0:
        return _Served.apply(x, w, offsets, out_dtype)
    return _serve(x, w, offsets, out_dtype)


class _Layer(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, offsets, out_dtype):
        rows, w_ = _flat(x), _stack(w)
        need_dx, need_dw = ctx.needs_input_grad[:2]
        rule = MX4_SCALE_FLOOR
        xa, xt = _blobs(rows, True, need_dw, rule, offsets)
        wa, wt = _blobs(w_, True, need_dx, rule)
        m, n, k = rows.shape[0], w.shape[-2], w.shape[-1]
        out = torch.empty((m, n), dtype=out_dtype or x.dtype, device=x.device)
        mx4_product(xa, wa, k, out, offsets=offsets, stream=_stream_of(x))
        ctx.save_for_backward(xt, wt, offsets)
        ctx.x_shape, ctx.x_dtype, ctx.w_shape, ctx.w_dtype = x.shape, x.dtype, w.shape, w.dtype
        return out.view(*x.shape[:-1], n)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        xt, wt, offsets = ctx.saved_tensors
        need_dx, need_dw = ctx.needs_input_grad[:2]
        n, k = ctx.w_shape[-2:]
        dy = _flat(dy)
        ga, gt = _blobs(dy, need_dx, need_dw, MX4_SCALE_FLOOR, offsets)
        dx = dw = None
        if need_dx:
            dx = torch.empty((dy.shape[0], k), dtype=ctx.x_dtype, device=dy.device)
            mx4_product(ga, wt, n, dx, offsets=offsets, stream=_stream_of(dy))
            dx = dx.view(ctx.x_shape)
        if need_dw:
            dw = torch.empty(ctx.w_shape, dtype=ctx.w_dtype, device=dy.device)
            mx4_gradient(gt, xt, dy.shape[0], dw, offsets=offsets, stream=_stream_of(dy))
        return dx, dw, None, None


def _on_gpu(x):
    if not x.is_cuda:
        raise ValueError(f"a tensor on a GPU is needed, not on {x.device}")


def _check_operands(x, w, mats):
    shape, w_shape = x.shape, w.shape
    if len(w_shape) != (3 if mats else 2):
        raise ValueError(f"the weight must have {3 if mats else 2} dimensions, not {len(w_shape)}")
    if not shape or shape[-1] != w_shape[-1]:
        raise ValueError(f"rows of {shape[-1] if shape else 0} values do not fit a weight of shape {tuple(w_shape)}")
    _on_gpu(x)
    if (w.blob if isinstance(w, Mx4Matrix) else w).get_device() != x.get_device():
        raise ValueError("the weight must be on the device of the rows")


def linear(x, weight, out_dtype=None):
    """x [..., k] times weight [n, k], both in microscaled 4-bit floating point: [..., n] of x's type, or of out_dtype.

    weight: an `Mx4Matrix` (serving: a backward pass through it raises), or a tensor of bfloat16, float16 or float32, which is compressed by the call; gradients
    then reach x and weight, each in its own type."""
    _check_operands(x, weight, False)
    if _elsewhere(x):
        with torch.cuda.device(x.get_device()):
            return linear(x, weight, out_dtype)
    if isinstance(weight, Mx4Matrix):
        return _served(x, weight, None, out_dtype)
    return _Layer.apply(x, weight, None, out_dtype)


def experts(x, offsets, weight, out_dtype=None):
    """x [rows, k], rows sorted by expert, times the expert's own weight [n, k]: [rows, n].

    offsets: int32 tensor of experts + 1 entries on x's device; expert e has the rows offsets[e] to offsets[e + 1] (none, if they are equal).  It is
    read on the device, so nothing waits for it.  Rows behind the last expert's give zeros.  weight: an `Mx4Matrix` of shape
    [experts, n, k], or a tensor of it; gradients, or none, as in `linear`."""
    _check_operands(x, weight, True)
    if x.dim() != 2:
        raise ValueError("x must be a matrix")
    if offsets.get_device() != x.get_device():
        raise ValueError("offsets must be on the device of x")
    if offsets.numel() != weight.shape[0] + 1:
        raise ValueError(f"{weight.shape[0]} experts need {weight.shape[0] + 1} offsets, not {offsets.numel()}")
    if _elsewhere(x):
        with torch.cuda.device(x.get_device()):
            return experts(x, offsets, weight, out_dtype)
    if isinstance(weight, Mx4Matrix):
        return _served(x, weight, offsets, out_dtype)
    return _Layer.apply(x, weight, offsets, out_dtype)

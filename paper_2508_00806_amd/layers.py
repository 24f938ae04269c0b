"""The layers whose saved activations the paper compresses (Section 3.2: LayerNorm, GELU, Linear), with the compression in them.

`SavedActivationCompression` compresses what other operators save, in passes of its own; these layers write the 8-bit rows of their input while they read it, and their
gradients are computed from the codes as they are: nothing is restored to memory.

    layer_norm   y = (x - mean) / sigma * weight + bias
    activation   gelu, gelu_tanh, silu
    gated        act(gate) * up
    linear       act(x weight^T + bias) + residual, the last three in the product's epilogue

saved="codes": the backward pass has its input in 8 bits (groups of 128 values of a row, one scale each: 1.03 bytes a value), and the gradients are those at
the restored values; saved="input": as it was.  An input that holds an Inf or NaN has NaN for its whole group of 128 in the backward pass.

Calls can be captured into graphs, forward and backward; a captured backward pass, as of any function of torch, with no eager graph of the same leaves alive.

Plumbing only: buffers and calls; every step runs in the HIP kernels.
"""
import functools

import torch
from torch import _C
from torch.autograd import forward_ad

from . import ACT_GELU, ACT_GELU_TANH, ACT_NONE, ACT_SILU, LINEAR_ROWS_GRADIENT, LINEAR_SERVED, LINEAR_TRAINED, LINEAR_WEIGHT_GRADIENT, MX4_BF16, MX4_F16, MX4_F32
from . import _check, _layer, linear_columns_workspace_bytes, linear_workspace_bytes, norm_workspace_bytes, rows8_layout_of
from .mx4 import _buffer, _elsewhere, _flat, _on_gpu, _stream_of

ACTIVATIONS = {"gelu": ACT_GELU, "gelu_tanh": ACT_GELU_TANH, "silu": ACT_SILU}
_TYPES = {torch.bfloat16: MX4_BF16, torch.float16: MX4_F16, torch.float32: MX4_F32}
_STRIDE_MOST = 1 << 23  # elements between the rows of a product's operands: fewer
_PLAIN = torch.contiguous_format


def _kind(name):
    try:
        return ACTIVATIONS[name]
    except (KeyError, TypeError):
        raise ValueError(f"an activation is one of {', '.join(ACTIVATIONS)}, not {name!r}") from None


def _codes(saved):
    if saved != "codes" and saved != "input":
        raise ValueError(f"saved is 'codes' or 'input', not {saved!r}")
    return saved == "codes"


def _call(name, *args):
    """The library's function; the arguments have been checked here."""
    _check(_layer(name)(*args), name)


@functools.lru_cache(maxsize=4096)
def _rows8_bytes(rows, cols):
    return int(rows8_layout_of(rows, cols).total_bytes)


_norm_room = functools.lru_cache(maxsize=4096)(norm_workspace_bytes)
_linear_room = functools.lru_cache(maxsize=4096)(linear_workspace_bytes)
_columns_room = functools.lru_cache(maxsize=4096)(linear_columns_workspace_bytes)


def _stride(m):
    """Between the rows of a matrix that _flat made."""
    return m.stride(0) if m.shape[0] > 1 else m.shape[1]


def _place(t):
    """(address, stride) of such a matrix, or of None"""
    return (None, 0) if t is None else (t.data_ptr(), _stride(t))


def _at(t):
    return None if t is None else t.data_ptr()


def _bytes(t):
    """(address, size) of a buffer, or of None"""
    return (None, 0) if t is None else (t.data_ptr(), t.numel())


def _room(nbytes, device):
    return _buffer(nbytes, device) if nbytes else None


def _blob(rows, cols, device):
    return _buffer(_rows8_bytes(rows, cols), device)


def _differentiable(*tensors):
    if forward_ad._current_level >= 0:
        return True
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                return True
    return False


def _check_place(x):
    if _C._get_tracing_state() is not None:
        raise RuntimeError("a layer's call can not be recorded by torch.jit.trace, which sees the result's allocation alone; it can be captured into a graph")
    _on_gpu(x)


def _check_type(x, most=MX4_F32):
    _check_place(x)
    kind = _TYPES.get(x.dtype, MX4_F32 + 1)
    if kind > most:
        raise TypeError(f"{', '.join(str(t)[6:] for t, k in _TYPES.items() if k <= most)} is needed, not {x.dtype}")
    if x.dim() == 0:
        raise ValueError("rows of values are needed, not a single one")
    return kind


def _check_vector(v, what, n, x):
    if v.dim() != 1 or v.shape[0] != n:
        raise ValueError(f"{what} must have shape ({n},), not {tuple(v.shape)}")
    if v.dtype != x.dtype and v.dtype != torch.float32:
        raise TypeError(f"{what} must be {x.dtype} or torch.float32, not {v.dtype}")
    if v.get_device() != x.get_device():
        raise ValueError(f"{what} must be on the device of the rows")
    return _TYPES[v.dtype]


def _adjacent(v):
    return v if v is None or v.is_contiguous() else v.contiguous()


class Rows8:
    """A tensor in 8 bits: groups of 128 values along the last dimension with one scale each."""
    __slots__ = ("blob", "shape")

    def __init__(self, blob, shape):
        self.blob, self.shape = blob, tuple(shape)

    @property
    def nbytes(self):
        return self.blob.numel()

    def restore(self, dtype=torch.bfloat16):
        """The values that the codes stand for."""
        _check_place(self.blob)
        if _elsewhere(self.blob):
            with torch.cuda.device(self.blob.get_device()):
                return self.restore(dtype)
        if dtype not in _TYPES:
            raise TypeError(f"bfloat16, float16 or float32 is needed, not {dtype}")
        out = torch.empty(self.shape, dtype=dtype, device=self.blob.device)
        rows = _flat(out)
        _call("rows8_decompress", *_bytes(self.blob), *rows.shape, out.data_ptr(), _TYPES[dtype], rows.shape[1], _stream_of(self.blob))
        return out


def _compressed(rows, kind, stream):
    blob = _blob(*rows.shape, rows.device)
    _call("rows8_compress", kind, rows.data_ptr(), *rows.shape, _stride(rows), *_bytes(blob), stream)
    return blob


def compress(x):
    """x [..., cols] of bfloat16, float16 or float32 in 8 bits, as the layers save it.  The result is bytes: no gradient passes."""
    kind = _check_type(x)
    if _elsewhere(x):
        with torch.cuda.device(x.get_device()):
            return compress(x)
    return Rows8(_compressed(_flat(x.detach()), kind, _stream_of(x)), x.shape)


# ---------------------------------------------------------------- layer norm
def _normed(x, kind, wkind, w, b, eps, blob, stats):
    rows = _flat(x)
    n, cols = rows.shape
    y = torch.empty_like(x, memory_format=_PLAIN)
    _call("norm_forward", kind, rows.data_ptr(), n, cols, _stride(rows), wkind, _at(w), _at(b), eps, y.data_ptr(), cols, *_bytes(blob), _at(stats), _stream_of(x))
    return y


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, codes, kind, wkind):
        w = _adjacent(weight)
        cols = x.shape[-1]
        n = x.shape[:-1].numel()
        need = ctx.needs_input_grad[0] or ctx.needs_input_grad[1]  # (the bias's gradient takes nothing of x)
        blob = _blob(n, cols, x.device) if codes and need else None
        stats = torch.empty((n, 2), dtype=torch.float32, device=x.device)
        y = _normed(x, kind, wkind, w, _adjacent(bias), eps, blob, stats)
        ctx.save_for_backward(x if need and not codes else None, blob, stats, w)
        ctx.kinds = kind, wkind
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, blob, stats, w = ctx.saved_tensors
        need_x, need_w, need_b = ctx.needs_input_grad[:3]
        kind, wkind = ctx.kinds
        rows = _flat(dy)
        n, cols = rows.shape
        if x is not None:
            x = _flat(x)
        elif blob is None:
            x = rows  # (something of x's shape: db alone is wanted)
        dx = torch.empty_like(dy, memory_format=_PLAIN) if need_x else None
        wtype = torch.float32 if wkind == MX4_F32 else dy.dtype
        dw = torch.empty(cols, dtype=wtype, device=dy.device) if need_w else None
        db = torch.empty(cols, dtype=wtype, device=dy.device) if need_b else None
        room = _room(_norm_room(n, cols), dy.device) if need_w or need_b else None
        _call("norm_backward", kind, *_place(x), *_bytes(blob), n, cols, wkind, _at(w), stats.data_ptr(), rows.data_ptr(), _stride(rows), _at(dx), cols, _at(dw), _at(db), *_bytes(room),
              _stream_of(dy))
        return dx, dw, db, None, None, None, None


def layer_norm(x, weight=None, bias=None, eps=1e-5, saved="codes"):
    """The last dimension of x [..., cols] less its mean, divided by the root of its variance (about the mean, of the whole row) plus eps, times weight [cols], plus bias [cols].

    x: bfloat16, float16 or float32; the result is of its type.  weight and bias: of that type or float32, both of one; None: ones, zeros.  Gradients reach x, weight and bias."""
    codes = _codes(saved)
    kind = wkind = _check_type(x)
    cols = x.shape[-1]
    if bias is not None:
        wkind = _check_vector(bias, "bias", cols, x)
    if weight is not None:
        bkind, wkind = wkind, _check_vector(weight, "weight", cols, x)
        if bias is not None and bkind != wkind:
            raise TypeError("weight and bias must be of one type")
    eps = float(eps)
    if not eps >= 0:
        raise ValueError(f"eps must not be negative, it is {eps}")
    if _elsewhere(x):
        with torch.cuda.device(x.get_device()):
            return layer_norm(x, weight, bias, eps, saved)
    if _differentiable(x, weight, bias):
        return _LayerNorm.apply(x, weight, bias, eps, codes, kind, wkind)
    return _normed(x, kind, wkind, _adjacent(weight), _adjacent(bias), eps, None, None)


# ---------------------------------------------------------------- activations
def _halves(rows):
    half = rows.shape[1] // 2
    return rows[:, :half], rows[:, half:]


def _inputs(x, up, gated):
    """(gate, up) as matrices.  gated: 0 no, 1 by a tensor of its own, 2 by the second half of x"""
    if gated == 2:
        return _halves(_flat(x))
    return _flat(x), None if up is None else _flat(up)


def _activated(x, a, u, act, kind, a8, u8):
    n, cols = a.shape
    y = torch.empty_like(x, memory_format=_PLAIN) if cols == x.shape[-1] else torch.empty((*x.shape[:-1], cols), dtype=x.dtype, device=x.device)
    _call("act_forward", kind, act, a.data_ptr(), _stride(a), *_place(u), n, cols, y.data_ptr(), cols, *_bytes(a8), *_bytes(u8), _stream_of(x))
    return y


class _Activation(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, up, act, codes, gated, kind):
        a, u = _inputs(x, up, gated)
        a8 = _blob(*a.shape, x.device) if codes else None
        u8 = _blob(*a.shape, x.device) if codes and gated else None
        y = _activated(x, a, u, act, kind, a8, u8)
        if gated == 1 and not ctx.needs_input_grad[0]:  # up's gradient takes nothing of up
            up = u8 = None
        ctx.save_for_backward(*((None, None) if codes else (x, up)), a8, u8)
        ctx.how = act, kind, gated, x.shape
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, up, a8, u8 = ctx.saved_tensors
        act, kind, gated, shape = ctx.how
        need_x, need_up = ctx.needs_input_grad[:2]
        rows = _flat(dy)
        n, cols = rows.shape
        a, u = (None, None) if x is None else _inputs(x, up, gated)
        dx = dup = da = du = None
        if gated == 2:
            dx = torch.empty(shape, dtype=dy.dtype, device=dy.device)
            da, du = _halves(_flat(dx))
        else:
            if gated and up is None and u8 is None:
                u, u8 = (None, a8) if x is None else (rows, None)  # (something of up's shape)
            if need_x:
                dx = torch.empty_like(dy, memory_format=_PLAIN)
                da = _flat(dx)
            if gated and need_up:
                dup = torch.empty_like(dy, memory_format=_PLAIN)
                du = _flat(dup)
        _call("act_backward", kind, act, *_place(a), *_bytes(a8), *_place(u), *_bytes(u8), rows.data_ptr(), _stride(rows), n, cols, *_place(da), *_place(du), _stream_of(dy))
        return dx, dup, None, None, None, None


def _activate(x, up, act, codes, gated, kind):
    if _differentiable(x, up):
        return _Activation.apply(x, up, act, codes, gated, kind)
    return _activated(x, *_inputs(x, up, gated), act, kind, None, None)


def activation(x, kind="gelu", saved="codes"):
    """act(x) for x [..., cols] of bfloat16, float16 or float32: "gelu" (x Phi(x)), "gelu_tanh" (its form with the hyperbolic tangent) or "silu" (x / (1 + exp(-x)))."""
    act, codes = _kind(kind), _codes(saved)
    type_ = _check_type(x)
    if _elsewhere(x):
        with torch.cuda.device(x.get_device()):
            return _activate(x, None, act, codes, 0, type_)
    return _activate(x, None, act, codes, 0, type_)


def gated(gate, up=None, kind="silu", saved="codes"):
    """act(gate) * up, of two tensors of one shape and type, or of the halves of one [..., 2 * cols], the gate's first.  Gradients reach both, or the one."""
    act, codes = _kind(kind), _codes(saved)
    type_ = _check_type(gate)
    if up is None:
        if gate.shape[-1] % 2:
            raise ValueError(f"two halves are needed, the last dimension is {gate.shape[-1]}")
    else:
        if up.shape != gate.shape or up.dtype != gate.dtype:
            raise ValueError(f"gate and up must be alike, not {gate.dtype} {tuple(gate.shape)} and {up.dtype} {tuple(up.shape)}")
        if up.get_device() != gate.get_device():
            raise ValueError("gate and up must be on one device")
    how = 2 if up is None else 1
    if _elsewhere(gate):
        with torch.cuda.device(gate.get_device()):
            return _activate(gate, up, act, codes, how, type_)
    return _activate(gate, up, act, codes, how, type_)


# ---------------------------------------------------------------- products
def _operand(x):
    """As a product takes it: rows with adjacent values, not too far apart."""
    x = _flat(x)
    return x if x.stride(0) < _STRIDE_MOST or x.shape[0] <= 1 else x.contiguous()


def _linear(x, rows, w, bias, residual, act, kind, bkind, which, pre, pre8):
    m, k = rows.shape
    n = w.shape[0]
    y = torch.empty((*x.shape[:-1], n), dtype=x.dtype, device=x.device)
    room = _room(_linear_room(which, m, n, k), x.device)
    _call("linear", kind, act, rows.data_ptr(), _stride(rows), w.data_ptr(), _stride(w), m, n, k, bkind, _at(bias), *_place(residual), y.data_ptr(), n, _at(pre), n, *_bytes(pre8),
          *_bytes(room), _stream_of(x))
    return y


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, residual, act, codes, kind, bkind):
        rows, w = _operand(x), _operand(weight)
        m, n = rows.shape[0], w.shape[0]
        need_x, need_w, need_b = ctx.needs_input_grad[:3]
        pre = pre8 = x8 = None
        which = LINEAR_SERVED
        if act != ACT_NONE and (need_x or need_w or need_b):
            which = LINEAR_TRAINED
            pre, pre8 = (None, _blob(m, n, x.device)) if codes else (torch.empty((m, n), dtype=x.dtype, device=x.device), None)
        y = _linear(x, rows, w, _adjacent(bias), None if residual is None else _flat(residual), act, kind, bkind, which, pre, pre8)
        if need_w and codes:
            x8 = _compressed(rows, kind, _stream_of(x))
        ctx.save_for_backward(x if need_w and not codes else None, x8, weight if need_x else None, pre, pre8)
        ctx.how = act, kind, bkind, x.shape
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, x8, weight, pre, pre8 = ctx.saved_tensors
        act, kind, bkind, shape = ctx.how
        need_x, need_w, need_b, need_r = ctx.needs_input_grad[:4]
        dpre = _operand(dy)
        m, n = dpre.shape
        k = shape[-1]
        device, stream = dy.device, _stream_of(dy)
        dx = dw = db = None
        if need_b:
            db = torch.empty(n, dtype=torch.float32 if bkind == MX4_F32 else dy.dtype, device=device)
        if need_b or (act != ACT_NONE and (need_x or need_w)):
            rows = dpre
            dpre = torch.empty((m, n), dtype=dy.dtype, device=device) if act != ACT_NONE else rows
            room = _room(_columns_room(m, n), device) if need_b else None
            _call("linear_columns", kind, act, rows.data_ptr(), _stride(rows), m, n, _at(pre), n, *_bytes(pre8), dpre.data_ptr() if act != ACT_NONE else None, n, bkind, _at(db), *_bytes(room),
                  stream)
        if need_x:
            dx = torch.empty(shape, dtype=dy.dtype, device=device)
            w = _operand(weight)
            _call("linear_rows_gradient", kind, *_place(dpre), *_place(w), m, n, k, dx.data_ptr(), k, *_bytes(_room(_linear_room(LINEAR_ROWS_GRADIENT, m, n, k), device)), stream)
        if need_w:
            dw = torch.empty((n, k), dtype=dy.dtype, device=device)
            x = None if x is None else _operand(x)
            _call("linear_weight_gradient", kind, *_place(dpre), *_place(x), *_bytes(x8), m, n, k, dw.data_ptr(), k, *_bytes(_room(_linear_room(LINEAR_WEIGHT_GRADIENT, m, n, k), device)), stream)
        return dx, dw, db, dy if need_r else None, None, None, None, None


def linear(x, weight, bias=None, activation=None, residual=None, saved="codes"):
    """act(x [..., k] weight [n, k]^T + bias [n]) + residual [..., n], in one pass; sums in binary32, rounded once.

    x, weight and residual: bfloat16 or float16, all of one type; bias: of that type or float32.  activation: None, "gelu", "gelu_tanh" or "silu".  Gradients reach x, weight, bias
    and residual.  saved="codes": x (for the weight's gradient) and what the activation is given are kept in 8 bits; "input": in x's type, finite values beyond its range as its largest.
    The gradient of what the activation is given is rounded to x's type, as the products take it that make those of x and weight; the bias's is its sum before that."""
    act, codes = ACT_NONE if activation is None else _kind(activation), _codes(saved)
    kind = bkind = _check_type(x, MX4_F16)
    shape = weight.shape
    if len(shape) != 2 or shape[1] != x.shape[-1]:
        raise ValueError(f"rows of {x.shape[-1]} values do not fit a weight of shape {tuple(shape)}")
    if weight.dtype != x.dtype:
        raise TypeError(f"x and weight must be of one type, not {x.dtype} and {weight.dtype}")
    at = x.get_device()
    if weight.get_device() != at:
        raise ValueError("the weight must be on the device of the rows")
    if bias is not None:
        bkind = _check_vector(bias, "bias", shape[0], x)
    if residual is not None:
        if residual.shape != (*x.shape[:-1], shape[0]) or residual.dtype != x.dtype:
            raise ValueError(f"residual must be {x.dtype} of shape {(*x.shape[:-1], shape[0])}, not {residual.dtype} of {tuple(residual.shape)}")
        if residual.get_device() != at:
            raise ValueError("residual must be on the device of the rows")
    if _elsewhere(x):
        with torch.cuda.device(at):
            return linear(x, weight, bias, activation, residual, saved)
    if _differentiable(x, weight, bias, residual):
        if shape[0] >= _STRIDE_MOST and (x.requires_grad or weight.requires_grad) and x.shape[:-1].numel() > 1:
            raise ValueError(f"gradients of rows and weight are products of the result's gradient, whose rows must be fewer than {_STRIDE_MOST} values long, not {shape[0]}")
        return _Linear.apply(x, weight, bias, residual, act, codes, kind, bkind)
    return _linear(x, _operand(x), _operand(weight), _adjacent(bias), None if residual is None else _flat(residual), act, kind, bkind, LINEAR_SERVED, None, None)

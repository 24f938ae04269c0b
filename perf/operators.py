"""perf/operators.py: matrices in microscaled 4-bit floating point and their products, as cases that can be timed and compared.

Four families.  "restore": a tensor is compressed to 4-bit codes with one power of two per 32 values and restored, as a saved activation is between
the forward and the backward pass.  "linear": rows of 16 or 32 bits times a weight that is kept in that form.  "linear_step" / "experts_step": a layer's
forward and backward pass, with gradients of the rows and of the weight.  "experts": the linear layer of a mixture of experts, rows sorted by expert, any
number of them for each.  Widths are those of the benchmark's activations (1024, 2048, 4096, 11008, 16384) or generic ones; inputs are drawn from the
seed, on the GPU.

Plain forms: a block of 32 values is divided by its power of two, rounded to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and multiplied back, all in binary32;
products are binary32 products of such values, rounded once to the output's type.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BLOCK = 32
MOST_FLOPS = 2 * 16384 * 4096 * 11008  # of the largest listed case


# ---------------------------------------------------------------------------- the cases
def listed():
    return [
        # one token's hidden state of 2048 values: what a decoding step saves or sends; latency is all there is
        dict(name="restore_one_token", kind="restore", rows=1, cols=2048, dtype="bf16", rule="floor", both=False),
        # a layer's hidden states, blocks along the rows and along the tokens at once, as a training step keeps them
        dict(name="restore_hidden_both", kind="restore", rows=32768, cols=2048, dtype="bf16", rule="floor", both=True),
        # MLP activations, FP16, one token short of a round number; nothing is clipped
        dict(name="restore_mlp_fp16", kind="restore", rows=8191, cols=11008, dtype="f16", rule="fullrange", both=False),
        # binary32 master weights with odd sides, both directions
        dict(name="restore_odd_f32", kind="restore", rows=1999, cols=4093, dtype="f32", rule="fullrange", both=True),
        # a decoding step of one sequence: the weight is read once
        dict(name="linear_one_token", kind="linear", rows=1, cols=4096, out=11008, dtype="bf16"),
        # a decoding step of 16 sequences, down projection
        dict(name="linear_16_tokens", kind="linear", rows=16, cols=11008, out=4096, dtype="bf16"),
        # a short prompt, FP16, sides that no tile divides
        dict(name="linear_odd_fp16", kind="linear", rows=777, cols=2040, out=1003, dtype="f16"),
        # a prompt batch through the up projection
        dict(name="linear_prompt", kind="linear", rows=16384, cols=4096, out=11008, dtype="bf16"),
        # forward and backward pass of an MLP's up projection over 8192 tokens
        dict(name="linear_step", kind="linear_step", rows=8192, cols=2048, out=8192, dtype="bf16", weight="bf16"),
        # a decoding step of 32 sequences, two of 32 experts each: most experts see a few rows, some none
        dict(name="experts_decode", kind="experts", rows=64, cols=2048, out=2048, experts=32, skew=0.5, dtype="bf16"),
        # a prompt of 8192 tokens, two of 16 experts each, unevenly
        dict(name="experts_prompt", kind="experts", rows=16384, cols=2048, out=4096, experts=16, skew=1.0, dtype="bf16"),
        # forward and backward pass of the experts' down projection; binary32 master weights, so their gradients are binary32
        dict(name="experts_step", kind="experts_step", rows=8192, cols=4096, out=1024, experts=8, skew=0.7, dtype="bf16", weight="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Half of the widths are round, the others anything."""
    w = _log(rng, lo, hi)
    return max(lo, w // 128 * 128) if rng.random() < 0.5 else w


def draw(rng):
    kind = rng.choice(["restore", "restore", "linear", "linear", "linear_step", "experts", "experts", "experts_step"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "restore":
        cols = _width(rng, 64, 16384)
        rows = _log(rng, 1, min(32768, (1 << 26) // cols))
        return dict(kind=kind, rows=rows, cols=cols, dtype=dtype, rule=rng.choice(["floor", "fullrange"]), both=rng.random() < 0.5)
    if kind == "linear":
        cols, out = _width(rng, 256, 11008), _width(rng, 256, 11008)
        rows = _log(rng, 1, 64) if rng.random() < 0.5 else _log(rng, 65, min(16384, MOST_FLOPS // (2 * cols * out)))
        return dict(kind=kind, rows=rows, cols=cols, out=out, dtype=dtype)
    if kind == "linear_step":
        cols, out = _width(rng, 256, 4096), _width(rng, 256, 8192)
        return dict(kind=kind, rows=_log(rng, 64, min(8192, MOST_FLOPS // (6 * cols * out))), cols=cols, out=out, dtype=rng.choice(["bf16", "f16"]),
                    weight=rng.choice(["same", "f32"]))
    experts = rng.choice([2, 5, 8, 16, 32, 64])
    cols, out = _width(rng, 256, 4096), _width(rng, 256, 4096)
    if kind == "experts":
        rows = _log(rng, 1, 128) if rng.random() < 0.5 else _log(rng, 129, 16384)
        return dict(kind=kind, rows=rows, cols=cols, out=out, experts=experts, skew=rng.choice([0.0, 0.7, 1.5]), dtype=dtype)
    return dict(kind=kind, rows=_log(rng, 64, 8192), cols=cols // 2, out=out // 2, experts=experts, skew=rng.choice([0.0, 0.7, 1.5]),
                dtype=rng.choice(["bf16", "f16"]), weight=rng.choice(["same", "f32"]))


# ---------------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _activations(rows, cols, g, dtype):
    """N(0, 1.5); one channel in 200 is twenty times as large, as hidden states have them."""
    x = torch.randn((rows, cols), generator=g, device="cuda")
    big = torch.rand(cols, generator=g, device="cuda") < 0.005
    return (x * torch.where(big, 30.0, 1.5)).to(dtype)


def _sizes(case, g):
    """How many rows each expert has: shares exp(skew * N(0, 1)), every row drawn by them."""
    share = torch.softmax(case["skew"] * torch.randn(case["experts"], generator=g, device="cuda"), 0)
    pick = torch.multinomial(share, case["rows"], replacement=True, generator=g)
    return torch.bincount(pick, minlength=case["experts"]).tolist()


def _inputs(case, seed):
    g = _gen(seed)
    dtype = DTYPES[case["dtype"]]
    s = dict(case=case, dtype=dtype)
    kind, rows, cols = case["kind"], case["rows"], case["cols"]
    s["x"] = _activations(rows, cols, g, dtype)
    if kind == "restore":
        return s
    lead = ()
    if kind.startswith("experts"):
        s["sizes"] = _sizes(case, g)
        ends = [0]
        for n in s["sizes"]:
            ends.append(ends[-1] + n)
        s["offsets"] = torch.tensor(ends, dtype=torch.int32, device="cuda")
        lead = (case["experts"],)
    out = case["out"]
    s["w"] = (torch.randn((*lead, out, cols), generator=g, device="cuda") * (1.0 / math.sqrt(cols))).to(DTYPES.get(case.get("weight"), dtype))
    if kind.endswith("_step"):
        scale = torch.exp(torch.randn((rows, 1), generator=g, device="cuda")) * 1e-2
        s["dy"] = (torch.randn((rows, out), generator=g, device="cuda") * scale).to(dtype)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["kind"].endswith("_step"):
        if own:
            s["x"].requires_grad_()
            s["w"].requires_grad_()
    elif "w" in s:  # a serving program keeps its weights in the form that the product reads
        w = s.pop("w")
        if own:
            from paper_2508_00806_amd import mx4
            s["weight"] = mx4.compress(w)
        else:
            s["weight"] = _rounded(w)
    return s


# ---------------------------------------------------------------------------- one pass
def _rounded(x, rule="floor"):
    """Blocks of 32 along the last dimension, divided by their power of two, rounded to 4-bit floating point and multiplied back: binary32."""
    cols = x.shape[-1]
    short = -cols % BLOCK
    x = x.float()
    if short:
        x = torch.cat([x, x.new_zeros((*x.shape[:-1], short))], -1)
    x = x.reshape(*x.shape[:-1], -1, BLOCK)
    most = x.abs().amax(-1, keepdim=True)
    mant, exp = torch.frexp(most)  # most = mant * 2^exp, 0.5 <= mant < 1
    e = exp - 3
    if rule == "fullrange":
        e = e + (mant > 0.75)
    e = torch.where(most > 0, e, 0).clamp(min=-127)
    v = torch.ldexp(x, -e)
    a = v.abs()
    # the codes are 0.5 apart up to 2, 1 apart up to 4, 2 apart beyond; round() takes ties to the even multiple
    a = torch.where(a < 2, (a * 2).round() / 2, torch.where(a < 4, a.round(), (a / 2).round() * 2)).clamp(max=6)
    back = torch.ldexp(torch.copysign(a, v), e)
    return back.reshape(*back.shape[:-2], -1)[..., :cols]


def _across(x, rule="floor"):
    """The same with blocks along the last dimension but one."""
    return _rounded(x.transpose(-1, -2).contiguous(), rule)


def _plain(s):
    case, x = s["case"], s["x"]
    kind, dtype = case["kind"], s["dtype"]
    if kind == "restore":
        y = _rounded(x, case["rule"]).to(dtype)
        return [y, _across(x, case["rule"]).to(dtype)] if case["both"] else [y]
    if kind == "linear":
        return [(_rounded(x) @ s["weight"].t()).to(dtype)]
    if kind == "linear_step":
        w, dy = s["w"], s["dy"]
        y = _rounded(x) @ _rounded(w).t()
        dx = _rounded(dy) @ _across(w).t()
        dw = _across(dy) @ _across(x).t()
        return [y.to(dtype), dx.to(dtype), dw.to(w.dtype)]
    y = torch.empty((case["rows"], case["out"]), dtype=dtype, device=x.device)
    xr = _rounded(x)
    at = 0
    if kind == "experts":
        for e, n in enumerate(s["sizes"]):
            y[at:at + n] = (xr[at:at + n] @ s["weight"][e].t()).to(dtype)
            at += n
        return [y]
    w, dy = s["w"], s["dy"]
    wr, wa, dyr = _rounded(w), _across(w), _rounded(dy)
    dx = torch.empty_like(x)
    dw = torch.zeros_like(w)
    for e, n in enumerate(s["sizes"]):
        if n == 0:
            continue
        y[at:at + n] = (xr[at:at + n] @ wr[e].t()).to(dtype)
        dx[at:at + n] = (dyr[at:at + n] @ wa[e].t()).to(dtype)
        dw[e] = (_across(dy[at:at + n]) @ _across(x[at:at + n]).t()).to(w.dtype)
        at += n
    return [y, dx, dw]


def _own(s):
    from paper_2508_00806_amd import mx4
    case, x = s["case"], s["x"]
    kind = case["kind"]
    if kind == "restore":
        if not case["both"]:
            return [mx4.compress(x, scale_rule=case["rule"]).restore(x.dtype)]
        along, across = mx4.compress_both(x, scale_rule=case["rule"])
        return [along.restore(x.dtype), across.restore(x.dtype)]
    if kind == "linear":
        return [mx4.linear(x, s["weight"])]
    if kind == "experts":
        return [mx4.experts(x, s["offsets"], s["weight"])]
    if kind == "linear_step":
        y = mx4.linear(x, s["w"])
    else:
        y = mx4.experts(x, s["offsets"], s["w"])
    dx, dw = torch.autograd.grad(y, (x, s["w"]), s["dy"])
    return [y.detach(), dx, dw]


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------- what a pass can not do without
def _size(dtype):
    return 4 if dtype == "f32" else 2


def _packed(rows, cols):
    """Bytes of a compressed matrix: half a byte a value and one a block."""
    return rows * (-(-cols // 2) + -(-cols // BLOCK))


def work(case):
    kind, rows, cols = case["kind"], case["rows"], case["cols"]
    size = _size(case["dtype"])
    if kind == "restore":
        # two calls: one reads the tensor and writes the blobs, the other reads the blobs and writes tensors
        n = rows * cols
        ways = [_packed(rows, cols)] + ([_packed(cols, rows)] if case["both"] else [])
        return {"bytes": n * size + sum(2 * p + n * size for p in ways), "flops": 0}
    out = case["out"]
    experts = case.get("experts", 1)
    # experts with at least one row, whose weights are read (at most; an uneven draw has fewer)
    live = min(experts, rows)
    if kind in ("linear", "experts"):
        return {"bytes": rows * cols * size + live * _packed(out, cols) + rows * out * size, "flops": 2 * rows * cols * out}
    wsize = 4 if case["weight"] == "f32" else size
    # x, dy and the weight are read; y, dx and the weight's gradient are written
    return {"bytes": 2 * rows * (cols + out) * size + (live + experts) * cols * out * wsize, "flops": 6 * rows * cols * out}


# ---------------------------------------------------------------------------- the definition in 64 bits
_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_rounded(x, rule):
    """Blocks along the rows of a matrix, one block of columns after the other: the block's power of two from its logarithm, made
    sure of by comparison; every value's code by counting the borders that it passes."""
    x = x.double()
    out = torch.empty_like(x)
    grid = torch.tensor(_GRID, dtype=torch.float64, device=x.device)
    border = (grid[1:] + grid[:-1]) / 2
    rows, cols = x.shape
    step = max(BLOCK, (1 << 24) // max(rows, 1) // BLOCK * BLOCK)
    for c0 in range(0, cols, step):
        part = x[:, c0:c0 + step]
        n = part.shape[1]
        room = torch.zeros((rows, -(-n // BLOCK) * BLOCK), dtype=torch.float64, device=x.device)
        room[:, :n] = part
        b = room.view(rows, -1, BLOCK)
        a = b.abs()
        top = a.max(-1, keepdim=True).values
        e = torch.floor(torch.log2(top.clamp(min=2.0 ** -160)))
        e = e - (torch.exp2(e) > top).double() + (torch.exp2(e + 1) <= top).double()
        e = e - 2
        if rule == "fullrange":
            e = e + (top > 6 * torch.exp2(e)).double()
        unit = torch.exp2(e.clamp(min=-127))
        ratio = a / unit
        code = torch.zeros_like(ratio, dtype=torch.int64)
        for i in range(7):  # on a border the even code has it: border i lies between codes i and i + 1
            code += (ratio >= border[i]) if i % 2 else (ratio > border[i])
        out[:, c0:c0 + n] = (grid[code] * unit * torch.sign(b)).view(rows, -1)[:, :n]
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    kind, x = case["kind"], s["x"]
    if kind == "restore":
        outs = [_exact_rounded(x, case["rule"])]
        if case["both"]:
            outs.append(_exact_rounded(x.t(), case["rule"]))
        return outs
    step = kind.endswith("_step")
    weights, sizes = (s["w"][None], [case["rows"]]) if kind.startswith("linear") else (s["w"], s["sizes"])
    y = torch.zeros((case["rows"], case["out"]), dtype=torch.float64, device="cuda")
    dx = torch.zeros(x.shape, dtype=torch.float64, device="cuda") if step else None
    dw = torch.zeros(weights.shape, dtype=torch.float64, device="cuda") if step else None
    first = 0
    for i, n in enumerate(sizes):
        last = first + n
        if n:
            y[first:last] = torch.mm(_exact_rounded(x[first:last], "floor"), _exact_rounded(weights[i], "floor").t())
            if step:
                dy = s["dy"][first:last]
                dx[first:last] = torch.mm(_exact_rounded(dy, "floor"), _exact_rounded(weights[i].t(), "floor").t())
                dw[i] = torch.mm(_exact_rounded(dy.t(), "floor"), _exact_rounded(x[first:last].t(), "floor").t())
        first = last
    if not step:
        return [y]
    return [y, dx, dw[0] if kind.startswith("linear") else dw]

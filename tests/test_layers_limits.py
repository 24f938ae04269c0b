"""Calls at the limits of the layers' sizes, and what the layers and their binding refuse; no GPU is needed.  What is taken would be launched, on addresses that do not exist: without a GPU the launch
fails, with one those tests are skipped."""
import pytest
import torch

import paper_2508_00806_amd as adacc
from paper_2508_00806_amd import layers
from test_layers_host import BIG, CALLS, P

EHIP, ELIMIT = adacc.EHIP, adacc.ELIMIT
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="the call would be launched")


def call(name, **change):
    return getattr(adacc.lib(), "adacc_" + name)(*{**CALLS[name], **change}.values())


@no_gpu
@pytest.mark.parametrize("cols", [1 << 27, (1 << 28) + 1, 1 << 30])
def test_sums_of_columns_of_any_number_are_taken(cols):
    """(Of no rows: the sums' launch is the only one.)"""
    assert call("norm_backward", rows=0, cols=cols, dx=None) == EHIP
    assert call("norm_backward", rows=0, cols=cols, dx=None, dweight=None) == EHIP
    assert call("linear_columns", m=0, n=cols) == EHIP


def test_the_first_launch_of_many_wide_rows_is_taken():
    """A workgroup for 2048 columns of each of the partial sums, fewer than 2^32 threads in all."""
    for rows, cols in ((32, 1 << 30), (64, 1 << 29), (1 << 20, (1 << 30) - 5)):
        partials = adacc.norm_workspace_bytes(rows, cols) // (8 * cols)
        assert 1 <= partials <= 64 and partials * -(-cols // 2048) * 256 < 1 << 32


@no_gpu
@pytest.mark.parametrize("rows,cols", [(1 << 30, 1), (1 << 29, 200), ((1 << 30) - 3, 100), (1, 1 << 30)])
def test_as_many_groups_as_the_limit_says_are_taken(rows, cols):
    given = dict(rows=rows, cols=cols)
    assert call("rows8_compress", stride=cols, **given) == EHIP
    assert call("rows8_decompress", stride=cols, **given) == EHIP
    assert call("act_forward", a_stride=cols, up_stride=cols, y_stride=cols, **given) == EHIP
    assert call("act_backward", dy_stride=cols, da_stride=cols, dup_stride=cols, **given) == EHIP


@pytest.mark.parametrize("rows,cols", [(1 << 30, 129), ((1 << 23) + 1, 128 * 128)])
def test_more_groups_are_refused(rows, cols):
    given = dict(rows=rows, cols=cols)
    assert call("rows8_compress", stride=cols, **given) == call("rows8_decompress", stride=cols, **given) == ELIMIT
    assert call("act_forward", a_stride=cols, up_stride=cols, y_stride=cols, **given) == ELIMIT
    assert call("act_backward", dy_stride=cols, da_stride=cols, dup_stride=cols, **given) == ELIMIT


@no_gpu
@pytest.mark.parametrize("k", [1 << 23, 1 << 30])
def test_a_weights_gradient_from_one_row_of_any_length_is_taken(k):
    """From codes as from the row itself: no other row lies behind it."""
    wide = dict(m=1, n=1, k=k, d_stride=1, dw_stride=k)
    assert call("linear_weight_gradient", **wide) == call("linear_weight_gradient", x=P, x_stride=k, x_blob=None, **wide) == EHIP


@no_gpu
@pytest.mark.parametrize("n", [(1 << 30) - 15, 1 << 30])
@pytest.mark.parametrize("m", [1, 17])
def test_few_rows_by_as_many_as_there_may_be_are_taken(m, n):
    given = dict(m=m, n=n, k=8, x_stride=8, w_stride=8, r_stride=n, y_stride=n, pre_blob=None)
    assert call("linear", **given) == EHIP


def test_more_tiles_than_are_counted_are_refused_ahead_of_every_launch():
    """(Rows of fewer than eight values are copied first: with a GPU, that launch would not refuse.)"""
    assert call("linear", m=1 << 30, n=1 << 30, k=5, x_stride=5, w_stride=5, r_stride=1 << 30, y_stride=1 << 30, pre_blob=None, kind=0) == ELIMIT


# ---------------------------------------------------------------- the layers
@pytest.fixture
def calls(monkeypatch):
    """Names of the library's functions that would have been called, with tensors in host memory."""
    seen = []
    monkeypatch.setattr(layers, "_on_gpu", lambda x: None)
    monkeypatch.setattr(layers, "_stream_of", lambda x: 0)
    monkeypatch.setattr(layers, "_call", lambda name, *args: seen.append(name))
    return seen


def t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def test_a_forward_pass_whose_gradients_would_be_refused_is_refused(calls):
    """The result's gradient is an operand of both products of the backward pass, and its rows lie apart as far as they are long."""
    n = 1 << 23
    for x, w in ((t(2, 8).requires_grad_(), t(1, 8).expand(n, 8)), (t(2, 8), t(1, 8).requires_grad_().expand(n, 8)), (t(2, 1, 8).requires_grad_(), t(1, 8).expand(n, 8))):
        with pytest.raises(ValueError, match="fewer than"):
            layers.linear(x, w)
    assert calls == []
    x, w = t(2, 8).requires_grad_(), t(1, 8).expand(n, 8)
    with torch.no_grad():
        layers.linear(x, w)
    layers.linear(x[:1], w)                                 # one row: nothing lies apart
    layers.linear(x, w[1:])
    y = layers.linear(x.detach(), w, t(n).requires_grad_())  # sums of columns have no such limit
    y.backward(y)
    assert calls == ["linear"] * 4 + ["linear_columns"]


def test_codes_that_were_moved_to_host_memory_are_not_restored_there(monkeypatch):
    seen = []
    monkeypatch.setattr(layers, "_stream_of", lambda x: 0)
    monkeypatch.setattr(layers, "_call", lambda name, *args: seen.append(name))
    kept = layers.Rows8(t(2048, dtype=torch.uint8), (6, 64))
    with pytest.raises(ValueError, match="GPU"):
        kept.restore()
    assert seen == []


@pytest.mark.filterwarnings("ignore")
@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("call", [lambda x: layers.layer_norm(x), lambda x: layers.activation(x), lambda x: layers.gated(x), lambda x: layers.linear(x, x),
                                  lambda x: (x, layers.compress(x))[0], lambda x: layers.Rows8(t(8, dtype=torch.uint8), (6, 64)).restore() + x],
                         ids=["layer_norm", "activation", "gated", "linear", "compress", "restore"])
def test_a_trace_that_is_recorded_is_refused_in_words(calls, call, grad):
    """The library's call is none of torch's operators: what was recorded would give back memory that nothing has written."""
    with pytest.raises(RuntimeError, match="torch.jit.trace"):
        torch.jit.trace(call, (t(6, 64).requires_grad_(grad),))
    assert calls == []


# ---------------------------------------------------------------- the binding
@pytest.mark.parametrize("stats", [t(6, 2, dtype=torch.float32), t(7, dtype=torch.float32), t(14, dtype=torch.float32), t(7, 2), t(2, 7, dtype=torch.float32).t(), t(7, 3, dtype=torch.float32)[:, :2],
                                   t(7, 2, dtype=torch.float64)], ids=range(7))
def test_statistics_that_are_not_two_numbers_a_row_are_refused(monkeypatch, stats):
    def reached(*args):
        raise AssertionError("the library was reached")
    monkeypatch.setattr(adacc, "_layer", lambda name: reached)
    monkeypatch.setattr(adacc, "_stream", lambda s: 0)
    for call in (lambda: adacc.norm_forward(t(7, 8), None, None, 1e-5, t(7, 8), stats=stats), lambda: adacc.norm_backward(t(7, 8), None, None, stats, t(7, 8), dx=t(7, 8))):
        with pytest.raises((ValueError, TypeError)):
            call()


def test_statistics_reach_the_library(monkeypatch):
    seen = []
    monkeypatch.setattr(adacc, "_layer", lambda name: lambda *args: seen.append(args) or 0)
    monkeypatch.setattr(adacc, "_stream", lambda s: 0)
    stats = t(7, 2, dtype=torch.float32)
    adacc.norm_forward(t(7, 8), None, None, 1e-5, t(7, 8), stats=stats)
    adacc.norm_forward(t(7, 8), None, None, 1e-5, t(7, 8))
    adacc.norm_backward(t(7, 8), None, None, stats, t(7, 8), dx=t(7, 8))
    assert seen[0][13] == stats.data_ptr() and seen[1][13] is None and seen[2][9] == stats.data_ptr()

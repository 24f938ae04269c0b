"""mx4.linear and mx4.experts with a kept weight: what becomes of a gradient that is asked for.  Without a GPU: the product itself is left out."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2508_00806_amd import mx4


@pytest.fixture(params=["linear", "experts"])
def serve(request, monkeypatch):
    monkeypatch.setattr(mx4, "_on_gpu", lambda t: None)
    monkeypatch.setattr(mx4, "_stream_of", lambda t: 0)
    monkeypatch.setattr(mx4, "mx4_linear", lambda x, b, out, **k: out.fill_(2.0))
    blob = torch.zeros(8, dtype=torch.uint8)
    if request.param == "linear":
        return lambda x: mx4.linear(x, mx4.Mx4Matrix(blob, (5, 64)))
    offsets = torch.zeros(3, dtype=torch.int32)
    return lambda x: mx4.experts(x, offsets, mx4.Mx4Matrix(blob, (2, 5, 64)))


def test_a_gradient_through_a_kept_weight_is_refused(serve):
    """The rows have another way to the loss: without it there would be an error, with it a gradient that lacks a part."""
    x = torch.ones(6, 64, requires_grad=True)
    y = serve(x)
    assert y.shape == (6, 5) and (y == 2.0).all()
    with pytest.raises(RuntimeError, match="Mx4Matrix has no gradient"):
        (y.sum() + x.sum()).backward()
    assert x.grad is None


def test_serving_asks_for_none(serve):
    x = torch.ones(6, 64, requires_grad=True)
    with torch.no_grad():
        assert not serve(x).requires_grad
    with torch.inference_mode():
        assert not serve(x).requires_grad
    assert not serve(x.detach()).requires_grad
    (serve(x.detach()).sum() + x.sum()).backward()
    assert (x.grad == 1.0).all()


def test_a_tangent_through_a_kept_weight_is_refused(serve):
    with forward_ad.dual_level():
        assert (serve(torch.ones(6, 64)) == 2.0).all()
        with pytest.raises((RuntimeError, NotImplementedError)):
            serve(forward_ad.make_dual(torch.ones(6, 64), torch.ones(6, 64)))

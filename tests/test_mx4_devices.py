"""mx4: which device is current while the library is called, without a GPU (tensors in host memory say that they are on device 1)."""
import pytest
import torch

from paper_2508_00806_amd import mx4


@pytest.fixture
def calls(monkeypatch):
    """[(name of the library's function, current device)], with device 0 current at first."""
    current, seen = [0], []

    class Device:
        def __init__(self, at):
            self.at = at

        def __enter__(self):
            self.before, current[0] = current[0], self.at

        def __exit__(self, *error):
            current[0] = self.before

    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 1)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[0])
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(mx4, "_on_gpu", lambda t: None)
    monkeypatch.setattr(mx4, "_stream_of", lambda t: 0)
    for name in ("mx4_compress", "mx4_decompress", "mx4_product", "mx4_linear"):
        monkeypatch.setattr(mx4, name, lambda *a, _name=name, **k: seen.append((_name, current[0])))
    yield seen
    assert current == [0]


X, W, E = torch.zeros(6, 64), torch.zeros(5, 64), torch.zeros(2, 5, 64)
OFFSETS = torch.zeros(3, dtype=torch.int32)


@pytest.mark.parametrize("call,names", [
    (lambda: mx4.compress(X), ["mx4_compress"]),
    (lambda: mx4.compress_both(X, "fullrange"), ["mx4_compress"]),
    (lambda: mx4.Mx4Matrix(torch.zeros(8, dtype=torch.uint8), (6, 64)).restore(torch.float16), ["mx4_decompress"]),
    (lambda: mx4.linear(X, mx4.Mx4Matrix(torch.zeros(8, dtype=torch.uint8), (5, 64))), ["mx4_linear"]),
    (lambda: mx4.linear(X, W, torch.float16), ["mx4_compress", "mx4_compress", "mx4_product"]),
    (lambda: mx4.experts(X, OFFSETS, mx4.Mx4Matrix(torch.zeros(8, dtype=torch.uint8), (2, 5, 64))), ["mx4_linear"]),
    (lambda: mx4.experts(X, OFFSETS, E), ["mx4_compress", "mx4_compress", "mx4_product"])], ids=range(7))
def test_the_tensors_device_is_current(calls, call, names):
    call()
    assert calls == [(name, 1) for name in names]


def test_a_current_device_stays_as_it_is(calls, monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    monkeypatch.setattr(torch.cuda, "device", None)
    mx4.compress(X)
    mx4.linear(X, W)
    assert len(calls) == 4


@pytest.mark.parametrize("blob,out", [("cpu", None), ("cpu", "cpu"), ("meta", "meta")])
def test_a_matrix_that_is_not_on_a_gpu_is_not_restored(blob, out, monkeypatch):
    monkeypatch.setattr(mx4, "_stream_of", lambda t: 0)
    monkeypatch.setattr(mx4, "mx4_decompress", None)  # (no call)
    m = mx4.Mx4Matrix(torch.zeros(8, dtype=torch.uint8, device=blob), (6, 64))
    with pytest.raises(ValueError, match="on a GPU"):
        m.restore(out=None if out is None else torch.zeros(6, 64, device=out))


def test_a_matrix_is_restored_on_its_own_device_only(calls):
    """An address in host memory, or on another device, would reach the kernel."""
    m = mx4.Mx4Matrix(torch.zeros(8, dtype=torch.uint8), (6, 64))
    with pytest.raises(ValueError, match="out is on meta"):
        m.restore(out=torch.zeros(6, 64, device="meta"))
    assert calls == []

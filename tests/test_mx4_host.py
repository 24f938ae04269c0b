"""adacc_mx4_*: layouts, sizes and refusals, which need no GPU (the addresses are never touched)."""
import ctypes

import pytest
import torch

import paper_2508_00806_amd as adacc
from paper_2508_00806_amd import mx4

P = 1 << 20  # an aligned address
BIG = 1 << 40


@pytest.fixture(scope="module")
def L():
    return adacc.lib()


def a256(v):
    return -(-v // 256) * 256


def test_layout_closed_form(L):
    assert ctypes.sizeof(adacc.CMx4Layout) == 40
    for rows, cols in ((1, 1), (3, 128), (16, 129), (17, 4096), (1000, 2040), (0, 5), (5, 0)):
        lay = adacc.mx4_layout_of(rows, cols)
        steps = -(-cols // 128)
        assert lay.step_bytes == 64 * rows and lay.scale_pitch == -(-rows // 16) * 16
        assert lay.codes_off == 0 and lay.scales_off == a256(rows * 64 * steps)
        assert lay.total_bytes == lay.scales_off + a256(4 * steps * lay.scale_pitch)
    assert L.adacc_mx4_layout_of(1, 1, None) == adacc.ENULL
    assert L.adacc_mx4_layout_of((1 << 30) + 1, 1, ctypes.byref(adacc.CMx4Layout())) == adacc.ELIMIT
    assert L.adacc_mx4_layout_of(1, (1 << 30) + 1, ctypes.byref(adacc.CMx4Layout())) == adacc.ELIMIT


def test_grouped_columns_hold_any_division():
    for rows, groups in ((0, 3), (1, 1), (1, 8), (127, 2), (128, 1), (129, 1), (1000, 7), (5, 64)):
        cap = adacc.mx4_grouped_cols(rows, groups)
        assert cap % 128 == 0
        # the worst division: as many groups as there are rows for, each one row into its last step
        live = min(rows, groups)
        if live:
            worst = [1] * (live - 1) + [rows - (live - 1)]
            assert sum(-(-w // 128) * 128 for w in worst) <= cap
            spread = rows - live
            more = [1 + 128 * (spread // 128 // live)] * (live - 1)
            more.append(rows - sum(more))
            assert sum(-(-w // 128) * 128 for w in more) <= cap
    assert adacc.mx4_grouped_cols((1 << 30) + 1, 1) == 0 and adacc.mx4_grouped_cols(1, 4097) == 0


def compress(L, kind=0, rule=0, src=P, mats=1, rows=100, cols=200, rs=200, ms=0, off=None, groups=0, along=P, ab=BIG, across=P, cb=BIG):
    return L.adacc_mx4_compress(kind, rule, src, mats, rows, cols, rs, ms, off, groups, along, ab, across, cb, None)


def test_compress_refusals(L):
    assert compress(L, kind=3) == adacc.EINVAL
    assert compress(L, rule=2) == adacc.EINVAL
    assert compress(L, rs=199) == adacc.EINVAL
    assert compress(L, mats=2, off=P, groups=2) == adacc.EINVAL
    assert compress(L, off=P) == adacc.EINVAL
    assert compress(L, groups=2) == adacc.ENULL
    assert compress(L, off=P + 2, groups=2) == adacc.EALIGN
    assert compress(L, off=P, groups=4097) == adacc.ELIMIT
    assert compress(L, rows=(1 << 30) + 1) == adacc.ELIMIT
    assert compress(L, mats=1 << 20, rows=1 << 11) == adacc.ELIMIT
    assert compress(L, src=None) == adacc.ENULL
    assert compress(L, along=None, across=None) == adacc.ENULL
    assert compress(L, src=P + 1) == adacc.EALIGN
    assert compress(L, kind=2, src=P + 2) == adacc.EALIGN
    assert compress(L, along=P + 128) == adacc.EALIGN
    assert compress(L, across=P + 128) == adacc.EALIGN
    need = adacc.mx4_layout_of(100, 200).total_bytes
    assert compress(L, ab=need - 1) == adacc.ESIZE
    need = adacc.mx4_layout_of(200, 100).total_bytes
    assert compress(L, cb=need - 1) == adacc.ESIZE
    need = adacc.mx4_layout_of(200, adacc.mx4_grouped_cols(100, 5)).total_bytes
    assert compress(L, off=P, groups=5, cb=need - 1) == adacc.ESIZE
    for empty in (dict(rows=0), dict(cols=0, rs=0), dict(mats=0)):
        assert compress(L, src=None, along=None, across=None, **empty) == adacc.OK


def test_decompress_refusals(L):
    def f(blob=P, nb=BIG, rows=10, cols=20, dst=P, kind=0, rs=20):
        return L.adacc_mx4_decompress(blob, nb, rows, cols, dst, kind, rs, None)
    assert f(kind=3) == adacc.EINVAL and f(rs=19) == adacc.EINVAL
    assert f(rows=(1 << 30) + 1) == adacc.ELIMIT
    assert f(blob=None) == adacc.ENULL and f(dst=None) == adacc.ENULL
    assert f(blob=P + 16) == adacc.EALIGN and f(dst=P + 1) == adacc.EALIGN
    assert f(nb=adacc.mx4_layout_of(10, 20).total_bytes - 1) == adacc.ESIZE
    assert f(rows=0, blob=None, dst=None) == adacc.OK and f(cols=0, rs=0, blob=None, dst=None) == adacc.OK


def test_product_refusals(L):
    def f(a=P, ab=BIG, m=10, b=P, bb=BIG, n=20, k=300, off=None, groups=0, out=P, kind=0, os=20):
        return L.adacc_mx4_product(a, ab, m, b, bb, n, k, off, groups, out, kind, os, None)
    assert f(kind=3) == adacc.EINVAL and f(os=19) == adacc.EINVAL and f(off=P) == adacc.EINVAL
    assert f(groups=3) == adacc.ENULL and f(a=None) == adacc.ENULL and f(b=None) == adacc.ENULL and f(out=None) == adacc.ENULL
    assert f(a=P + 16) == adacc.EALIGN and f(b=P + 16) == adacc.EALIGN and f(out=P + 1) == adacc.EALIGN and f(kind=2, out=P + 2) == adacc.EALIGN
    assert f(k=(1 << 30) + 1) == adacc.ELIMIT and f(m=(1 << 30) + 1) == adacc.ELIMIT and f(off=P, groups=4097) == adacc.ELIMIT
    assert f(off=P, groups=4096, n=1 << 20, os=1 << 20) == adacc.ELIMIT
    assert f(ab=adacc.mx4_layout_of(10, 300).total_bytes - 1) == adacc.ESIZE
    assert f(bb=adacc.mx4_layout_of(20, 300).total_bytes - 1) == adacc.ESIZE
    assert f(off=P, groups=3, bb=adacc.mx4_layout_of(60, 300).total_bytes - 1) == adacc.ESIZE
    assert f(m=0, a=None, b=None, out=None) == adacc.OK and f(n=0, os=0, a=None, b=None, out=None) == adacc.OK


def test_linear_refusals(L):
    def f(kind=0, rule=0, x=P, m=100, xs=300, b=P, bb=BIG, n=20, k=300, off=None, groups=0, out=P, ok=0, os=20, ws=P, wb=BIG):
        return L.adacc_mx4_linear(kind, rule, x, m, xs, b, bb, n, k, off, groups, out, ok, os, ws, wb, None)
    assert f(kind=3) == adacc.EINVAL and f(rule=2) == adacc.EINVAL and f(xs=299) == adacc.EINVAL and f(ok=3) == adacc.EINVAL
    assert f(x=None) == adacc.ENULL and f(b=None) == adacc.ENULL and f(out=None) == adacc.ENULL and f(ws=None) == adacc.ENULL
    assert f(x=P + 1) == adacc.EALIGN and f(ws=P + 16) == adacc.EALIGN
    need = adacc.mx4_linear_workspace_bytes(100, 20, 300)
    assert need == adacc.mx4_layout_of(100, 300).total_bytes
    assert f(wb=need - 1) == adacc.ESIZE
    assert f(m=0, x=None, b=None, out=None, ws=None) == adacc.OK
    assert adacc.mx4_linear_workspace_bytes(0, 20, 300) == 0


def test_gradient_refusals(L):
    def f(a=P, ab=BIG, m=10, b=P, bb=BIG, n=20, rows=500, off=P, groups=3, out=P, kind=0, os=20):
        return L.adacc_mx4_gradient(a, ab, m, b, bb, n, rows, off, groups, out, kind, os, None)
    assert f(kind=3) == adacc.EINVAL and f(os=19) == adacc.EINVAL and f(groups=0) == adacc.EINVAL
    assert f(off=None) == adacc.ENULL and f(a=None) == adacc.ENULL and f(b=None) == adacc.ENULL and f(out=None) == adacc.ENULL
    assert f(a=P + 16) == adacc.EALIGN and f(off=P + 1) == adacc.EALIGN
    assert f(rows=(1 << 30) + 1) == adacc.ELIMIT and f(groups=4097) == adacc.ELIMIT
    need = adacc.mx4_layout_of(10, adacc.mx4_grouped_cols(500, 3)).total_bytes
    assert f(ab=need - 1) == adacc.ESIZE
    assert f(m=0, a=None, b=None, out=None) == adacc.OK


def test_python_refusals():
    x = torch.zeros(4, 8)
    with pytest.raises(TypeError):
        adacc.mx4_compress(x.double(), None, None)
    with pytest.raises(ValueError):
        adacc.mx4_compress(x.t(), None, None)
    with pytest.raises(TypeError):
        adacc.mx4_compress(x, None, None, offsets=torch.zeros(3))
    with pytest.raises(ValueError, match="scale_rule"):
        mx4._rule("ceil")
    with pytest.raises(ValueError):
        mx4.linear(x, torch.zeros(3, 9))
    with pytest.raises(ValueError):
        mx4.linear(x, torch.zeros(2, 3, 8))
    with pytest.raises(ValueError):
        mx4.experts(x, torch.zeros(2, dtype=torch.int32), torch.zeros(2, 3, 8))
    with pytest.raises(ValueError):
        adacc.mx4_gradient(None, None, 4, torch.zeros(3, 8), offsets=torch.zeros(3, dtype=torch.int32))
    for call in (lambda: mx4.compress(x), lambda: mx4.compress_both(x), lambda: mx4.linear(x, torch.zeros(3, 8)),
                 lambda: mx4.experts(x, torch.zeros(3, dtype=torch.int32), torch.zeros(2, 3, 8))):
        with pytest.raises(ValueError, match="on a GPU"):
            call()


def test_the_two_ways_of_a_call_agree(monkeypatch):
    """Refusals and sizes by the native marshalling and by ctypes."""
    x, out, small = torch.zeros(3, 8), torch.zeros(3, 5), torch.zeros(4, dtype=torch.uint8)

    def refusals():
        for call in (lambda: adacc.mx4_compress(x, small, stream=0), lambda: adacc.mx4_decompress(small, out, stream=0),
                     lambda: adacc.mx4_product(small, small, 8, out, stream=0), lambda: adacc.mx4_linear(x, small, out, stream=0),
                     lambda: adacc.mx4_gradient(small, small, 8, out, stream=0)):
            with pytest.raises(adacc.AdaccError) as e:
                call()
            yield e.value.code
        yield adacc.mx4_linear_workspace_bytes(1000, 20, 300)

    native = list(refusals())
    assert native[:5] == [adacc.ESIZE] * 5
    monkeypatch.setattr(adacc, "_mx4_entries", {})
    monkeypatch.setattr(adacc, "_calls", adacc._LeavesAll())
    assert list(refusals()) == native

"""Conversions of so many rows that a call takes more than one launch (2^24 workgroups): every value, where every value is representable."""
import pytest
import torch

from paper_2508_00806_amd import mx4

pytestmark = pytest.mark.gpu


def test_more_rows_than_one_launch_converts():
    rows = (1 << 29) + 40
    print(f"[mx4 launches] {rows} rows", flush=True)
    x = torch.randint(1, 5, (rows, 1), dtype=torch.uint8, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).bfloat16()
    m = mx4.compress(x)
    torch.cuda.synchronize()
    print("[mx4 launches] compressed", flush=True)
    back = m.restore()
    assert torch.equal(back, x)


def test_more_matrices_than_one_launch_converts():
    mats = (1 << 24) + 5
    print(f"[mx4 launches] {mats} matrices", flush=True)
    x = (torch.randint(0, 2, (mats, 2, 32), dtype=torch.uint8, device="cuda", generator=torch.Generator("cuda").manual_seed(2)).bfloat16() + 2) * 0.5
    along, across = mx4.compress_both(x)
    torch.cuda.synchronize()
    print("[mx4 launches] compressed", flush=True)
    assert torch.equal(along.restore(), x)
    del along
    assert torch.equal(across.restore(), x.transpose(1, 2))

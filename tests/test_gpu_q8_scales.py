"""Scale bytes that a caller's own matrices in 8 bits may hold: far from 1, and 255, which is NaN for its block of one row.

Products of codes under scales whose powers cancel are those of the codes themselves: they have to agree bit for bit with the call under scales of 1."""
import pytest
import torch

from paper_2506_00812_amd import binding as vf

pytestmark = pytest.mark.gpu


def operands(m, n, k):
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    x, w = (vf.quantize(torch.randn((r, k), generator=g, device="cuda")) for r in (m, n))
    x.scales.fill_(127)
    w.scales.fill_(127)
    return x, w


SIZES = [(1, 64, 256), (5, 100, 300), (40, 200, 700), (300, 513, 640), (1500, 1000, 256)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_scales_far_from_one(m, n, k, dtype):
    x, w = operands(m, n, k)
    want = vf.linear_q8(x, w, dtype=dtype)
    for byte in (16, 60, 200, 238):
        x.scales.fill_(byte)
        w.scales.fill_(254 - byte)
        assert torch.equal(vf.linear_q8(x, w, dtype=dtype), want), byte


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_nan_scale_stays_in_its_row(m, n, k, dtype):
    x, w = operands(m, n, k)
    want = vf.linear_q8(x, w, dtype=dtype).float()
    row, column = m // 2, n - 3
    x.scales[row, 1] = 255
    w.scales[column, 0] = 255
    got = vf.linear_q8(x, w, dtype=dtype).float()
    assert got[row].isnan().all() and got[:, column].isnan().all()
    bad = torch.zeros((m, n), dtype=torch.bool, device="cuda")
    bad[row] = True
    bad[:, column] = True
    assert torch.equal(got[~bad], want[~bad])


def test_nan_scale_read_back():
    x, _ = operands(3, 1, 300)
    want = vf.dequantize(x, torch.float32)
    x.scales[1, 1] = 255
    got = vf.dequantize(x, torch.float32)
    assert got[1, 128:256].isnan().all()
    got[1, 128:256] = want[1, 128:256]
    assert torch.equal(got, want)

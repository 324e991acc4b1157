"""The gated encoder's operators on matrices of more than 2^31 elements: what lies beyond is computed as it would be by itself."""
import math

import pytest
import torch

from paper_2506_00812_amd import binding as vf
from .test_gpu_ops_offsets import rows

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def close(a, b, part):
    return (a.float() - b.float()).abs().max() <= part * b.float().abs().max()


def tail(q, n):
    return q._replace(codes=q.codes[-n:], scales=q.scales[-n:])


def test_gated_linear():
    m, n, k = 270_000, 4104, 16
    x, w = rows(m, k), rows(2 * n, k)
    y, z = vf.gated_linear(x, w, save=True)
    last, lz = vf.gated_linear(x[-300:].contiguous(), w, save=True)
    assert close(y[-300:], last, 2 ** -7) and close(z[-300:], lz, 2 ** -7) and torch.equal(y[:7], y[7:14])
    dx, _, _ = vf.gated_linear_backward(y, x, w, z, dweight=False)
    want = vf.gated_linear_backward(y[-300:], x[-300:], w, z[-300:], dweight=False)[0]
    assert close(dx[-300:], want, 2 ** -6) and torch.equal(dx[:7], dx[7:14])


def test_operands_in_8_bits():
    m, n, k = 530_000, 20, 4200
    x = rows(m, k)
    q, w = vf.quantize(x), vf.quantize(rows(n, k, 2))
    want = vf.quantize(x[-300:].contiguous())
    assert torch.equal(q.codes[-300:].view(torch.uint8), want.codes.view(torch.uint8)) and torch.equal(q.scales[-300:, :33], want.scales[:, :33])
    del x
    y = vf.linear_q8(q, w)
    assert close(y[-300:], vf.linear_q8(want, w), 2 ** -7) and torch.equal(y[:7], y[7:14])
    assert torch.equal(vf.dequantize(q, BF)[-300:], vf.dequantize(want, BF))


def test_outputs_in_8_bits_and_wide():
    m, n, k = 530_000, 4200, 128
    x, w, wg = vf.quantize(rows(m, k)), vf.quantize(rows(n, k, 2)), vf.quantize(rows(2 * n, k, 3))
    few = tail(x, 300)
    y = vf.linear_q8(x, w)
    want = vf.linear_q8(few, w)
    assert close(y[-300:], want, 2 ** -7) and torch.equal(y[:7], y[7:14])
    assert torch.equal(vf.linear_q8(x, w, residual=y, out=y)[:7], y[7:14])
    del y
    for gated in (False, True):
        out = vf.linear_q8(x, wg if gated else w, activation="silu", gated=gated, quantize=True)
        one = vf.linear_q8(few, wg if gated else w, activation="silu", gated=gated, quantize=True)
        # (a sum in another order may take the next code: 2^-3 of a value)
        assert close(vf.dequantize(tail(out, 300), BF), vf.dequantize(one, BF), 2 ** -3) and torch.equal(out.codes[:7].view(torch.uint8), out.codes[7:14].view(torch.uint8))
        del out


def test_rms_norm():
    m, d = 2_200_000, 1024
    x = rows(m, d)
    y, total, rs = vf.rms_norm(x, residual=x, save=True)
    want = vf.rms_norm(x[-5:].contiguous(), residual=x[-5:].contiguous(), save=True)
    assert all(torch.equal(a[-5:], b) for a, b in zip((y, total, rs), want)) and torch.equal(y[:7], y[7:14])
    q, _ = vf.rms_norm(x, residual=x, quantize=True, out_total=total)
    one, _ = vf.rms_norm(x[-5:].contiguous(), residual=x[-5:].contiguous(), quantize=True)
    assert torch.equal(q.codes[-5:].view(torch.uint8), one.codes.view(torch.uint8)) and torch.equal(q.scales[-5:], one.scales)
    del q
    dx, _ = vf.rms_norm_backward(x, total, rs, d_total=x, dweight=False, out=y)
    one, _ = vf.rms_norm_backward(x[-5:], total[-5:], rs[-5:].clone(), d_total=x[-5:], dweight=False)
    assert torch.equal(dx[-5:], one)


def test_distill():
    m, v = 11_000, 200_001
    x = rows(m, v)
    ids = ((v - 1) - torch.arange(m * 40, device="cuda") % 7000).to(torch.int32).view(m, 40)
    val = torch.randn((m, 40), device="cuda")
    loss, lse = vf.distill(x, ids, val)
    want = vf.distill(x[-4:].clone(), ids[-4:].clone(), val[-4:].clone())
    assert (loss[-4:] - want[0]).abs().max() < 1e-4 and (lse[-4:] - want[1]).abs().max() < 1e-4
    d = torch.ones(m, device="cuda")
    last = vf.distill_backward(x[-4:].clone(), lse[-4:].clone(), ids[-4:].clone(), val[-4:].clone(), d[-4:].clone())
    g = vf.distill_backward(x, lse, ids, val, d, out=x)
    assert torch.equal(g[-4:], last)


def test_long_rows():
    """One row of 2^31 - 1 labels, and norms of rows of 2^24."""
    v = (1 << 31) - 1
    x = torch.zeros((1, v), dtype=BF, device="cuda")
    x[0, -1] = 25.0
    ids = torch.tensor([[v - 1, 0]], dtype=torch.int32, device="cuda")
    loss, lse = vf.distill(x, ids, torch.zeros((1, 2), device="cuda"))
    total = (v - 1) + math.exp(25)
    want = math.log(total)
    assert abs(lse.item() - want) < 1e-3 and abs(loss.item() - (-math.log(2) - 12.5 + want)) < 1e-3
    dx = vf.distill_backward(x, lse, ids, torch.zeros((1, 2), device="cuda"), torch.ones(1, device="cuda"), out=x)
    p = math.exp(25) / total
    assert abs(dx[0, -1].item() - (p - 0.5)) < 0.004 and abs(dx[0, 0].item() + 0.5) < 0.004
    del x, dx
    d = 1 << 24
    x = torch.ones((3, d), dtype=BF, device="cuda")
    y, rs = vf.rms_norm(x, eps=0.0, save=True)
    assert (y == 1).all() and ((rs - 1).abs() < 1e-4).all()
    q = vf.rms_norm(x, eps=0.0, quantize=True)
    assert (q.scales == 119).all() and torch.equal(vf.dequantize(q, BF), x)

"""The gated encoder's operators on slices of one buffer; outputs over inputs are refused."""
import pytest
import torch

from paper_2506_00812_amd import binding as vf

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("lead", [0, 3, 8])
def test_slices_of_one_buffer(lead):
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    m, k, n = 300, 96, 64
    wide = torch.randn((m, lead + k + 2 * n), generator=g, device="cuda").to(BF)
    w = torch.randn((2 * n, k), generator=g, device="cuda").to(BF)
    x, r, out = wide[:, lead:lead + k], wide[:, lead + k:lead + k + n], wide[:, lead + k + n:]
    want = vf.gated_linear(x.contiguous(), w)
    left = wide[:, :lead + k + n].clone()
    assert torch.equal(vf.gated_linear(x, w, out=out), want) and torch.equal(wide[:, :lead + k + n], left)
    x8, w8 = vf.quantize(x), vf.quantize(w[:n])
    want = vf.linear_q8(x8, w8, residual=r.contiguous())
    assert torch.equal(vf.linear_q8(x8, w8, residual=r, out=out), want) and torch.equal(wide[:, :lead + k + n], left)
    assert torch.equal(vf.linear_q8(x8, w8, residual=r, out=r), want)
    a, b, c = wide[:, :n], wide[:, n:2 * n], torch.empty((m, n), dtype=BF, device="cuda")
    want = vf.rms_norm(a.contiguous(), residual=b.contiguous())
    y, total = vf.rms_norm(a, residual=b, out=c, out_total=a)
    assert torch.equal(y, want[0]) and torch.equal(a, want[1])


def test_refusals():
    x = torch.randn((20, 32), device="cuda")
    w = torch.randn((64, 32), device="cuda")
    rs = torch.ones(20, device="cuda")
    buf = torch.randn((21, 32), device="cuda")
    ids = torch.zeros((20, 4), dtype=torch.int32, device="cuda")
    val = torch.zeros((20, 4), device="cuda")
    x8, w8 = vf.quantize(x), vf.quantize(w)
    over = torch.zeros((20, 128), dtype=torch.uint8, device="cuda")
    y8 = over.view(torch.float32)      # [20, 32], the codes' own memory
    bad = [lambda: vf.gated_linear(x, w, out=x), lambda: vf.gated_linear(x, w[:40], out=w[:20, :20]), lambda: vf.gated_linear(buf[1:], w, out=buf[:20]),
           lambda: vf.linear_q8(x8._replace(codes=over.view(torch.float8_e4m3fn)), vf.quantize(w[:32]), dtype=torch.float32, out=y8),
           lambda: vf.linear_q8(x8, vf.quantize(w[:32]), residual=buf[1:], out=buf[:20], dtype=torch.float32),
           lambda: vf.dequantize(x8._replace(codes=over.view(torch.float8_e4m3fn)), torch.float32, out=y8),
           lambda: vf.rms_norm(buf[1:], out=buf[:20]), lambda: vf.rms_norm(x, residual=buf[1:], out_total=buf[:20]), lambda: vf.rms_norm(x, residual=buf[1:], out=buf[:20]),
           lambda: vf.rms_norm_backward(buf[1:], x, rs, out=buf[:20]), lambda: vf.rms_norm_backward(w[:20], x, rs, out=x),
           lambda: vf.rms_norm_backward(x, w[:20], rs, d_total=buf[1:], out=buf[:20]),
           lambda: vf.distill_backward(buf[1:], rs, ids, val, rs, out=buf[:20]), lambda: vf.distill_backward(x, buf.view(-1)[5:25], ids, val, rs, out=buf[:20])]
    for f in bad:
        with pytest.raises(vf.VecflowError, match="overlap"):
            f()

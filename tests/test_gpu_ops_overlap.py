"""Outputs beside inputs in one buffer are written; outputs over inputs are refused."""
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
    w = torch.randn((n, k), generator=g, device="cuda").to(BF)
    x, r, out = wide[:, lead:lead + k], wide[:, lead + k:lead + k + n], wide[:, lead + k + n:]
    want = vf.linear(x.contiguous(), w, residual=r.contiguous())
    left = wide[:, :lead + k + n].clone()
    assert torch.equal(vf.linear(x, w, residual=r, out=out), want) and torch.equal(wide[:, :lead + k + n], left)
    assert torch.equal(vf.linear(x, w, residual=r, out=r), want)
    a, b = wide[:, :n], wide[:, n:2 * n]
    want = vf.layer_norm(a.contiguous())
    assert torch.equal(vf.layer_norm(a, out=b), want) and torch.equal(vf.layer_norm(a, out=a), want)


def test_refusals():
    x = torch.randn((20, 32), device="cuda")
    w = torch.randn((32, 32), device="cuda")
    mu, rs = torch.zeros(20, device="cuda"), torch.ones(20, device="cuda")
    buf = torch.randn((21, 32), device="cuda")
    lse = buf.view(-1)[5:25]
    bad = [lambda: vf.linear(x, w, out=x), lambda: vf.linear(x, w[:20], out=w[:20, :20]), lambda: vf.linear(buf[1:], w, out=buf[:20]),
           lambda: vf.linear(x, w, residual=buf[1:], out=buf[:20]), lambda: vf.layer_norm(buf[1:], out=buf[:20]),
           lambda: vf.layer_norm_backward(buf[1:], x, mu, rs, out=buf[:20]), lambda: vf.layer_norm_backward(w[:20], x, mu, rs, out=x),
           lambda: vf.log_probs_backward(buf[1:], mu, out=buf[:20]), lambda: vf.log_probs_backward(x, lse, out=buf[:20])]
    for f in bad:
        with pytest.raises(vf.VecflowError, match="overlap"):
            f()

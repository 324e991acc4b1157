"""Logits far from zero: the forward pass loses nothing but the logits' own rounding, the gradient what its one float per row does.

p = exp(x - lse) with an lse that is rounded by 2^-24 |lse|, a difference that is exact or rounds by 2^-24 |x - lse|, and an exponential of
2^-23 (1 + |x - lse|): all relative errors of p.  The gradient of logp is d (1 - p) at the target and -d p elsewhere; its sum over a row, 0, is off by
the shared part times d and by the sum of the others'."""
import pytest
import torch

from paper_2506_00812_amd import binding as vf

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("offset", [0.0, 100.0, 1e4, -1e4, 1e6])
@pytest.mark.parametrize("v", [100, 5000])
def test_gradient(v, offset):
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    m = 64
    x = torch.randn((m, v), generator=g, device="cuda") * 2 + offset
    x[0, 7] += 40          # one label has everything
    t = torch.randint(0, v, (m,), generator=g, device="cuda", dtype=torch.int32)
    t[0] = 7
    d = torch.randn(m, generator=g, device="cuda")
    logp, _, lse = vf.log_probs(x, t)
    l = torch.log_softmax(x.double(), 1)
    want_logp = l.gather(1, t.long()[:, None])[:, 0]
    assert ((logp.double() - want_logp).abs() <= 2.0 ** -20 * (8 + want_logp.abs())).all()      # whatever the offset
    got = vf.log_probs_backward(x, lse, t, d)
    p, d = l.exp(), d.double()
    want = -d[:, None] * p
    want[torch.arange(m, device="cuda"), t.long()] += d
    shared = (2.0 ** -23 * lse.abs().double())[:, None]
    own = 2.0 ** -22 * (4 + l.abs())
    off = d.abs()[:, None] * p * (torch.expm1(shared) + own) + 2.0 ** -22 * want.abs() + 1e-36
    assert ((got.double() - want).abs() <= off).all()
    assert (got.double().sum(1).abs() <= off.sum(1)).all()


def test_an_offset_taken_off_first():
    """What the header says to do: the same logits less their offset (exact here) have a gradient whose sums are 0 to 1e-5."""
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = (torch.randn((50, 1000), generator=g, device="cuda") * 64).round() / 64 + 8192
    t = torch.arange(50, dtype=torch.int32, device="cuda")
    d = torch.ones(50, device="cuda")
    _, _, lse = vf.log_probs(x - 8192, t)
    assert (vf.log_probs_backward(x - 8192, lse, t, d).double().sum(1).abs() < 1e-5).all()

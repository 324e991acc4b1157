"""The encoder operators on matrices of more than 2^31 elements: what lies beyond is computed as it would be by itself."""
import pytest
import torch

from paper_2506_00812_amd import binding as vf

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def rows(m, d, seed=1):
    """[m, d] of a few repeated rows, the last three their own."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((7, d), generator=g, device="cuda").to(BF).repeat(-(-m // 7), 1)[:m]
    x[-3:] = torch.randn((3, d), generator=g, device="cuda").to(BF)
    return x


def test_linear():
    m, n, k = 530_000, 4104, 16
    x, w = rows(m, k), rows(n, k)
    y, z = vf.linear(x, w, activation="gelu", save=True)
    last = vf.linear(x[-300:].contiguous(), w, activation="gelu")
    assert (y[-300:].float() - last.float()).abs().max() <= 2 ** -7 * last.float().abs().max() and torch.equal(y[:7], y[7:14])
    dx, dw, db = vf.linear_backward(y, x, w, z=z, activation="gelu", dweight=False)
    want = vf.linear_backward(y[-300:], x[-300:], w, z=z[-300:], activation="gelu", dweight=False)[0]
    assert (dx[-300:].float() - want.float()).abs().max() <= 2 ** -6 * want.float().abs().max() and torch.equal(dx[:7], dx[7:14])


def test_layer_norm():
    m, d = 2_200_000, 1024
    x = rows(m, d)
    y, mu, rs = vf.layer_norm(x, save=True)
    want = vf.layer_norm(x[-5:].contiguous(), save=True)
    assert all(torch.equal(a[-5:], b) for a, b in zip((y, mu, rs), want)) and torch.equal(y[:7], y[7:14])
    dx, _, _ = vf.layer_norm_backward(x, x, mu, rs, dweight=False, dbias=False, out=y)
    one, _, _ = vf.layer_norm_backward(x[-5:], x[-5:], mu[-5:].clone(), rs[-5:].clone(), dweight=False, dbias=False)
    assert torch.equal(dx[-5:], one)


def test_log_probs():
    m, v = 11_000, 200_001
    x = rows(m, v)
    t = torch.arange(m, dtype=torch.int32, device="cuda") + (v - m)
    out = vf.log_probs(x, t, top=3)
    want = vf.log_probs(x[-4:].clone(), t[-4:].clone(), top=3)
    for a, b in zip(out, want):
        assert torch.equal(a[-4:], b) if a.dtype == torch.int32 else (a[-4:] - b).abs().max() < 1e-4
    d = torch.ones(m, device="cuda")
    last = vf.log_probs_backward(x[-4:].clone(), out[2][-4:].clone(), t[-4:].clone(), d[-4:].clone())
    g = vf.log_probs_backward(x, out[2], t, d, out=x)
    assert torch.equal(g[-4:], last)


def test_adamw():
    n = (1 << 31) + 1000
    p = torch.ones(n, dtype=BF, device="cuda")
    g = torch.full((n,), 0.5, dtype=BF, device="cuda")
    st = vf.adamw_state(p, 8)
    vf.adamw_step([p], [g], [st[0]], [st[1]], step=1, lr=0.25, m_scales=[st[2]], v_scales=[st[3]])
    for t in (p[-2000:], p[:2000]):
        assert (t == 0.75).all()
    assert (st[0][-1000:] == 127).all() and (st[1][-1000:] == 254).all() and (st[2] == st[2][0]).all()

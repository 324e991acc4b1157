"""Column sums and row-contiguous products of matrices of more than 2^31 elements: only what lies beyond contributes."""
import math

import pytest
import torch

from paper_2506_00812_amd import binding as vf

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("lead", [0, 3])
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_linear_backward(act, lead):
    """dy is 0 but in the last `live` rows, all of them beyond 2^31 elements; x there is that of rows of its own.  lead: x's rows start on
    16 bytes or between."""
    m, n, k, live = 530_000, 4104, 16, 4000
    assert (m - live) * n > 1 << 31
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn((m, k + 8), generator=g, device="cuda").to(BF)[:, lead:lead + k]
    w = torch.randn((n, k), generator=g, device="cuda").to(BF)
    dy = torch.zeros((m, n), dtype=BF, device="cuda")
    dy[-live:] = torch.randn((live, n), generator=g, device="cuda").to(BF)
    z = None
    dz = dy[-live:].double()
    e = 0 * dz
    if act == "gelu":
        z = torch.zeros((m, n), dtype=BF, device="cuda")
        z[-live:] = torch.randn((live, n), generator=g, device="cuda").to(BF)
        Z = z[-live:].double()
        dz = dz * (torch.erfc(-Z / math.sqrt(2)) / 2 + Z * torch.exp(-Z * Z / 2) / math.sqrt(2 * math.pi))
        e = (2.0 ** -8 + 2.0 ** -20) * dz.abs() + 2.0 ** -20 * dy[-live:].double().abs()
    dx, dw, db = vf.linear_backward(dy, x, w, z=z, activation=act)
    X, W = x[-live:].double(), w.double()
    # the sums have at most live terms that are not 0, and m additions at most
    for got, want, err in ((dw, dz.t() @ X, e.t() @ X.abs() + (live + 8) * 2.0 ** -24 * ((dz.abs() + e).t() @ X.abs())),
                           (db, dz.sum(0), 2.0 ** -19 * (dz.abs() + dy[-live:].double().abs()).sum(0) + (live + 8) * 2.0 ** -24 * dz.abs().sum(0)),
                           (dx[-live:], dz @ W, e @ W.abs() + (n + 8) * 2.0 ** -24 * ((dz.abs() + e) @ W.abs()))):
        assert ((got.double() - want).abs() <= err + 2.0 ** -8 * (want.abs() + err)).all()
    assert not dx[:-live].any()


def test_layer_norm_backward():
    m, d, live = 2_200_000, 1024, 4000
    assert (m - live) * d > 1 << 31
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    x = torch.zeros((m, d), dtype=BF, device="cuda")
    dy = torch.zeros((m, d), dtype=BF, device="cuda")
    for t in (x, dy):
        t[-live:] = torch.randn((live, d), generator=g, device="cuda").to(BF)
    mu, rs = torch.zeros(m, device="cuda"), torch.ones(m, device="cuda")
    _, dw, db = vf.layer_norm_backward(dy, x, mu, rs, dx=False)
    Y, H = dy[-live:].double(), x[-live:].double()
    for got, t in ((dw, Y * H), (db, Y)):
        want, err = t.sum(0), (live + 16) * 2.0 ** -24 * t.abs().sum(0)
        assert ((got.double() - want).abs() <= err + 2.0 ** -8 * (want.abs() + err)).all()

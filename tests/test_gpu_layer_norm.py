"""Layer norm and its gradients against their definition in 64 bits.

Bounds: a row's mean is off by at most (d + 8) 2^-24 avg|x|; the centred values by that and 2^-24 |x|; sums of d (of m) terms by d (m) 2^-24 of
the sum of their sizes; an output rounds by its type's unit roundoff."""
import math

import pytest
import torch

from paper_2506_00812_amd import binding as vf
from .ops_util import DTYPES, TINY, U, cut, within

pytestmark = pytest.mark.gpu

SIZES = [(1, 1), (3, 2), (130, 7), (5, 64), (33, 100), (1, 1024), (257, 511), (64, 1024), (40, 2049), (9, 5000), (300, 192), (3, 16392),
         (2, 40000), (5000, 96)]


def inputs(m, d, T, seed, mean=0.5, pad=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    make = lambda *s, std=1.0, mean=0.0: (torch.randn(s, generator=g, device="cuda") * std + mean).to(T)   # noqa: E731
    x, w, b, dy = make(m, d, std=2.0, mean=mean), make(d, std=0.3, mean=1.0), make(d, std=0.3), make(m, d)
    return (cut(x, pad), w, b, cut(dy, pad)) if pad else (x, w, b, dy)


def stats(x, eps=1e-5):
    X = x.double()
    mean = X.mean(1)
    c = X - mean[:, None]
    return c, mean, 1 / torch.sqrt((c * c).mean(1) + eps)


def check_forward(m, d, T, pad=0, mean=0.5, weights=True):
    x, w, b, _ = inputs(m, d, T, 1, mean, pad)
    y, mu, rs = vf.layer_norm(x, w if weights else None, b if weights else None, save=True)
    c, mean64, rstd64 = stats(x)
    size = x.double().abs().mean(1)
    e_mean = (d + 8) * 2.0 ** -24 * size
    within(mu, mean64, e_mean + 1e-30, "mean")
    # d(rstd) / rstd = -d(var) / 2 (var + eps): from the shifted mean (its square), from rounding x - mean, from the sum
    shift = e_mean ** 2 + 2 * e_mean * 2.0 ** -24 * size
    e_c = 2.0 ** -23 * (c.abs().mean(1) + e_mean) * 2 * c.abs().amax(1)
    rel = ((shift + e_c) * rstd64 ** 2 + (d + 16) * 2.0 ** -24) / 2 + 2.0 ** -22
    within(rs, rstd64, rel * rstd64, "rstd")
    h = c * rstd64[:, None]
    W, B = (w.double(), b.double()) if weights else (torch.ones(d, device="cuda").double(), torch.zeros(d, device="cuda").double())
    y64 = h * W + B
    e = W.abs() * (h.abs() * (rel + 2.0 ** -22)[:, None] + ((e_mean + 2.0 ** -24 * size) * rstd64)[:, None]) + 2.0 ** -23 * (y64.abs() + B.abs())
    within(y, y64, e + U[T] * (y64.abs() + e) + TINY[T], "y")


def check_backward(m, d, T, pad=0, weights=True):
    x, w, b, dy = inputs(m, d, T, 3, pad=pad)
    c, mean64, rstd64 = stats(x)
    mu, rs = mean64.float(), rstd64.float()
    dx, dw, db = vf.layer_norm_backward(dy, x, mu, rs, w if weights else None)
    X, Y, M, R = x.double(), dy.double(), mu.double()[:, None], rs.double()[:, None]
    h = (X - M) * R
    g = Y * (w.double() if weights else 1)
    a, b2 = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    dx64 = R * (g - a - h * b2)
    n = (d + 16) * 2.0 ** -24
    e = R * (n * g.abs().mean(1, keepdim=True) + 2.0 ** -22 * (g.abs() + a.abs()) + h.abs() * (n * (g * h).abs().mean(1, keepdim=True) + 2.0 ** -21 * b2.abs()))
    e = e + 2.0 ** -22 * (X.abs() + M.abs()) * R * R * (b2.abs() + g.abs().mean(1, keepdim=True))
    within(dx, dx64, e + U[T] * (dx64.abs() + e) + TINY[T], "dx")
    n = (m + 16) * 2.0 ** -24
    e_h = 2.0 ** -23 * ((X.abs() + M.abs()) * R)
    for got, terms, extra, what in ((dw, Y * h, (Y.abs() * e_h).sum(0), "dweight"), (db, Y, 0, "dbias")):
        want = terms.sum(0)
        e = n * terms.abs().sum(0) + extra
        within(got, want, e + U[T] * (want.abs() + e) + TINY[T], what)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,d", SIZES)
def test_sizes(m, d, dtype):
    check_forward(m, d, dtype)
    check_backward(m, d, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad", [3, 8])
def test_strides_and_no_weights(pad, dtype):
    for m, d in ((70, 131), (9, 2056), (2, 20001)):
        check_forward(m, d, dtype, pad=pad)
        check_forward(m, d, dtype, weights=False)
        check_backward(m, d, dtype, pad=pad)
        check_backward(m, d, dtype, weights=False)


def test_a_large_mean_cancels_nothing():
    for m, d in ((50, 1000), (3, 30000)):
        check_forward(m, d, torch.float32, mean=3000.0)


def test_many_rows_and_constant_rows():
    check_backward(70000, 64, torch.bfloat16)
    x = torch.full((4, 96), 2.5, device="cuda")
    y, mu, rs = vf.layer_norm(x, eps=1e-5, save=True)
    assert not y.any() and (mu == 2.5).all() and torch.allclose(rs, torch.full_like(rs, 1e-5 ** -0.5))


def test_rows_do_not_touch_each_other():
    for d in (96, 3000, 40000):
        x, w, b, dy = inputs(7, d, torch.float32, 5)
        want = vf.layer_norm(x, w, b, save=True)
        bad = x.clone()
        bad[3, d // 2] = math.nan
        bad[5, 0] = math.inf
        got = vf.layer_norm(bad, w, b, save=True)
        keep = [0, 1, 2, 4, 6]
        assert all(torch.equal(g[keep], h[keep]) for g, h in zip(got, want))
        assert torch.isnan(got[0][3]).all() and torch.isnan(got[0][5]).all()


def test_empty_and_partial_gradients():
    x, w, b, dy = inputs(0, 100, torch.bfloat16, 1)
    y, mu, rs = vf.layer_norm(x, w, b, save=True)
    assert y.shape == (0, 100)
    dx, dw, db = vf.layer_norm_backward(dy, x, mu, rs, w)
    assert dx.shape == (0, 100) and not dw.any() and not db.any()
    for d in (100, 30000):
        x, w, b, dy = inputs(9, d, torch.float32, 1)
        _, mu, rs = vf.layer_norm(x, w, b, save=True)
        full = vf.layer_norm_backward(dy, x, mu, rs, w)
        only = [vf.layer_norm_backward(dy, x, mu, rs, w, dx=i == 0, dweight=i == 1, dbias=i == 2) for i in range(3)]
        for i in range(3):
            assert torch.equal(only[i][i], full[i]) and all(only[i][j] is None for j in range(3) if j != i)
        assert torch.equal(vf.layer_norm_backward(dy, x, mu, rs, w, out=dy)[0], full[0]) and torch.equal(dy, full[0])
        want = vf.layer_norm(x, w, b)
        assert torch.equal(vf.layer_norm(x, w, b, out=x), want) and torch.equal(x, want)


def test_gradients_against_differences():
    """Central differences in 64 bits, h = 1e-4: third derivatives stay below 100, so 1e-6."""
    m, d, h = 3, 6, 1e-4
    x, w, b, dy = inputs(m, d, torch.float32, 8)
    _, mu, rs = vf.layer_norm(x, w, b, save=True)
    got = vf.layer_norm_backward(dy, x, mu, rs, w)
    args = [t.double() for t in (x, w, b)]
    for which in range(3):
        num = torch.zeros_like(args[which])
        for i in range(num.numel()):
            side = []
            for s in (h, -h):
                moved = [t.clone() for t in args]
                moved[which].view(-1)[i] += s
                c, _, r = stats(moved[0])
                side.append(((c * r[:, None] * moved[1] + moved[2]) * dy.double()).sum())
            num.view(-1)[i] = (side[0] - side[1]) / (2 * h)
        assert (got[which].double() - num).abs().max() < 2e-5


def test_refusals():
    x, w, b, dy = inputs(4, 16, torch.float32, 1)
    mu, rs = torch.zeros(4, device="cuda"), torch.ones(4, device="cuda")
    bad = [lambda: vf.layer_norm(x.double()), lambda: vf.layer_norm(x, w[:8]), lambda: vf.layer_norm(x, w.half()), lambda: vf.layer_norm(x, eps=-1.0),
           lambda: vf.layer_norm(x, eps=math.nan), lambda: vf.layer_norm(x[:, :0]), lambda: vf.layer_norm(x.cpu()), lambda: vf.layer_norm(x[0]),
           lambda: vf.layer_norm_backward(dy, x[:2], mu, rs), lambda: vf.layer_norm_backward(dy, x, mu[:3], rs),
           lambda: vf.layer_norm_backward(dy, x, mu.double(), rs), lambda: vf.layer_norm(x.t())]
    for f in bad:
        with pytest.raises(vf.VecflowError):
            f()

"""Log probabilities, entropy, alternatives and their gradient against the definition in 64 bits.

Bounds: S sums terms of relative error 2^-22 (1 + |d|) in lanes of at most v / 64 + 64 additions, so log S is off by the sum of those; the
alternatives are whole numbers and equal."""
import math

import numpy as np
import pytest
import torch

from paper_2506_00812_amd import binding as vf
from .ops_util import DTYPES, TINY, U, cut

pytestmark = pytest.mark.gpu


def make(m, v, T, seed, masked=0.1, pad=0, std=2.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((m, v), generator=g, device="cuda") * std
    if masked:
        x[torch.rand((m, v), generator=g, device="cuda") < masked] = -math.inf
    if m > 3:
        x[1] = -math.inf
    t = torch.randint(0, v, (m,), generator=g, device="cuda", dtype=torch.int32)
    if m > 3:
        t[2] = -1
    x = x.to(T)
    return cut(x, pad) if pad else x, t


def reference(x, t, top):
    X = x.double()
    lse = torch.logsumexp(X, 1)
    l = X - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[:, None]
    p = l.exp()
    h = -torch.special.xlogy(p, p).sum(1)
    logp = l.gather(1, t.clamp_min(0).long()[:, None])[:, 0].masked_fill(t < 0, 0.0)
    a = X.cpu().numpy()
    ids = np.argsort(-a, axis=1, kind="stable")[:, :top]
    val = np.take_along_axis(l.cpu().numpy(), ids, 1)
    return logp, h, lse, np.where(np.isneginf(val), -1, ids), val, p, l


def close(got, want, tol, what):
    got, want = got.double(), want.double()
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), what
    off = (got - want).abs()[~inf]
    tol = torch.as_tensor(tol, device=off.device, dtype=off.dtype).expand_as(want)[~inf]
    assert (off <= tol).all(), f"{what}: {(off - tol).max().item():.3g} beyond the bound"


def check(m, v, T, top, masked=0.1, pad=0, seed=1):
    x, t = make(m, v, T, seed, masked, pad)
    out = vf.log_probs(x, t, top=top)
    logp, h, lse, ids, val, p, l = reference(x, t, max(top, 1))
    e_log = (v / 64 + 80) * 2.0 ** -24 * (2 + math.log(v + 1)) * 4
    big = x.double().masked_fill(x == -math.inf, 0).abs().amax(1) + 20
    tol = e_log + 2.0 ** -22 * big
    close(out[0], logp, tol, "logp")
    close(out[1], h, (e_log + 2.0 ** -20) * (2 + math.log(v + 1)), "entropy")
    close(out[2], lse, tol, "lse")
    if top:
        k = min(top, v)
        assert (out[3][:, :k].cpu().numpy() == ids[:, :k]).all(), "alternatives"
        assert (out[3][:, k:] == -1).all() and (out[4][:, k:] == -math.inf).all()
        close(out[4][:, :k], torch.from_numpy(val[:, :k]).cuda(), tol[:, None], "top_logp")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,v", [(1, 1), (5, 2), (7, 63), (300, 100), (33, 1000), (5, 2048), (5, 2049), (40, 5000), (3, 10001), (1, 70001)])
def test_sizes(m, v, dtype):
    check(m, v, dtype, 8)
    check(m, v, dtype, 0, masked=0.0)


@pytest.mark.parametrize("top", [1, 2, 31, 63, 64])
def test_alternatives(top):
    for v in (50, 777, 3000, 40000):
        check(9, v, torch.bfloat16, top, masked=0.5)
        check(9, v, torch.float32, top, masked=0.999)


@pytest.mark.parametrize("pad", [3, 8])
def test_strides(pad):
    for dtype in DTYPES:
        check(20, 333, dtype, 5, pad=pad)
        check(6, 9001, dtype, 5, pad=pad)


def test_vocabulary_of_200000_and_many_rows():
    check(1, 200_000, torch.bfloat16, 8)
    check(70, 200_000, torch.float32, 3)
    check(3000, 1000, torch.float32, 10)
    check(2000, 3000, torch.bfloat16, 4)


def test_ascending_and_equal_rows():
    """Every label beats all before it; all labels tie (the lowest win)."""
    for v in (64, 1000, 5000, 20000):
        x = torch.stack([torch.arange(v, dtype=torch.float32), torch.zeros(v), -torch.arange(v, dtype=torch.float32)]).cuda()
        x[1, 1::2] = -0.0      # -0 and 0 are the same value
        ids = vf.log_probs(x, top=20)[3].cpu()
        assert ids[0].tolist() == list(range(v - 1, v - 21, -1)) and ids[1].tolist() == ids[2].tolist() == list(range(20))


def test_extremes():
    f = torch.finfo(torch.float32)
    for v in (100, 3000, 30000):
        x = torch.zeros((7, v), device="cuda")
        x[0] = f.min                         # the type's lowest value everywhere: uniform
        x[1, :] = f.min
        x[1, 3] = f.max                      # one label has everything
        x[2, 5] = math.nan
        x[3, 6] = math.inf
        x[4] = -math.inf
        x[4, v - 1] = -5.0                   # one label is left
        x[5] = -math.inf                     # none is
        x[5, 9] = math.nan                   # ... but a NaN
        x[6] = -math.inf
        t = torch.tensor([1, 3, 0, 0, v - 1, 0, 0], dtype=torch.int32, device="cuda")
        logp, h, lse, ids, tl = vf.log_probs(x, t, top=2)
        assert abs(logp[0].item() + math.log(v)) < 1e-4 and abs(h[0].item() - math.log(v)) < 1e-4 and ids[0].tolist() == [0, 1]
        assert logp[1].item() == 0 and h[1].item() == 0 and lse[1].item() == f.max and ids[1].tolist() == [3, 0]
        for r in (2, 3, 5):
            assert all(torch.isnan(u[r]).all() for u in (logp, h, lse)), r
        assert ids[2].tolist() == [5, 0] and ids[3].tolist() == [6, 0] and ids[5].tolist() == [9, -1]
        assert logp[4].item() == 0 and h[4].item() == 0 and ids[4].tolist() == [v - 1, -1] and tl[4].tolist() == [0.0, -math.inf]
        assert logp[6].item() == -math.inf and lse[6].item() == -math.inf and h[6].item() == 0 and ids[6].tolist() == [-1, -1]
        # targets outside the vocabulary: NaN, and no gradient of their own
        t[:] = v
        assert torch.isnan(vf.log_probs(x, t)[0]).all()
        t[:] = -7
        assert torch.isnan(vf.log_probs(x, t)[0]).all()
        g = vf.log_probs_backward(x, lse, t, torch.ones(7, device="cuda"))
        assert not g[[0, 1, 4, 6]].any()


def check_backward(m, v, T, masked=0.1, pad=0, entropy=True, seed=4):
    x, t = make(m, v, T, seed, masked, pad)
    _, _, _, _, _, p, l = reference(x, t, 1)
    X = x.double()
    lse = torch.logsumexp(X, 1)
    h = -torch.special.xlogy(p, p).sum(1).masked_fill(lse == -math.inf, 0)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dl, dh = torch.randn(m, generator=g, device="cuda"), torch.randn(m, generator=g, device="cuda")
    got = vf.log_probs_backward(x, lse.float(), t, dl, entropy=h.float() if entropy else None, d_entropy=dh if entropy else None)
    d = dl.double().masked_fill(t < 0, 0)
    want = -d[:, None] * p
    want[torch.arange(m, device="cuda"), t.clamp_min(0).long()] += d
    size = want.abs() + d.abs()[:, None] * p
    if entropy:
        term = torch.special.xlogy(p, p) + p * h[:, None]
        want = want - dh.double()[:, None] * term
        size = size + dh.double().abs()[:, None] * (torch.special.xlogy(p, p).abs() + p * h[:, None])
    want[lse == -math.inf] = 0
    reach = (l.masked_fill(l == -math.inf, 0).abs() + X.masked_fill(X == -math.inf, 0).abs().amax(1, keepdim=True) + 8)
    e = size * 2.0 ** -22 * reach + 1e-36
    off = (got.double() - want).abs() - (e + U[T] * (want.abs() + e) + TINY[T])
    assert (off <= 0).all(), off.max()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,v", [(1, 1), (5, 2), (300, 100), (33, 1000), (40, 5003), (3, 70001), (9000, 33)])
def test_backward(m, v, dtype):
    check_backward(m, v, dtype)
    check_backward(m, v, dtype, masked=0.0, entropy=False)
    check_backward(m, v, dtype, pad=3)


def test_gradients_against_differences():
    """Central differences in 64 bits, h = 1e-4: third derivatives below 10, so 1e-7."""
    m, v, h = 3, 7, 1e-4
    x, t = make(m, v, torch.float32, 6, masked=0)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    dl, dh = torch.randn(m, generator=g, device="cuda"), torch.randn(m, generator=g, device="cuda")
    _, ent, lse = vf.log_probs(x, t)
    got = vf.log_probs_backward(x, lse, t, dl, entropy=ent, d_entropy=dh)
    num = torch.zeros(m, v, dtype=torch.float64, device="cuda")
    for i in range(m * v):
        side = []
        for s in (h, -h):
            moved = x.double()
            moved.view(-1)[i] += s
            logp, H = reference(moved, t, 1)[:2]
            side.append((logp * dl.double() + H * dh.double()).sum())
        num.view(-1)[i] = (side[0] - side[1]) / (2 * h)
    assert (got.double() - num).abs().max() < 1e-5


def test_gradient_in_place():
    x, t = make(50, 4000, torch.bfloat16, 9)
    d = torch.randn(50, device="cuda")
    lse = vf.log_probs(x, t)[2]
    grad = vf.log_probs_backward(x, lse, t, d)
    assert torch.equal(vf.log_probs_backward(x, lse, t, d, out=x), grad) and torch.equal(x, grad)


def test_refusals():
    x, t = make(4, 50, torch.float32, 1)
    lse = torch.zeros(4, device="cuda")
    bad = [lambda: vf.log_probs(x.double(), t), lambda: vf.log_probs(x, t.long()), lambda: vf.log_probs(x, t[:2]), lambda: vf.log_probs(x, t, top=65),
           lambda: vf.log_probs(x, t, top=-1), lambda: vf.log_probs(x[:, :0], t), lambda: vf.log_probs(x.t(), t), lambda: vf.log_probs(x.cpu(), t),
           lambda: vf.log_probs_backward(x, lse, t), lambda: vf.log_probs_backward(x, lse[:2], t, lse), lambda: vf.log_probs_backward(x, lse, entropy=lse),
           lambda: vf.log_probs_backward(x, lse, t, lse, out=x[:, :9])]
    for f in bad:
        with pytest.raises(vf.VecflowError):
            f()

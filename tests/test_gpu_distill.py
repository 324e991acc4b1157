"""The divergence from a teacher's entries and its gradient against their definition in 64 bits.

Bounds: u = logits / t is rounded twice, exp by 2^-22 (1 + |exponent|); a row's sum of v terms, in up to 64 partial sums at least, is off by (v / 64 + 64) 2^-24; so
lse by e_lse = (v / 64 + 64) 2^-24 + 2^-21 (1 + max |u|).  q is off by r = 2^-21 (2 + max |teacher / t| + range) of itself, log q by as much; the loss by
sum q (r |log q - log p| + r + e_lse + 2^-22 |u|)."""
import math

import pytest
import torch

from paper_2506_00812_amd import binding as vf
from .ops_util import DTYPES, TINY, U, cut, within

pytestmark = pytest.mark.gpu
INF = math.inf


def make(m, v, top, T, seed, masked=0.1, pad=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((m, v), generator=g, device="cuda") * 2
    teacher = x + torch.randn((m, v), generator=g, device="cuda")
    gone = torch.rand((m, v), generator=g, device="cuda") < masked
    if m > 3:
        gone[m // 3] = True
    x[gone], teacher[gone] = -INF, -INF
    val, ids = teacher.topk(min(top, v), dim=1)
    fill = (0, top - val.shape[1])
    val = torch.nn.functional.pad(val, fill, value=-INF).contiguous()
    ids = torch.nn.functional.pad(ids.int(), fill, value=-1)
    ids = ids.masked_fill(val == -INF, -1).contiguous()
    return (cut(x.to(T), pad) if pad else x.to(T)), ids, val


def defined(x, ids, val, t):
    """(loss, lse, q by label, what rows have entries) in 64 bits."""
    u = x.double() / t
    lse = torch.logsumexp(u, 1)
    there = (ids >= 0) & (val > -INF)
    w = (val.double() / t).masked_fill(~there, -INF)
    any_ = there.any(1)
    q = torch.softmax(w.masked_fill(~any_[:, None], 0.0), 1).masked_fill(~there, 0.0)
    log_q = torch.log_softmax(w.masked_fill(~any_[:, None], 0.0), 1)
    at = ids.clamp_min(0).long()
    log_p = (u.gather(1, at) - lse[:, None])
    terms = torch.where(q > 0, q * (log_q - log_p), torch.zeros_like(q))
    by_label = torch.zeros_like(u)
    by_label.scatter_add_(1, at, q)
    return terms.sum(1), lse, by_label, any_, q, (log_q - log_p)


def check(m, v, top, T, t=2.0, masked=0.1, pad=0, seed=1):
    x, ids, val = make(m, v, top, T, seed, masked, pad)
    loss, lse = vf.distill(x, ids, val, temperature=t)
    want, lse64, by_label, any_, q, gap = defined(x, ids, val, t)
    u = torch.where(x == -INF, torch.zeros_like(x), x).double() / t
    big = u.abs().amax(1)
    e_lse = (v / 64 + 64) * 2.0 ** -24 + 2.0 ** -21 * (1 + big)
    empty = lse64 == -INF
    assert (lse[empty] == -INF).all()
    within(lse[~empty], lse64[~empty], e_lse[~empty], "lse")
    assert not loss[~any_].any()
    w = torch.where(val > -INF, val, torch.zeros_like(val)).double() / t
    r = 2.0 ** -21 * (2 + 2 * w.abs().amax(1))
    e = torch.where(q > 0, q * (r[:, None] * (gap.abs() + 1) + (e_lse + 2.0 ** -22 * (big + 1))[:, None]), torch.zeros_like(q)).sum(1) + 2.0 ** -22
    within(loss[any_], want[any_], e[any_], "loss")
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 7)
    d = torch.randn(m, generator=g, device="cuda")
    dx = vf.distill_backward(x, lse, ids, val, d, temperature=t)
    l = lse.double()[:, None]
    p = torch.where(torch.isinf(l), torch.zeros_like(u), torch.exp(x.double() / t - l))
    live = (any_ & ~empty)[:, None]
    want = torch.where(live, (d.double()[:, None] / t) * (p - by_label), torch.zeros_like(p))
    e = (d.double().abs()[:, None] / t) * (p * 2.0 ** -21 * (3 + 2 * u.abs() + 2 * torch.where(torch.isinf(l), torch.zeros_like(l), l).abs())
                                          + by_label * r[:, None]) + 2.0 ** -22 * want.abs()
    within(dx, want, e + U[T] * (want.abs() + e) + TINY[T], "dlogits")
    over = x.clone()
    assert torch.equal(vf.distill_backward(over, lse, ids, val, d, temperature=t, out=over), dx) and torch.equal(over, dx)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,v,top", [(1, 1, 1), (5, 2, 1), (9, 7, 8), (300, 100, 8), (33, 512, 32), (17, 513, 64), (200, 1000, 8), (10, 2049, 65), (7, 5000, 256),
                                     (1, 200_000, 64), (3, 70_001, 200), (600, 3001, 32), (5000, 300, 4)])
def test_sizes(m, v, top, dtype):
    check(m, v, top, dtype)


@pytest.mark.parametrize("pad", [3, 8])
@pytest.mark.parametrize("t", [0.5, 1.0, 4.0])
def test_strides_temperatures_and_masks(t, pad):
    for dtype in DTYPES:
        check(40, 777, 16, dtype, t=t, masked=0.0, pad=pad)
        check(40, 777, 16, dtype, t=t, masked=0.95, pad=pad)
        check(2, 9001, 100, dtype, t=t, masked=0.5, pad=pad)


def test_the_same_label_twice_and_rows_without_entries():
    x = torch.randn((4, 3000), device="cuda")
    ids = torch.tensor([[5, 9, 5, 5, -1, 2999], [-1] * 6, [7] * 6, [0, 1, 2, 3, 4, 5]], dtype=torch.int32, device="cuda")
    val = torch.randn((4, 6), device="cuda")
    val[3, 2] = -INF
    d = torch.tensor([1.0, 2.0, 3.0, -1.0], device="cuda")
    loss, lse = vf.distill(x, ids, val)
    want, lse64, by_label, *_ = defined(x, ids, val, 1.0)
    assert (loss.double() - want)[[0, 2, 3]].abs().max() < 1e-4 and loss[1] == 0
    dx = vf.distill_backward(x, lse, ids, val, d)
    p = torch.exp(x.double() - lse64[:, None])
    p[1] = 0
    assert (dx.double() - d.double()[:, None] * (p - by_label)).abs().max() < 1e-5 and not dx[1].any()
    many = ids[2:3].repeat(1, 40).contiguous()       # 240 entries, all the same label
    loss, lse = vf.distill(x[2:3], many, torch.zeros((1, 240), device="cuda"))
    dx = vf.distill_backward(x[2:3], lse, many, torch.zeros((1, 240), device="cuda"), d[:1])
    assert abs(dx[0, 7].item() - (math.exp(x[2, 7].item() - lse.item()) - 1)) < 1e-5


def test_masks_infinities_and_ids_outside():
    x = torch.randn((8, 600), device="cuda")
    ids = torch.arange(8, device="cuda", dtype=torch.int32).repeat(8, 1).contiguous()
    val = torch.zeros((8, 8), device="cuda")
    clean = vf.distill(x, ids, val)
    x[1, 3] = -INF            # a label of the teacher's that the student cannot give
    x[2] = -INF               # no label is left
    x[3, 50] = math.nan
    x[4, 50] = INF
    ids[5, 2] = 600
    ids[6, 1] = -2
    val[7, 0] = math.nan
    loss, lse = vf.distill(x, ids, val)
    assert loss[1] == INF and loss[2] == INF and torch.isnan(loss[3:]).all()
    assert torch.equal(loss[0], clean[0][0]) and lse[2] == -INF
    d = torch.ones(8, device="cuda")
    dx = vf.distill_backward(x, lse, ids, val, d)
    assert torch.isfinite(dx[0]).all() and torch.isfinite(dx[1]).all() and dx[1, 3] == -0.125
    assert not dx[2].any() and not dx[5].any() and not dx[6].any() and torch.isnan(dx[3]).any()
    # an entry whose probability vanishes at a masked label costs nothing
    val[1] = 0.0
    val[1, 3] = -1e30
    assert torch.isfinite(vf.distill(x, ids, val)[0][1])
    # the type's lowest value as a mask
    low = torch.randn((3, 700), device="cuda")
    low[:, 100:] = torch.finfo(torch.float32).min
    loss, lse = vf.distill(low, ids[:3], torch.zeros((3, 8), device="cuda"))
    assert (lse.double() - torch.logsumexp(low[:, :100].double(), 1)).abs().max() < 1e-5 and torch.isfinite(loss).all()


def test_it_takes_what_log_probs_gives():
    """A teacher that is the student itself: no divergence beyond the labels left out, no gradient on the entries' own balance."""
    x, _, _ = make(50, 400, 8, torch.float32, 3)
    _, _, lse, ids, logp = vf.log_probs(x, top=16)
    loss, lse2 = vf.distill(x, ids, logp)
    live = lse > -INF
    assert (lse - lse2)[live].abs().max() < 1e-5
    inside = torch.where(logp > -INF, logp.double().exp(), torch.zeros_like(logp).double()).sum(1)
    assert (loss.double() + inside.log())[live].abs().max() < 1e-5 and not loss[~live].any()


def test_gradients_against_differences():
    """Central differences in 64 bits, h = 1e-4: third derivatives below 10, so 1e-7; float32 p and q are off by 2^-20."""
    x, ids, val = make(2, 12, 4, torch.float32, 5, masked=0.0)
    d = torch.tensor([0.7, -1.3], device="cuda")
    _, lse = vf.distill(x, ids, val, temperature=1.5)
    got = vf.distill_backward(x, lse, ids, val, d, temperature=1.5)
    num = torch.zeros((2, 12), dtype=torch.float64, device="cuda")
    for i in range(24):
        side = []
        for s in (1e-4, -1e-4):
            moved = x.double()
            moved.view(-1)[i] += s
            side.append((defined(moved, ids, val, 1.5)[0] * d.double()).sum())
        num.view(-1)[i] = (side[0] - side[1]) / 2e-4
    assert (got.double() - num).abs().max() < 1e-5


def test_empty_and_refusals():
    x, ids, val = make(4, 50, 4, torch.float32, 1)
    loss, lse = vf.distill(x[:0], ids[:0], val[:0])
    assert loss.shape == (0,) and vf.distill_backward(x[:0], lse, ids[:0], val[:0], loss).shape == (0, 50)
    d = torch.ones(4, device="cuda")
    buf = torch.randn((5, 50), device="cuda")
    bad = [lambda: vf.distill(x, ids[:3], val[:3]), lambda: vf.distill(x, ids, val[:, :2]), lambda: vf.distill(x, ids.long(), val), lambda: vf.distill(x, ids, val.half()),
           lambda: vf.distill(x, ids[:, :0], val[:, :0]), lambda: vf.distill(x, ids, val, temperature=0.0), lambda: vf.distill(x, ids, val, temperature=math.nan),
           lambda: vf.distill(x, ids, val, temperature=-1.0), lambda: vf.distill(x.double(), ids, val), lambda: vf.distill(x, ids.t().contiguous().t(), val),
           lambda: vf.distill(x, ids.repeat(1, 65), val.repeat(1, 65)), lambda: vf.distill_backward(x, d[:2], ids, val, d),
           lambda: vf.distill_backward(x, d, ids, val, d.half()), lambda: vf.distill_backward(buf[1:], d, ids, val, d, out=buf[:4]),
           lambda: vf.distill(x, ids.cpu(), val)]
    for f in bad:
        with pytest.raises(vf.VecflowError):
            f()

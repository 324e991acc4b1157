"""The gated encoder's operators on small whole numbers, whose products and sums float32 holds exactly in any order: one row, column or label that a long sum
leaves out is off by a whole number, where bounds that grow with a sum's length would let it pass.

What is left are the roundings of single results, counted at each check; where a result is only near the definition the check says how far one lost term
would move it."""
import math

import pytest
import torch

from paper_2506_00812_amd import binding as vf
from .ops_util import DTYPES, U, within
from .test_gpu_q8 import held
from .test_gpu_q8_tilings import CASES, CODE

pytestmark = pytest.mark.gpu
INF = math.inf
EPS = 1e-6


def whole(g, *shape, most=2):
    """Whole numbers from -most to most without 0."""
    v = torch.randint(1, most + 1, shape, generator=g, device="cuda")
    return v * (2 * torch.randint(0, 2, shape, generator=g, device="cuda") - 1)


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


# columns at both sides of each border between kernels, and lengths whose last ones are a part of a thread's eight
WIDTHS = [1, 7, 127, 128, 129, 255, 256, 257, 511, 512, 513, 1023, 1024, 1025, 2047, 2048, 2049, 4096, 4097, 8192, 8199, 12_008, 16_384, 16_385, 40_000, 100_003]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", WIDTHS)
def test_norm_has_every_column(d, dtype):
    """The sum of squares is exact.  Its mean is rounded twice (the division, epsilon), the root and its inverse once each: 3 2^-24 of rstd; a lost column
    that is not 0 moves rstd by half of 1 / sum at least."""
    for m in (1, 5):
        g = generator(d + m)
        x, r, w = whole(g, m, d).to(dtype), whole(g, m, d).to(dtype), whole(g, d).to(dtype)
        x[:, -1], r[:, -1] = 2, 2     # (a last column that counts)
        total = x + r
        assert (2.0 ** -22 < 0.25 / total.double().square().sum(1)).all()
        rstd64 = (total.double().square().mean(1) + EPS) ** -0.5
        y64 = total.double() * rstd64[:, None] * w.double()
        y, kept, rstd = vf.rms_norm(x, w, residual=r, eps=EPS, save=True)
        assert torch.equal(kept, total)
        within(rstd, rstd64, 2.0 ** -22 * rstd64, "rstd")
        e = 2.0 ** -21 * y64.abs()
        within(y, y64, e + U[dtype] * (y64.abs() + e) + (2.0 ** -24 if dtype == torch.float16 else 0), "y")
        q, kept, again = vf.rms_norm(x, w, residual=r, eps=EPS, save=True, quantize=True)
        assert torch.equal(again, rstd) and torch.equal(kept, total)
        y, rstd = vf.rms_norm(total, w, eps=EPS, save=True)
        assert torch.equal(rstd, again)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,d", [(1, 5), (9, 64), (70_000, 64), (32, 100), (33, 100), (5001, 96), (9, 256), (3000, 257), (8, 1000), (701, 1024), (3, 1500), (300, 2048),
                                 (203, 4097), (1500, 8192), (101, 16_384), (7, 16_385), (1027, 20_000), (130, 40_001)])
def test_norm_gradients_have_every_row_and_column(m, d, dtype):
    """With rstd a power of two everything is exact but dx's b = sum / d, h b, g - h b and the last addition, a rounding each: 2^-24 of each.  dweight is the exact
    sum's rounding to its type."""
    g = generator(m + d)
    s, dy, w, more = whole(g, m, d).to(dtype), whole(g, m, d).to(dtype), whole(g, d).to(dtype), whole(g, m, d, most=8).to(dtype)
    rstd = torch.full((m,), 0.5, device="cuda")
    dx, dw = vf.rms_norm_backward(dy, s, rstd, w, d_total=more)
    h, gw = s.double() / 2, dy.double() * w.double()
    b = (gw * h).mean(1, keepdim=True)
    want = 0.5 * (gw - h * b) + more.double()
    e = 2.0 ** -23 * (0.5 * (gw.abs() + 2 * (h * b).abs()) + more.double().abs() + want.abs())
    within(dx, want, e + U[dtype] * (want.abs() + e) + (2.0 ** -24 if dtype == torch.float16 else 0), "dx")
    assert torch.equal(dw, (dy.double() * h).sum(0).to(dtype))
    none, alone = vf.rms_norm_backward(dy, s, rstd, w, d_total=more, dx=False)
    assert none is None and torch.equal(alone, dw)


LABELS = [1, 63, 64, 511, 513, 1024, 1025, 2047, 2048, 2049, 3001, 4096, 6143, 6144, 6145, 9001, 70_001, 200_000]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("v", LABELS)
def test_distillation_has_every_label(v, dtype):
    """Logits of 0 and -inf: a row's sum is the number of its labels n, exactly, and lse its logarithm, off by 2^-22 of itself; one lost label moves it by 1 / n.
    Equal entries have q = 1 / top, off by 3 2^-24, and the loss log(n / top), the difference of two logarithms."""
    for m in (1, 3) + ((1100,) if v <= 9001 else ()):
        g = generator(v + m)
        x = torch.zeros((m, v), dtype=dtype, device="cuda")
        x[torch.rand((m, v), generator=g, device="cuda") < 0.25] = -INF
        x[:, [0, v // 2, v - 1]] = 0
        top = min(3, v)
        ids = torch.tensor([0, v // 2, v - 1], dtype=torch.int32, device="cuda")[:top].repeat(m, 1).contiguous()
        loss, lse = vf.distill(x, ids, torch.full((m, top), -1.5, device="cuda"), temperature=2.0)
        n = (x == 0).double().sum(1)
        e = 2.0 ** -22 * n.log() + 2.0 ** -24
        assert (e < 1 / n / 1.5).all()
        within(lse, n.log(), e, "lse")
        within(loss, (n / top).log(), e + 2.0 ** -21 * (1 + math.log(top)), "loss")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("v", LABELS[3:])
def test_distillation_has_labels_anywhere(v, dtype):
    """One label of 90 among labels of 0 is its row's lse, to a rounding of 90: 200,000 exp(-90) is below 2^-100."""
    at = sorted({0, 1, 7, 8, 63, 64, 255, 256, v // 3, 4095 % v, 4096 % v, v // 2, v - 9, v - 8, v - 2, v - 1})
    m = len(at)
    x = torch.zeros((m, v), dtype=dtype, device="cuda")
    x[torch.arange(m, device="cuda"), torch.tensor(at, device="cuda")] = 90
    ids = torch.tensor(at, dtype=torch.int32, device="cuda")[:, None].contiguous()
    loss, lse = vf.distill(x, ids, torch.zeros((m, 1), device="cuda"))
    assert ((lse - 90).abs() <= 2.0 ** -17).all() and (loss.abs() <= 2.0 ** -17).all()
    dx = vf.distill_backward(x, lse, ids, torch.zeros((m, 1), device="cuda"), torch.ones(m, device="cuda"))
    assert (dx.abs() <= 2.0 ** -16).all()


GATED = [(1, 5, 3), (9, 40, 200), (33, 131, 1000), (64, 17, 4097), (70, 40, 264), (200, 72, 776), (300, 96, 3001), (1000, 1000, 264), (3000, 100, 136), (70_001, 24, 16),
         (9001, 130, 72), (2500, 1024, 512), (700, 2500, 1024), (4100, 390, 321)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", GATED)
def test_gated_layer_has_every_term(m, n, k, dtype):
    """x, w and bias in {-1, 1}: z is exact, its rounding the only one of z, its product's the only one of y.  dy and z in {-2 .. 2}: dz is exact in every type,
    and each gradient the exact sum's rounding."""
    g = generator(m + n + k)
    x, w, b = (whole(g, *s, most=1).to(dtype) for s in ((m, k), (2 * n, k), (2 * n,)))
    y, z = vf.gated_linear(x, w, b, activation="relu", save=True)
    z64 = x.double() @ w.double().t() + b.double()
    assert torch.equal(z, z64.to(dtype)) and torch.equal(y, (z64[:, :n].clamp_min(0) * z64[:, n:]).to(dtype))
    z, dy = whole(g, m, 2 * n).to(dtype), whole(g, m, n).to(dtype)
    dx, dw, db = vf.gated_linear_backward(dy, x, w, z, activation="relu")
    gate, up, D = z[:, :n].double(), z[:, n:].double(), dy.double()
    dz = torch.cat([D * up * (gate > 0), D * gate.clamp_min(0)], 1)
    assert torch.equal(dx, (dz @ w.double()).to(dtype)) and torch.equal(dw, (dz.t() @ x.double()).to(dtype)) and torch.equal(db, dz.sum(0).to(dtype))


@pytest.mark.parametrize("T,m,n,k,gated,quantize,tiling,split", CASES)
def test_products_in_8_bits_have_every_term(T, m, n, k, gated, quantize, tiling, split):
    """Codes of -2 .. 2 times 2^6: products of eight neighbours are within 2^2 of each other, so that the matrix cores lose nothing.  An output is its
    exact sum's rounding to its type or to 8 bits (gated: the product of two)."""
    assert vf.debug_linear_q8(CODE[T], m, n, k, gated, quantize)[0] == tiling
    g = generator(m + n + k)
    x, w, b = whole(g, m, k).float(), whole(g, n * (1 + gated), k).float(), whole(g, n * (1 + gated)).to(T)
    y = vf.linear_q8(vf.quantize(x), vf.quantize(w), b, activation="relu", gated=bool(gated), dtype=T, quantize=bool(quantize))
    z = x.double() @ w.double().t() + b.double()
    want = z[:, :n].clamp_min(0) * z[:, n:] if gated else z.clamp_min(0)
    if quantize:
        values, byte = held(want)
        assert torch.equal(vf.dequantize(y, torch.float32).double(), values) and torch.equal(y.scales[:, :byte.shape[1]], byte)
    else:
        assert torch.equal(y, want.float().to(T))

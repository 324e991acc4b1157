"""The linear layer on slices of wider matrices whose rows start on 16 bytes: operands and outputs whose row distance is not their length, in
every tiling that goes straight to LDS, with the bounds of test_gpu_linear.  Everything around the slices is NaN and stays NaN."""
import math

import pytest
import torch

from paper_2506_00812_amd import binding as vf
from .ops_util import TINY, U, within
from .test_gpu_linear import slope, value

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16
CODE = {BF: vf.VF_BF16, HF: vf.VF_F16}
# (m, n, k, dtype)
CASES = [(2049, 1096, 520, HF), (2500, 2056, 520, BF), (5001, 4104, 1032, BF), (9000, 4104, 1032, HF), (700, 4000, 4104, BF), (3001, 2056, 2056, HF),
         (10000, 520, 4104, BF), (10000, 1032, 1032, HF), (300, 1000, 520, BF), (40, 1000, 200, BF)]
LEAD, TAIL = 8, 16       # elements before and behind a slice's columns


def outer(rows, cols, dtype):
    return torch.full((rows + 2, LEAD + cols + TAIL), math.nan, dtype=dtype, device="cuda")


def inner(wide):
    return wide[1:-1, LEAD:-TAIL]


def around(wide):
    """Whether what surrounds the slice is NaN still."""
    keep = torch.ones_like(wide, dtype=torch.bool)
    inner(keep).fill_(False)
    return torch.isnan(wide[keep]).all()


def sliced(t):
    wide = outer(*t.shape, t.dtype)
    inner(wide).copy_(t)
    return inner(wide)


def direct(*operands):
    """Whether all operands' rows start on 16 bytes, whatever their distance; that distance is not their length."""
    for t in operands:
        assert t.stride(0) != t.shape[1]
    return all(t.data_ptr() % 16 == 0 and t.stride(0) % 8 == 0 for t in operands)


def make(m, n, k, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(41)
    normal = lambda *s, std=1.0: sliced((torch.randn(s, generator=g, device="cuda") * std).to(dtype))   # noqa: E731
    b = torch.randn(n, generator=g, device="cuda").to(dtype)
    return normal(m, k), normal(n, k, std=k ** -0.5), b, normal(m, n), normal(m, n)


def taken(m, n, k, dtype, x, w, dz):
    """The tilings of the three products, from the tensors themselves."""
    aligned = (direct(x, w), direct(w, dz) and k % 8 == 0, direct(x, dz) and k % 8 == 0 and n % 8 == 0)
    return [vf.debug_linear(CODE[dtype], m, n, k, p, aligned[p])[0] for p in range(3)]


def test_every_direct_tiling_is_reached():
    seen = [set(), set(), set()]
    for m, n, k, dtype in CASES:
        x, w, _, r, _ = make(m, n, k, dtype)
        for p, tiling in enumerate(taken(m, n, k, dtype, x, w, r)):
            seen[p].add(tiling)
    assert seen[0] >= {0, 3, 4, 5, 6} and seen[1] >= {3, 5, 6} and seen[2] >= {3, 5, 6}


def ptr(t):
    return None if t is None else t.data_ptr()


def ld(t):
    return 0 if t is None else t.stride(0)


def workspace(m, n, k, dtype, act, backward):
    size = vf._size_of("vf_linear_workspace", CODE[dtype], m, n, k, vf.ACTIVATIONS[act], backward)
    return torch.empty(max(size, 1), dtype=torch.uint8, device="cuda"), size


@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("case", CASES)
def test_forward(case, act):
    m, n, k, T = case
    x, w, b, r, _ = make(*case)
    wide_y, wide_z = outer(m, n, T), outer(m, n, T)
    y, z = inner(wide_y), inner(wide_z)
    ws, size = workspace(m, n, k, T, act, 0)
    vf._check(vf.load_library().vf_linear(CODE[T], m, n, k, ptr(x), ld(x), ptr(w), ld(w), ptr(b), vf.ACTIVATIONS[act], ptr(r), ld(r), ptr(y), ld(y), ptr(z),
                                          ld(z), ptr(ws), size, torch.cuda.current_stream().cuda_stream))
    z64 = x.double() @ w.double().t() + b.double()
    sums = (k + 8) * 2.0 ** -24 * (x.double().abs() @ w.double().abs().t() + b.double().abs())
    within(z, z64, sums + U[T] * (z64.abs() + sums) + TINY[T], "z")
    y64 = value(z64, act) + r.double()
    err = 1.13 * sums + 2.0 ** -20 * (z64.abs() + 1) + 2.0 ** -23 * r.double().abs()
    within(y, y64, err + U[T] * (y64.abs() + err) + TINY[T], "y")
    assert around(wide_y) and around(wide_z)
    assert torch.equal(vf.linear(x, w, b, residual=r, activation=act), y)


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("case", CASES)
def test_backward(case, act):
    m, n, k, T = case
    x, w, _, dy, z = make(*case)
    wide_x, wide_w = outer(m, k, T), outer(n, k, T)
    dx, dw, db = inner(wide_x), inner(wide_w), torch.empty(n, dtype=T, device="cuda")
    ws, size = workspace(m, n, k, T, act, 1)
    code = vf.ACTIVATIONS[act]
    vf._check(vf.load_library().vf_linear_backward(CODE[T], m, n, k, ptr(dy), ld(dy), ptr(x), ld(x), ptr(w), ld(w), ptr(z) if code else None, ld(z), code,
                                                   ptr(dx), ld(dx), ptr(dw), ld(dw), ptr(db), ptr(ws), size, torch.cuda.current_stream().cuda_stream))
    dz = dy.double() * slope(z.double(), act)
    e = 0 * dz if act == "none" else (U[T] + 2.0 ** -20) * dz.abs() + 2.0 ** -20 * dy.double().abs() + TINY[T]
    mag, X, W = dz.abs() + e, x.double(), w.double()
    for got, want, err, what in (
            (dx, dz @ W, e @ W.abs() + (n + 8) * 2.0 ** -24 * (mag @ W.abs()), "dx"),
            (dw, dz.t() @ X, e.t() @ X.abs() + (m + 8) * 2.0 ** -24 * (mag.t() @ X.abs()), "dw"),
            (db, dz.sum(0), (2.0 ** -20 * (dz.abs() + dy.double().abs())).sum(0) + (m + 8) * 2.0 ** -24 * mag.sum(0), "db")):
        within(got, want, err + U[T] * (want.abs() + err) + TINY[T], what)
    assert around(wide_x) and around(wide_w)
    again = vf.linear_backward(dy, x, w, z=z, activation=act)
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dw, db)))


@pytest.mark.parametrize("case", CASES[:4])
def test_rows_that_start_between(case):
    """The same sizes in rows that do not start on 16 bytes: no tiling that goes straight to LDS."""
    m, n, k, T = case
    x, w, b, r, _ = make(*case)
    off = [torch.full((t.shape[0], t.shape[1] + 12), math.nan, dtype=T, device="cuda")[:, 4:-8] for t in (x, w)]
    for a, t in zip(off, (x, w)):
        a.copy_(t)
    assert not direct(*off) and vf.debug_linear(CODE[T], m, n, k, 0, False)[0] <= 2
    z64 = x.double() @ w.double().t() + b.double()
    sums = (k + 8) * 2.0 ** -24 * (x.double().abs() @ w.double().abs().t() + b.double().abs())
    within(vf.linear(*off, b), z64, sums + U[T] * (z64.abs() + sums) + TINY[T], "z")

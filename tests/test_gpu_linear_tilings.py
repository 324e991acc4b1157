"""Every tiling of the linear layer's products at sizes that end inside its tiles, with the bounds of test_gpu_linear; and that what
a tile holds beyond the operands' ends reaches nothing."""
import math

import pytest
import torch

from paper_2506_00812_amd import binding as vf
from .test_gpu_linear import check_backward, check_forward, inputs

pytestmark = pytest.mark.gpu

BF, FP, HF = torch.bfloat16, torch.float32, torch.float16
CODE = {BF: vf.VF_BF16, FP: vf.VF_F32, HF: vf.VF_F16}
# (m, n, k, dtype, elements between rows beyond their ends): contractions of 8 beyond whole steps, tiles with 1 to 8 rows left
CASES = [(40, 1000, 200, BF, 0), (64, 4099, 1025, HF, 0), (300, 1000, 520, BF, 0), (2049, 1096, 520, BF, 0), (2049, 1096, 520, HF, 8),
         (2500, 2056, 520, BF, 0), (5000, 4104, 264, BF, 0), (700, 4000, 4104, HF, 0), (9000, 4104, 1032, BF, 0), (9000, 4104, 1032, HF, 8),
         (2500, 2056, 520, BF, 3), (9000, 4104, 1032, BF, 5), (3001, 1030, 777, FP, 0), (9000, 1032, 520, FP, 3), (130, 90, 5000, BF, 0),
         (64, 128, 4096, BF, 0), (10000, 96, 100, FP, 0), (257, 257, 8, BF, 0), (10000, 1032, 1032, HF, 0), (5001, 4104, 1032, BF, 8),
         (10000, 520, 4104, BF, 0), (3001, 2056, 2056, HF, 0)]


def plans(m, n, k, dtype, pad):
    aligned = dtype != FP and pad % 8 == 0 and k % 8 == 0
    return [vf.debug_linear(CODE[dtype], m, n, k, p, aligned and (p < 2 or n % 8 == 0)) for p in range(3)]


def test_the_cases_reach_every_tiling():
    seen = [set(), set(), set()]
    split = [False] * 3
    for c in CASES:
        for p, (tiling, splits) in enumerate(plans(*c)):
            seen[p].add(tiling)
            split[p] |= splits > 1
    assert seen[0] == {0, 1, 2, 3, 4, 5, 6} and seen[1] >= {1, 2, 3, 5, 6} and seen[2] >= {1, 2, 3, 5, 6} and all(split)


@pytest.mark.parametrize("case", CASES)
def test_forward(case):
    m, n, k, dtype, pad = case
    check_forward(m, n, k, dtype, "gelu", pad=pad, seed=31)
    check_forward(m, n, k, dtype, "none", pad=pad, residual=False, seed=32)


@pytest.mark.parametrize("case", CASES)
def test_backward(case):
    m, n, k, dtype, pad = case
    check_backward(m, n, k, dtype, "silu", pad=pad, seed=33)


@pytest.mark.parametrize("case", CASES)
def test_nan_stays_in_its_row_and_column(case):
    m, n, k, dtype, pad = case
    x, w, b, dy = inputs(m, n, k, dtype, 34, pad)
    y = vf.linear(x, w, b)
    dx, _, _ = vf.linear_backward(dy, x, w, dweight=False)
    x[m - 1, k - 1], w[n - 1, 0], dy[0, n - 1] = math.nan, math.inf, math.nan
    got = vf.linear(x, w, b)
    assert torch.isnan(got[m - 1]).all() and not torch.isfinite(got[:, n - 1]).any()
    assert torch.equal(got[:m - 1, :n - 1], y[:m - 1, :n - 1])
    w[n - 1, 0] = 0
    dx2, _, _ = vf.linear_backward(dy, x, w, dweight=False)
    assert torch.isnan(dx2[0]).all()
    assert torch.equal(dx2[1:, 1:], dx[1:, 1:])


@pytest.mark.parametrize("m,n,k,ld", [(3000, 2056, 1025, 1032), (9000, 4104, 1001, 1008), (2049, 1096, 515, 520), (40, 1000, 203, 208)])
def test_odd_contractions_in_aligned_rows(m, n, k, ld):
    """The last vector of a row holds what follows the row: NaN here, which must not get in."""
    x, w, _, _ = inputs(m, n, k, BF, 35)
    wide = [torch.full((t.shape[0], ld), math.nan, dtype=BF, device="cuda") for t in (x, w)]
    for a, t in zip(wide, (x, w)):
        a[:, :k] = t
    got = vf.linear(wide[0][:, :k], wide[1][:, :k])
    z = x.double() @ w.double().t()
    bound = (k + 8) * 2.0 ** -24 * (x.double().abs() @ w.double().abs().t())
    assert ((got.double() - z).abs() <= bound + 2.0 ** -8 * (z.abs() + bound)).all()

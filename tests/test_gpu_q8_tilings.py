"""Products in 8 bits: every tiling, with and without splits of the contraction, at sizes that end inside its tiles; NaN in one row reaches no other."""
import math

import pytest
import torch

from paper_2506_00812_amd import binding as vf
from .test_gpu_q8 import check, made

pytestmark = pytest.mark.gpu
F32, BF, HF = torch.float32, torch.bfloat16, torch.float16
CODE = {F32: vf.VF_F32, BF: vf.VF_BF16, HF: vf.VF_F16}

# dtype, m, n, k, gated, quantized: tiling, whether the contraction is split
CASES = [
    (F32, 63, 101, 300, 0, 0, 0, False), (F32, 63, 101, 300, 1, 1, 0, True), (BF, 17, 99, 300, 1, 0, 0, False), (HF, 33, 333, 1000, 0, 1, 0, True),
    (F32, 67, 101, 100, 1, 1, 1, False), (F32, 67, 101, 2100, 1, 1, 1, True), (BF, 130, 301, 100, 1, 1, 1, False), (HF, 67, 101, 2100, 1, 1, 1, True),
    (F32, 67, 101, 100, 0, 0, 2, False), (F32, 67, 101, 4096, 0, 0, 2, True), (F32, 131, 77, 200, 1, 0, 2, False), (F32, 67, 101, 4096, 1, 0, 2, True),
    (BF, 67, 101, 300, 0, 0, 2, False), (HF, 67, 101, 4096, 0, 0, 2, True), (HF, 131, 77, 200, 1, 0, 2, False), (BF, 67, 101, 4096, 1, 0, 2, True),
    (F32, 4999, 777, 100, 0, 0, 3, False), (F32, 67, 101, 100, 0, 1, 3, False), (F32, 67, 101, 2100, 0, 1, 3, True), (F32, 19999, 99, 100, 1, 0, 3, False),
    (BF, 9999, 1023, 100, 0, 0, 3, False), (BF, 67, 101, 300, 0, 1, 3, False), (HF, 67, 101, 4096, 0, 1, 3, True), (BF, 2999, 1499, 100, 1, 0, 3, False),
    (BF, 9999, 1499, 100, 0, 0, 4, False), (HF, 9999, 1499, 100, 0, 1, 4, False), (HF, 2999, 2099, 100, 1, 0, 4, False), (BF, 19999, 131, 100, 1, 1, 4, False),
    (HF, 9999, 777, 777, 0, 0, 5, False), (BF, 19999, 131, 4000, 0, 0, 5, True), (BF, 9999, 777, 777, 0, 1, 5, False), (BF, 4999, 777, 1024, 1, 0, 5, False),
    (BF, 19999, 131, 512, 1, 1, 5, False), (HF, 4999, 131, 4000, 1, 1, 5, True),
    (BF, 9999, 1499, 512, 0, 0, 6, False), (BF, 9999, 1499, 512, 0, 1, 6, False), (HF, 2999, 2099, 2100, 1, 0, 6, False), (BF, 2999, 2099, 2100, 1, 1, 6, False),
]


@pytest.mark.parametrize("T,m,n,k,gated,quantize,tiling,split", CASES)
def test_every_tiling(T, m, n, k, gated, quantize, tiling, split):
    taken = vf.debug_linear_q8(CODE[T], m, n, k, gated, quantize)
    assert taken[0] == tiling and (taken[1] > 0) == split, taken
    check(m, n, k, T, "silu" if gated else "none", gated=bool(gated), quantize=bool(quantize))
    heavy = vf.debug_linear_q8(CODE[T], m, n, k, gated, quantize, True)
    check(m, n, k, T, "gelu", gated=bool(gated), quantize=bool(quantize), residual=True, pad=heavy[0] % 2)


def test_the_list_has_them_all():
    """Tiling by whether sums are exact (float32), gated and in 8 bits."""
    seen = {(T == F32, gated, quantize, tiling) for T, _, _, _, gated, quantize, tiling, _ in CASES}
    assert {t for e, g, q, t in seen if not e and not g and not q} >= {2, 3, 4, 5, 6} and {t for e, g, q, t in seen if not e and not g and q} >= {3, 4, 5, 6}
    assert {t for e, g, q, t in seen if not e and g and not q} >= {0, 2, 3, 4, 5, 6} and {t for e, g, q, t in seen if not e and g and q} >= {1, 4, 5, 6}
    assert {(g, q, t) for e, g, q, t in seen if e} >= {(0, 0, 0), (1, 1, 0), (1, 1, 1), (0, 0, 2), (1, 0, 2), (0, 0, 3), (0, 1, 3), (1, 0, 3)}


@pytest.mark.parametrize("m,n,k,gated,quantize", [(67, 101, 300, 0, 0), (9999, 1023, 100, 0, 0), (9999, 1499, 100, 0, 1), (9999, 777, 777, 0, 0), (9999, 1499, 512, 0, 1),
                                                  (2999, 2099, 2100, 1, 1), (19999, 131, 100, 1, 1), (130, 301, 100, 1, 1)])
def test_rows_do_not_touch_each_other(m, n, k, gated, quantize):
    x, w = made(m, k, 1), vf.quantize(made(n * (1 + gated), k, 2, std=k ** -0.5))
    want = vf.linear_q8(vf.quantize(x), w, gated=bool(gated), quantize=bool(quantize))
    at = [0, m // 2 + 5, m - 1]
    x[at, k - 1] = math.nan
    got = vf.linear_q8(vf.quantize(x), w, gated=bool(gated), quantize=bool(quantize))
    if quantize:
        want, got = vf.dequantize(want, F32), vf.dequantize(got, F32)
    keep = torch.ones(m, dtype=torch.bool, device="cuda")
    keep[at] = False
    assert torch.equal(got[keep], want[keep]) and torch.isnan(got[at]).all()

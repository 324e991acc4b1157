"""Products in 8 bits whose outputs are in 8 bits, in every tiling: the sums that are rounded to a code are exact where float32 is.

The matrix cores' own products of codes drop what lies 2^-13 below the largest of eight neighbours: 2^16 + 2^2 is 2^16 to them.  Here each block of 128 columns has
2^16 and 2^2 side by side and -2^16 elsewhere, so that only the small products are left of a sum.  All partial sums stay below 2^24: float32 holds them."""
import pytest
import torch

from paper_2506_00812_amd import binding as vf
from .test_gpu_more_ops_exact import generator
from .test_gpu_q8 import held
from .test_gpu_q8_tilings import BF, CASES, CODE, F32, HF

pytestmark = pytest.mark.gpu


def planted(m, n, k, seed):
    """x, w float32: 256 and 2 among the first eight of each block, 256 again behind them where w has -256; the twos' signs are drawn."""
    g = generator(seed)
    x, w = torch.zeros((m, k), device="cuda"), torch.zeros((n, k), device="cuda")
    for c in range(0, k - 9, 128):
        big, small = 1 + c // 128 % 7, c // 128 % 7 // 6
        x[:, [c + big, c + 9]], w[:, c + big], w[:, c + 9] = 256.0, 256.0, -256.0
        for t in (x, w):
            t[:, c + small] = 4.0 * torch.randint(0, 2, (len(t),), generator=g, device="cuda") - 2
    return x, w


@pytest.mark.parametrize("T,m,n,k,gated,tiling,split", [(T, m, n, k, g, t, s) for T, m, n, k, g, q, t, s in CASES if q] +
                         [(BF, 1, 333, 1000, 0, 0, True), (HF, 16, 333, 1000, 1, 0, True), (F32, 1, 99, 300, 1, 0, True)])
def test_small_products_beside_large_ones(T, m, n, k, gated, tiling, split):
    taken = vf.debug_linear_q8(CODE[T], m, n, k, gated, 1)
    assert taken[0] == tiling and (taken[1] > 0) == split, taken
    x, w = planted(m, n * (1 + gated), k, m + n + k)
    z = x.double() @ w.double().t()
    assert z.abs().max() <= 4 * -(-k // 128)
    for act in ("none", "relu"):
        values, byte = held((z[:, :n].clamp_min(0) if act == "relu" else z[:, :n]) * z[:, n:] if gated else z.clamp_min(0) if act == "relu" else z)
        y = vf.linear_q8(vf.quantize(x), vf.quantize(w), activation=act, gated=bool(gated), dtype=T, quantize=True)
        assert torch.equal(vf.dequantize(y, F32).double(), values) and torch.equal(y.scales[:, :byte.shape[1]], byte)

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


@pytest.mark.parametrize("T", [F32, BF, HF])
@pytest.mark.parametrize("m,n,k,gated", [(5, 100, 300, 0), (130, 301, 700, 1), (1500, 1000, 256, 0), (2999, 2099, 640, 1), (9999, 777, 777, 0), (9999, 1499, 512, 0)])
def test_scales_of_the_callers_own(T, m, n, k, gated):
    """Scales whose powers cancel leave the outputs as they are; 255 is NaN for its row of x, or of w, and for no other one."""
    x, w = (vf.quantize(torch.randn((r, k), generator=generator(r), device="cuda")) for r in (m, n * (1 + gated)))
    x.scales.fill_(127)
    w.scales.fill_(127)
    call = lambda: vf.linear_q8(x, w, gated=bool(gated), dtype=T, quantize=True)   # noqa: E731
    want = call()
    for byte in (16, 238):
        x.scales.fill_(byte)
        w.scales.fill_(254 - byte)
        got = call()
        assert torch.equal(got.codes.view(torch.uint8), want.codes.view(torch.uint8)) and torch.equal(got.scales[:, :-(-n // 128)], want.scales[:, :-(-n // 128)]), byte
    x.scales.fill_(127)
    w.scales.fill_(127)
    x.scales[m // 2, 1], w.scales[n - 3, 0] = 255, 255
    got = call()
    lost = torch.zeros((m, n), dtype=torch.bool, device="cuda")
    lost[m // 2] = True
    lost[:, n - 3] = True
    values = vf.dequantize(got, F32)
    assert torch.equal(values.isnan(), lost)
    apart = torch.arange(n, device="cuda") // 128 != (n - 3) // 128     # blocks whose scale cannot have moved
    keep = torch.arange(m, device="cuda") != m // 2
    assert torch.equal(values[keep][:, apart], vf.dequantize(want, F32)[keep][:, apart])

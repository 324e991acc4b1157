"""Up to 64 rows in 8 bits, on both sides of where they leave the kernel of few rows for tiles: long contractions and many outputs.  The bounds are those of
any other size."""
import pytest
import torch

from paper_2506_00812_amd import binding as vf
from .test_gpu_q8 import check

pytestmark = pytest.mark.gpu
CODE = {torch.float32: vf.VF_F32, torch.bfloat16: vf.VF_BF16, torch.float16: vf.VF_F16}
SIZES = [(1, 333, 1000), (1, 77, 16500), (1, 33333, 600), (16, 99, 16500), (17, 20001, 130), (33, 5000, 2000), (48, 200, 4100), (64, 20001, 300), (64, 65, 8000)]


@pytest.mark.parametrize("gated,quantize", [(False, False), (False, True), (True, False), (True, True)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_small_batches(m, n, k, dtype, gated, quantize):
    check(m, n, k, dtype, act="silu", gated=gated, quantize=quantize)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_both_sides(dtype):
    taken = {(m, n, k): vf.debug_linear_q8(CODE[dtype], m, n, k, False, False)[0] for m, n, k in SIZES}
    assert taken[1, 333, 1000] == 0 and taken[64, 65, 8000] > 0 and taken[64, 20001, 300] > 0

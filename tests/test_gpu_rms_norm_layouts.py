"""Root-mean-square norms on either side of every length at which a row gets more threads, for one row, a few, and more than work at the same time."""
import pytest
import torch

from .ops_util import DTYPES
from .test_gpu_rms_norm import check_backward, check_forward

pytestmark = pytest.mark.gpu
EDGES = [128, 256, 512, 1024, 2048, 4096, 8192, 16384]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [e + more for e in EDGES for more in (0, 1)] + [1500, 6100, 12008])
def test_lengths(d, dtype):
    for m in (1, 2, 3, 9):
        check_forward(m, d, dtype)
        check_backward(m, d, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,d", [(5003, 300), (4999, 1025), (2500, 2049), (1300, 4097), (700, 9000)])
def test_more_rows_than_workgroups(m, d, dtype):
    check_forward(m, d, dtype, pad=1)
    check_backward(m, d, dtype, pad=1)

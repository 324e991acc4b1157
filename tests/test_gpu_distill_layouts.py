"""Divergence from a teacher on either side of the lengths and counts of rows at which a row gets more threads, or segments."""
import pytest

from .ops_util import DTYPES
from .test_gpu_distill import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,v,top", [(1023, 2048, 8), (1023, 2049, 8), (1024, 2049, 8), (1500, 6144, 70), (1500, 6145, 70), (1023, 6144, 3), (1, 2048, 64), (1, 2049, 65),
                                     (2, 4097, 256), (600, 8193, 64)])
def test_layouts(m, v, top, dtype):
    check(m, v, top, dtype)
    check(m, v, top, dtype, pad=3)

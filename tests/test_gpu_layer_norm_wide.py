"""Layer norm of rows that several waves share, with more rows than the backward pass has workgroups (512 to 1,024): the sums over a
workgroup's rows, and the row sums' memory used again.  Bounds of test_gpu_layer_norm."""
import pytest
import torch

from paper_2506_00812_amd import binding as vf
from .ops_util import DTYPES
from .test_gpu_layer_norm import check_backward, check_forward, inputs

pytestmark = pytest.mark.gpu

# rows of 257 to 512, 513 to 1,024 and 1,025 to 2,048 vectors of 16 bytes, and of more; lengths that end inside a vector
VECTORS = [257, 400, 700, 1024, 1025, 2048, 2060]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vectors", VECTORS)
def test_more_rows_than_workgroups(vectors, dtype):
    per = 4 if dtype == torch.float32 else 8
    check_backward(1300, vectors * per, dtype)
    check_backward(1029, vectors * per - 3, dtype, pad=8)
    check_forward(1029, vectors * per - 3, dtype, pad=3)


def test_many_more_rows():
    check_backward(20000, 2056, torch.bfloat16)
    check_forward(20000, 2056, torch.bfloat16)


@pytest.mark.parametrize("d", [2056, 5000, 16384])
def test_repeats_and_partial_gradients(d):
    x, w, b, dy = inputs(1300, d, torch.bfloat16, 5)
    _, mu, rs = vf.layer_norm(x, w, b, save=True)
    full = vf.layer_norm_backward(dy, x, mu, rs, w)
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(vf.layer_norm_backward(dy, x, mu, rs, w), full))
    assert torch.equal(vf.layer_norm_backward(dy, x, mu, rs, w, dweight=False, dbias=False)[0], full[0])
    got = vf.layer_norm_backward(dy, x, mu, rs, w, dx=False)
    assert torch.equal(got[1], full[1]) and torch.equal(got[2], full[2])
    assert torch.equal(vf.layer_norm_backward(dy, x, mu, rs, w, out=dy)[0], full[0])

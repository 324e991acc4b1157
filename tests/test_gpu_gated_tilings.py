"""The gated layer in every tiling, with and without splits of the contraction, at sizes that end inside its tiles, and on both sides of the border between few
rows and tiles.  Each case says which tiling it takes."""
import pytest
import torch

from paper_2506_00812_amd import binding as vf
from .test_gpu_gated_linear import check_forward
from .test_gpu_more_ops_exact import generator, whole

pytestmark = pytest.mark.gpu
F32, BF, HF = torch.float32, torch.bfloat16, torch.float16
CODE = {F32: vf.VF_F32, BF: vf.VF_BF16, HF: vf.VF_F16}

# dtype, m, n, k, rows that start on 16 bytes: tiling, whether the contraction is split
CASES = [
    (F32, 9, 41, 201, 0, 0, False), (F32, 91, 11, 23, 0, 1, False), (F32, 1, 9, 2249, 0, 1, True), (F32, 65, 777, 8192, 0, 2, True), (F32, 1623, 1429, 17, 0, 2, False),
    (F32, 9645, 41, 1181, 0, 2, True), (BF, 9, 41, 203, 0, 0, False), (BF, 129, 11, 17, 0, 1, False), (HF, 1, 17, 3063, 0, 1, True), (BF, 1009, 2295, 21, 0, 2, False),
    (BF, 139, 2937, 4045, 0, 2, True), (BF, 65, 9, 24, 1, 1, False), (BF, 1, 11, 6584, 1, 1, True), (BF, 801, 2629, 16, 1, 2, False), (HF, 1679, 1337, 24, 1, 2, False),
    (BF, 7035, 645, 40, 1, 3, False), (BF, 75, 433, 7496, 1, 3, True), (HF, 67, 2163, 1960, 1, 3, True), (BF, 4187, 1569, 24, 1, 4, False), (BF, 153, 3643, 7784, 1, 4, True),
    (HF, 225, 2991, 8152, 1, 4, True), (BF, 3975, 1187, 72, 1, 5, False), (BF, 265, 3373, 6696, 1, 5, True), (HF, 5541, 69, 6824, 1, 5, True), (BF, 8079, 857, 104, 1, 6, False),
    (BF, 735, 3205, 6136, 1, 6, True), (HF, 763, 2853, 5704, 1, 6, True),
    # few rows and tiles: on both sides of a border
    (BF, 32, 4097, 104, 1, 0, False), (BF, 33, 2817, 104, 1, 1, False), (BF, 33, 2801, 104, 1, 0, False), (F32, 33, 11409, 100, 0, 0, False), (F32, 33, 11425, 100, 0, 1, False),
    (BF, 16, 1009, 4096, 1, 1, True), (BF, 16, 1025, 4096, 1, 0, False), (F32, 16, 1009, 4096, 0, 1, True), (F32, 16, 1025, 4096, 0, 0, False),
]


@pytest.mark.parametrize("T,m,n,k,direct,tiling,split", CASES)
def test_every_tiling(T, m, n, k, direct, tiling, split):
    taken = vf.debug_gated_linear(CODE[T], m, n, k, "relu", direct)
    assert taken[0] == tiling and (taken[1] > 1) == split, taken
    check_forward(m, n, k, T, "relu")
    g = generator(m + n + k)     # whole numbers: each term counts, sums are exact in any order
    x, w, b = (whole(g, *s, most=1).to(T) for s in ((m, k), (2 * n, k), (2 * n,)))
    y, z = vf.gated_linear(x, w, b, activation="none", save=True)
    want = x.double() @ w.double().t() + b.double()
    assert torch.equal(z, want.to(T)) and torch.equal(y, (want[:, :n] * want[:, n:]).float().to(T))
    assert torch.equal(vf.gated_linear(x, w, b, activation="none"), y)
    heavy = vf.debug_gated_linear(CODE[T], m, n, k, "silu", direct)
    if heavy != taken:
        check_forward(m, n, k, T, "silu")


def test_the_list_has_them_all():
    seen = {(T == F32, tiling, split) for T, *_, tiling, split in CASES}
    assert seen >= {(True, 0, False)} | {(True, t, s) for t in (1, 2) for s in (False, True)}
    assert seen >= {(False, 0, False)} | {(False, t, s) for t in range(1, 7) for s in (False, True)}


def test_slices_of_a_wider_matrix():
    """Rows that start on 16 bytes and others, where the tiling differs: a caller's x cut out of a table."""
    for pad in (3, 8, 16):
        check_forward(700, 1000, 264, BF, "silu", pad=pad)
        check_forward(75, 433, 7496, HF, "gelu", pad=pad)

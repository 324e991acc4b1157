"""Products of too many output tiles, without a GPU: tilings that cannot take them are passed over, and what none can take is refused."""
import pytest

from paper_2506_00812_amd import binding
from .test_abi_ops import BF16, F32, P, lib  # noqa: F401

TILE = {1: (64, 64), 2: (128, 128), 3: (128, 128), 4: (128, 256), 5: (256, 192), 6: (256, 256)}     # rows of the first and the second operand
LIMIT = 1 << 22


def tiles(tiling, rows_p, rows_q):
    return -(-rows_p // TILE[tiling][0]) * -(-rows_q // TILE[tiling][1])


@pytest.mark.parametrize("dtype", [F32, BF16, binding.VF_F16])
def test_tilings_that_fit_are_taken(lib, dtype):  # noqa: F811
    for m, n, k in (((1 << 28) + 65, 1, 1), ((1 << 28) + 65, 60, 8), (1 << 22, 8192, 8), (9_000_000, 4096, 16), ((1 << 29) - 500, 64, 64)):
        for product, sides in ((0, (n, m)), (1, (k, m)), (2, (k, n))):
            for direct in (False, True):
                if tiles(2, *sides) >= LIMIT and (not direct or dtype == F32):
                    continue
                tiling, splits = binding.debug_linear(dtype, m, n, k, product, direct)
                assert tiling == 0 or tiles(tiling, *sides) * splits < LIMIT, (m, n, k, product, direct, tiling)


def test_what_no_tiling_takes(lib):  # noqa: F811
    m, n, k = 1 << 30, 64, 64
    for product in (0, 1):
        with pytest.raises(binding.VecflowError, match="output tiles"):
            binding.debug_linear(F32, m, n, k, product, False)
    assert binding.debug_linear(F32, m, n, k, 2, False)[0] in TILE
    for dx, dw, act in ((P, None, 0), (P, P, 2)):
        rc = lib.vf_linear_backward(BF16, m, n, k, P, n, P, k, P, k, P, n, act, dx, k, dw, k, P, P, 1 << 50, None)
        assert rc == -1 and b"output tiles" in lib.vf_last_error()
    rc = lib.vf_linear(BF16, m, n, k, P, k, P, k, None, 0, None, 0, P, n, None, 0, P, 1 << 50, None)
    assert rc == -1 and b"output tiles" in lib.vf_last_error()

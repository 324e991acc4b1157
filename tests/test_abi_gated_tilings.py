"""Which tiling the gated layer takes, asked without a GPU; bad arguments of the question."""
import ctypes as C

import pytest

from paper_2506_00812_amd import binding
from .test_abi_ops import BF16, F32, lib  # noqa: F401


def test_few_rows_or_tiles(lib):  # noqa: F811
    """Up to 64 rows: the kernel of few rows, but for short contractions of many outputs and long ones of few."""
    for dtype in (F32, BF16, binding.VF_F16):
        for m in (1, 16, 32, 64):
            assert binding.debug_gated_linear(dtype, m, 1024, 1024) == (0, 1)
        assert binding.debug_gated_linear(dtype, 33, 65536, 100) == (1, 1)
        assert binding.debug_gated_linear(dtype, 32, 65536, 100) == (0, 1)
        tiling, splits = binding.debug_gated_linear(dtype, 32, 1024, 4096)
        assert tiling == 1 and splits > 1
        assert binding.debug_gated_linear(dtype, 65, 1024, 1024)[0] > 0


def test_refusals(lib):  # noqa: F811
    a, b = C.c_int32(), C.c_int32()
    ask = lambda *v: lib.vf_debug_gated_linear(*v)   # noqa: E731
    assert ask(F32, 4, 8, 16, 3, 0, C.byref(a), C.byref(b)) == 0
    for bad in ((0, 4, 8, 16, 3, 0), (F32, -1, 8, 16, 3, 0), (F32, 4, (1 << 24) + 1, 16, 3, 0), (F32, 4, 8, -1, 3, 0), (F32, 4, 8, 16, 4, 0)):
        assert ask(*bad, C.byref(a), C.byref(b)) == -1 and b"gated linear" in lib.vf_last_error()
    assert ask(F32, 4, 8, 16, 3, 0, None, C.byref(b)) == -1 and ask(F32, 4, 8, 16, 3, 0, C.byref(a), None) == -1
    with pytest.raises(binding.VecflowError, match="output tiles"):
        binding.debug_gated_linear(BF16, (1 << 31) - 1, 1 << 24, 8)

"""Helpers shared by the tests of the encoder operators: types with their unit roundoffs, rows inside wider matrices, bounds."""
import math

import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -24}     # what an output may lose below the normal range
DTYPES = (torch.float32, torch.bfloat16, torch.float16)


def cut(t, pad):
    """The same values as rows of a wider matrix that is NaN elsewhere."""
    wide = torch.full((t.shape[0] + 2, t.shape[1] + pad), math.nan, dtype=t.dtype, device=t.device)
    lead = pad // 2
    wide[1:-1, lead:lead + t.shape[1]] = t
    return wide[1:-1, lead:lead + t.shape[1]]


def within(got, want, tol, what):
    assert got.shape == want.shape
    off = (got.double() - want).abs() - tol
    assert not torch.isnan(off).any() and (off <= 0).all(), f"{what}: {off.max().item():.3g} beyond the bound"

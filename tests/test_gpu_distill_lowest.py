"""Labels masked by their type's lowest number instead of -inf: probability 0 beside others; a row of nothing else has the loss of equal logits and, where the
sum of its exponentials no longer says how many they are, no gradient."""
import math

import pytest
import torch

from paper_2506_00812_amd import binding as vf

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", [1.0, 2.0])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("v", [100, 5000])
def test_lowest_numbers(v, dtype, t):
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x = torch.randn((4, v), generator=g, device="cuda").to(dtype)
    masked = torch.rand((4, v), generator=g, device="cuda") < 0.5
    masked[:, :8] = False
    masked[1] = True
    x[masked] = torch.finfo(dtype).min
    ids = torch.arange(8, device="cuda", dtype=torch.int32).repeat(4, 1)
    teacher = torch.randn((4, 8), generator=g, device="cuda")
    loss, lse = vf.distill(x, ids, teacher, temperature=t)
    dx = vf.distill_backward(x, lse, ids, teacher, torch.ones(4, device="cuda"), temperature=t)
    infinite = x.masked_fill(masked, -math.inf)
    want, want_lse = vf.distill(infinite, ids, teacher, temperature=t)
    want_dx = vf.distill_backward(infinite, want_lse, ids, teacher, torch.ones(4, device="cuda"), temperature=t)
    rows = [0, 2, 3]
    assert torch.equal(loss[rows], want[rows]) and torch.equal(lse[rows], want_lse[rows]) and torch.equal(dx[rows], want_dx[rows])
    q = torch.softmax(teacher[1].double() / t, 0)
    equal = (q * (q.log() + math.log(v))).sum()
    # log q and log p are off by some 2^-21 of themselves, the sum of v terms of 1 is exact; (x - max) is 0
    assert abs(loss[1].double() - equal) <= 2.0 ** -20 * (q * (q.log().abs() + math.log(v) + 1)).sum()
    if dtype != torch.float16:
        assert not dx[1].any()

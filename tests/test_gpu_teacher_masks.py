"""A teacher that names labels which its student cannot give (`absent`): those entries are none, the others' probabilities are taken among themselves."""
import math

import pytest
import torch

from paper_2506_00812_amd import binding as vf
from paper_2506_00812_amd.query_encoder import QueryEncoder
from .test_gpu_query_encoder import batch

pytestmark = pytest.mark.gpu
ABSENT = [2, 5]


def entries(m):
    """Labels 0 .. 3 and 4 .. 7 in turn with values of their own, so that each row names one label that is absent; row 1 names no other ones."""
    ids = (torch.arange(4, device="cuda")[None, :] + 4 * (torch.arange(m, device="cuda")[:, None] % 2)).int().contiguous()
    ids[1] = torch.tensor([5, 2, 5, -1], device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    return ids, torch.randn((m, 4), generator=g, device="cuda")


@pytest.mark.parametrize("gated", [True, False])
def test_gradients_against_a_float64_model(gated):
    """Against torch's own differentiation in 64 bits on the CPU; up to ten float32 operators with sums of up to 96 terms, errors of some
    100 x 2^-24 of the largest gradient: 2e-5.  What belongs to an absent label has no gradient at all."""
    enc = QueryEncoder(24, 12, 10, hidden=48, dtype=torch.float32, gated=gated, absent=ABSENT)
    x, y, _ = batch(16, 24, 12, 10)
    none = torch.full((16,), -1, dtype=torch.int32, device="cuda")
    ids, val = entries(16)
    kept = ids.clone(), val.clone()
    loss, grads = enc.gradients(x, y, none, teacher=(ids, val), teacher_weight=1.5, temperature=2.0)
    assert torch.equal(ids, kept[0]) and torch.equal(val, kept[1])     # the caller's own
    p = {k: v.double().cpu().requires_grad_() for k, v in enc.params.items()}
    X, Y = x.double().cpu(), y.double().cpu()
    if gated:
        rms = lambda v, w: v * (v.square().mean(1, keepdim=True) + 1e-6).rsqrt() * w   # noqa: E731
        u = rms(X, p["n1w"]) @ p["w1"].t() + p["b1"]
        g = rms(X + u[:, :48] * torch.special.expit(u[:, :48]) * u[:, 48:] @ p["w2"].t() + p["b2"], p["n2w"])
    else:
        ln = lambda v, w, b: torch.nn.functional.layer_norm(v, (24,), w, b)   # noqa: E731
        u = ln(X, p["n1w"], p["n1b"]) @ p["w1"].t() + p["b1"]
        g = ln(X + u * torch.special.ndtr(u) @ p["w2"].t() + p["b2"], p["n2w"], p["n2b"])
    live = [i for i in range(10) if i not in ABSENT]
    log_p = torch.log_softmax((g @ p["wl"][live].t() + p["bl"][live]) / 2, 1)
    apart = []
    for row, (names, values) in enumerate(zip(ids.tolist(), val.double().cpu())):
        at = [j for j, name in enumerate(names) if name in live]
        if not at:
            apart.append(log_p.new_zeros(()))
            continue
        log_q = torch.log_softmax(values[at] / 2, 0)
        apart.append((log_q.exp() * (log_q - log_p[row, [live.index(names[j]) for j in at]])).sum())
    want = ((g @ p["wv"].t() + p["bv"] - Y) ** 2).sum(1).mean() + 1.5 * torch.stack(apart).mean()
    want.backward()
    assert math.isfinite(loss.item()) and abs(loss.item() - want.item()) < 2e-5 * abs(want.item())
    for k, v in p.items():
        assert (grads[k].double().cpu() - v.grad).abs().max() <= 2e-5 * v.grad.abs().max(), k
    assert not grads["wl"][ABSENT].any() and not grads["bl"][ABSENT].any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_steps_stay_finite(dtype):
    enc = QueryEncoder(24, 12, 10, hidden=48, dtype=dtype, gated=True, absent=torch.tensor(ABSENT))
    big = QueryEncoder(24, 12, 10, dtype=dtype, seed=3)     # without the mask
    x, y, t = batch(64, 24, 12, 10)
    t[(t == 2) | (t == 5)] = -1
    rows = enc.params["wl"][ABSENT].clone()
    for _ in range(3):
        _, ids, logp, _ = big.encode(x.to(dtype), top=10)
        assert (ids == 2).any() and (ids == 5).any()
        assert torch.isfinite(enc.train_step(x.to(dtype), y, t, weight_decay=0.0, teacher=(ids, logp)))
    assert torch.equal(enc.params["wl"][ABSENT], rows)


def test_what_is_no_label_is_still_refused_or_nan():
    enc = QueryEncoder(24, 12, 10, hidden=48, dtype=torch.float32, absent=ABSENT)
    x, y, t = batch(6, 24, 12, 10)
    t[:] = -1
    ids, val = entries(6)
    for bad in ((ids.long(), val), (ids[:3], val[:3]), (ids.cpu(), val), (ids[:, :0], val[:, :0]), (ids, val.half())):
        with pytest.raises(vf.VecflowError):
            enc.gradients(x, y, t, teacher=bad)
    for name in (10, -2):
        wrong = ids.clone()
        wrong[3, 1] = name
        assert math.isnan(enc.gradients(x, y, t, teacher=(wrong, val))[0].item())

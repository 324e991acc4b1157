"""The query encoder where its batches and types are at their edges."""
import pytest
import torch

from paper_2506_00812_amd.query_encoder import QueryEncoder
from .test_gpu_query_encoder import batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_a_batch_of_nothing(dtype):
    enc = QueryEncoder(24, 12, 10, hidden=48, dtype=dtype)
    x, y, t = batch(4, 24, 12, 10)
    before = {k: v.clone() for k, v in enc.params.items()}
    loss, grads = enc.gradients(x[:0].to(dtype), y[:0], t[:0], entropy_weight=0.1)
    assert loss.item() == 0 and all(g.shape == enc.params[k].shape and not g.any() for k, g in grads.items())
    enc.train_step(x[:0].to(dtype), y[:0], t[:0], weight_decay=0.0)
    assert all(torch.equal(enc.params[k], v) for k, v in before.items())
    vectors, ids, logp, entropy = enc.encode(x[:0].to(dtype), top=3)
    assert vectors.shape == (0, 12) and ids.shape == logp.shape == (0, 3) and entropy.shape == (0,)


def test_float16_keeps_small_gradients():
    """10,000 queries and 10,000 labels: most entries of the logits' gradient, some 1e-8, are below float16's range.  They are carried
    times a scale, so their sum over the labels stays the targets' (an exact gradient's sum is 0): each of the m v entries rounds by 2^-11 of
    itself, all of them 2 in sum, or by 2^-25 / scale, 1e8 of them; the model in float32 has the same gradients but for what roundings
    of activations, weights and a chain of some ten float16 operands do to them, 2^-11 sqrt(10) of a gradient's size, here 8 times as much."""
    enc = QueryEncoder(64, 16, 10_000, dtype=torch.float16)
    ref = QueryEncoder(64, 16, 10_000, dtype=torch.float32)
    ref.params = {k: v.float() for k, v in enc.params.items()}
    x, y, t = batch(10_000, 64, 16, 10_000)
    x = x.half()
    for weight in (1.0, 0.25):
        _, got = enc.gradients(x, y, t, label_weight=weight)
        _, want = ref.gradients(x.float(), y, t, label_weight=weight)
        assert abs(got["bl"].double().sum().item()) <= weight * 2 * 2.0 ** -11 + 1e8 * 2.0 ** -25 / 1024 + 2.0 ** -10
        for k, g in got.items():
            assert (g.double() - want[k].double()).norm() <= 8 * 10 ** 0.5 * 2.0 ** -11 * want[k].double().norm(), k


def test_float16_steps_that_overflow_change_nothing():
    """Targets so far away that a scaled gradient passes 65,504: the step is left out and the scale halved until one fits."""
    enc = QueryEncoder(24, 12, 10, hidden=48, dtype=torch.float16)
    x, y, t = batch(16, 24, 12, 10)
    y = y * 300
    before = {k: v.clone() for k, v in enc.params.items()}
    scales, changed = [], []
    for _ in range(12):
        scales.append(enc.scale.item())
        enc.train_step(x.half(), y, t)
        changed.append(any(not torch.equal(enc.params[k], v) for k, v in before.items()))
        assert all(torch.isfinite(p).all() for p in enc.params.values())
    assert not changed[0] and changed[-1]
    first = changed.index(True)
    assert scales[:first + 1] == [scales[0] / 2 ** i for i in range(first + 1)] and set(scales[first:]) == {scales[first]}


def test_float16_scale_grows_again():
    enc = QueryEncoder(24, 12, 10, hidden=48, dtype=torch.float16)
    x, y, t = batch(16, 24, 12, 10)
    start = enc.scale.item()
    for _ in range(enc.GROWTH_STEPS):
        assert enc.scale.item() == start
        enc.train_step(x.half(), y, t, lr=1e-4)
    assert enc.scale.item() == 2 * start


def test_other_types_have_no_scale():
    for dtype in (torch.float32, torch.bfloat16):
        enc = QueryEncoder(24, 12, 10, hidden=48, dtype=dtype)
        x, y, t = batch(16, 24, 12, 10)
        _, grads = enc.gradients(x.to(dtype), y, t)
        assert enc.scale is None and all(g.dtype == dtype for g in grads.values())


def test_no_labels_asked_for():
    enc = QueryEncoder(24, 12, 10, hidden=48, dtype=torch.float32)
    x, _, _ = batch(16, 24, 12, 10)
    vectors, ids, logp, entropy = enc.encode(x, top=0)
    want = enc.encode(x, top=2)
    assert ids.shape == logp.shape == (16, 0) and ids.dtype == torch.int32 and torch.equal(vectors, want[0])
    assert (entropy - want[3]).abs().max() < 1e-5

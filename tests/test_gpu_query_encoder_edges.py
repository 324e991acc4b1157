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

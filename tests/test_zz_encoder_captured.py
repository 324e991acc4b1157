"""Encoding captured into a graph: every replay says what the eager call says of the same queries, bit for bit, with eager work in between.  Among the last files
by its name, as test_zz_ops_streams.py: it makes streams."""
import pytest
import torch

from paper_2506_00812_amd.query_encoder import QueryEncoder

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("gated,in_8_bits", [(True, False), (False, True), (True, True)])
@pytest.mark.parametrize("m", [1, 300])
def test_encode_captured(m, gated, in_8_bits, dtype):
    e = QueryEncoder(256, 96, 500, dtype=dtype, gated=gated, seed=3)
    e = e.in_8_bits() if in_8_bits else e
    batches = [torch.randn((m, 256), device="cuda").to(dtype) for _ in range(4)]
    x = batches[0].clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        e.encode(x, top=3)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = e.encode(x, top=3)
    for batch in batches:
        want = e.encode(batch, top=3)
        x.copy_(batch)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))

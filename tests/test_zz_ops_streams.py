"""The encoder operators on streams of the caller's and in graphs.

The last file of the GPU tests by its name: the streams that it makes share the process's few hardware queues with those of serving
sessions, whose tests count on kernels of other streams to run beside theirs."""
import pytest
import torch

from paper_2506_00812_amd import binding as vf
from .test_gpu_layer_norm import inputs as norm_inputs
from .test_gpu_linear import inputs as linear_inputs
from .test_gpu_log_probs import make

pytestmark = pytest.mark.gpu


def test_linear_on_another_stream():
    """Work on a stream of the caller's: the same results, its memory returned in that stream's order."""
    x, w, b, r = linear_inputs(600, 500, 300, torch.bfloat16, 11)
    y, z = vf.linear(x, w, b, activation="gelu", save=True)
    want = vf.linear_backward(r, x, w, z=z, activation="gelu")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = [vf.linear_backward(r, x, w, z=z, activation="gelu", stream=s) for _ in range(4)]
    s.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


def test_linear_in_a_graph():
    x, w, b, r = linear_inputs(64, 128, 2048, torch.bfloat16, 13)
    out = torch.empty((64, 128), dtype=torch.bfloat16, device="cuda")
    vf.linear(x, w, b, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        vf.linear(x, w, b, out=out)
        dx, dw, db = vf.linear_backward(out, x, w)
    for i in range(4):
        x.copy_(torch.randn(64, 2048, device="cuda").to(torch.bfloat16))
        g.replay()
        torch.cuda.synchronize()
        y = vf.linear(x, w, b)
        assert torch.equal(out, y)
        assert all(torch.equal(p, q) for p, q in zip((dx, dw, db), vf.linear_backward(y, x, w)))


def test_layer_norm_on_another_stream_and_in_a_graph():
    x, w, b, dy = norm_inputs(500, 768, torch.bfloat16, 9)
    want = vf.layer_norm_backward(dy, x, *vf.layer_norm(x, w, b, save=True)[1:], w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y, mu, rs = vf.layer_norm(x, w, b, save=True, stream=s)
    got = vf.layer_norm_backward(dy, x, mu, rs, w, stream=s)
    s.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y, mu, rs = vf.layer_norm(x, w, b, save=True)
        out = vf.layer_norm_backward(dy, x, mu, rs, w)
    for i in range(4):
        x.copy_(torch.randn(500, 768, device="cuda").to(torch.bfloat16))
        g.replay()
        torch.cuda.synchronize()
        y2, mu2, rs2 = vf.layer_norm(x, w, b, save=True)
        assert torch.equal(y, y2) and all(torch.equal(p, q) for p, q in zip(out, vf.layer_norm_backward(dy, x, mu2, rs2, w)))


def test_log_probs_on_another_stream_and_in_a_graph():
    x, t = make(50, 4000, torch.bfloat16, 9)
    d = torch.randn(50, device="cuda")
    want = vf.log_probs(x, t, top=4)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = [vf.log_probs(x, t, top=4, stream=s) for _ in range(3)]
    s.synchronize()
    for o in got:
        assert all(torch.equal(p, q) for p, q in zip(o, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = vf.log_probs(x, t, top=4)
        dx = vf.log_probs_backward(x, out[2], t, d)
    for i in range(4):
        x.copy_(make(50, 4000, torch.bfloat16, 20 + i)[0])
        g.replay()
        torch.cuda.synchronize()
        now = vf.log_probs(x, t, top=4)
        assert all(torch.equal(p, q) for p, q in zip(out, now)) and torch.equal(dx, vf.log_probs_backward(x, now[2], t, d))


def test_adamw_on_another_stream():
    p, g = torch.ones(1000, device="cuda"), torch.ones(1000, device="cuda")
    m, v = vf.adamw_state(p)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    vf.adamw_step([p], [g], [m], [v], step=1, lr=0.1, stream=s)
    out = vf.adamw_moments([m], [v], stream=s)
    s.synchronize()
    assert ((p - 0.9).abs() < 1e-6).all() and torch.equal(out[0][0], m) and torch.equal(out[1][0], v)

"""The gated encoder's operators on streams of the caller's and in graphs, several of them with their workspaces in one pool.  Named to run last: see
test_zz_ops_streams.py."""
import pytest
import torch

from paper_2506_00812_amd import binding as vf
from .test_gpu_distill import make
from .test_gpu_linear import inputs as linear_inputs
from .test_gpu_q8 import made
from .test_gpu_rms_norm import inputs as norm_inputs

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def run(x, r, w, wg, bg, wd, ids, val, d, stream=None):
    """Forward, backward and the form in 8 bits, one after the other."""
    k = dict(stream=stream)
    a, total, rstd = vf.rms_norm(x, w, residual=r, save=True, **k)
    h, z = vf.gated_linear(a, wg, bg, save=True, **k)
    y = vf.linear(h, wd, residual=total, **k)
    loss, lse = vf.distill(y, ids, val, temperature=2.0, **k)
    dy = vf.distill_backward(y, lse, ids, val, d, temperature=2.0, **k)
    dh, dwd, _ = vf.linear_backward(dy, h, wd, **k)
    da, dwg, dbg = vf.gated_linear_backward(dh, a, wg, z, **k)
    dx, dw = vf.rms_norm_backward(da, total, rstd, w, d_total=dy, **k)
    a8, _ = vf.rms_norm(x, w, residual=r, quantize=True, **k)
    h8 = vf.linear_q8(a8, vf.quantize(wg, **k), bg, activation="silu", gated=True, quantize=True, dtype=BF, **k)
    y8 = vf.linear_q8(h8, vf.quantize(wd, **k), residual=total, **k)
    return y, loss, lse, dwd, dwg, dbg, dx, dw, y8, vf.dequantize(h8, BF, **k)


def setup(m, seed):
    x, r, w, _ = norm_inputs(m, 256, BF, seed)
    _, wg, bg, _ = linear_inputs(1, 2 * 520, 256, BF, seed + 1)
    wd = linear_inputs(1, 256, 520, BF, seed + 2)[1]
    _, ids, val = make(m, 256, 16, BF, seed + 3)
    return [x, r, w, wg, bg, wd, ids, val, torch.randn(m, device="cuda")]


def test_on_another_stream():
    for m in (3, 700):
        args = setup(m, 5)
        want = run(*args)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        got = [run(*args, stream=s) for _ in range(3)]
        s.synchronize()
        for g in got:
            assert all(torch.equal(a, b) for a, b in zip(g, want))


def test_two_graphs_replayed_in_turn_beside_eager_work():
    graphs = []
    pool = torch.cuda.graph_pool_handle()
    for m in (5, 300):
        args = setup(m, 20 + m)
        run(*args)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, pool=pool):
            out = run(*args)
        graphs.append((g, args, out))
    for i in range(4):
        for g, args, out in graphs:
            args[0].copy_(made(args[0].shape[0], 256, 30 + i).to(BF))
            g.replay()
            torch.cuda.synchronize()
            kept = [t.clone() for t in out]     # the other graph's memory is this one's
            assert all(torch.equal(a, b) for a, b in zip(kept, run(*args)))


def test_a_call_repeats_bit_for_bit():
    args = setup(1500, 9)
    want = run(*args)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(run(*args), want))


def test_few_rows_in_a_graph():
    x, w = vf.quantize(made(1, 1024, 1)), vf.quantize(made(4096, 1024, 2))
    b = torch.randn(4096, device="cuda").to(BF)
    vf.linear_q8(x, w, b, activation="gelu", quantize=True)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = vf.linear_q8(x, w, b, activation="gelu", quantize=True)
    for i in range(4):
        new = vf.quantize(made(1, 1024, 10 + i))
        x.codes.view(torch.uint8).copy_(new.codes.view(torch.uint8))
        x.scales.copy_(new.scales)
        g.replay()
        torch.cuda.synchronize()
        want = vf.linear_q8(x, w, b, activation="gelu", quantize=True)
        assert torch.equal(out.codes.view(torch.uint8), want.codes.view(torch.uint8)) and torch.equal(out.scales[:, :32], want.scales[:, :32])

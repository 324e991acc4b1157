"""The encoder operators' `stream` argument: the work waits for that stream and no other, memory is that stream's.  (By its name one of the
last files, as test_zz_ops_streams.)

The inputs are NaN on the default stream; a side stream that is busy for milliseconds makes them what they should be.  Work that was launched
anywhere else reads NaN."""
import pytest
import torch

from paper_2506_00812_amd import binding as vf
from .test_gpu_layer_norm import inputs as norm_inputs
from .test_gpu_linear import inputs as linear_inputs
from .test_gpu_log_probs import make

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def busy():
    a = torch.randn((8192, 8192), device="cuda").to(BF)
    return a, torch.empty_like(a)


def late(stream, busy, *tensors):
    """Empties the tensors on the current stream and has `stream` fill them again after some 10 ms of work."""
    kept = [t.clone() for t in tensors]
    for t in tensors:
        t.fill_(float("nan") if t.is_floating_point() else -9)
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for _ in range(12):
            torch.mm(busy[0], busy[0], out=busy[1])
        for t, k in zip(tensors, kept):
            t.copy_(k)
            k.record_stream(stream)


def stream_of(t):
    """The stream whose pool a tensor's memory is from."""
    at = t.data_ptr()
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= at < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not the allocator's memory")


@pytest.fixture
def side(monkeypatch):
    """A stream, and a check that workspaces come from its pool."""
    s = torch.cuda.Stream()
    seen = []
    make_workspace = vf._workspace

    def watched(like, nbytes, stream):
        t, at = make_workspace(like, nbytes, stream)
        if t is not None:
            seen.append((stream_of(t), None if stream is None else stream.cuda_stream))
        return t, at
    monkeypatch.setattr(vf, "_workspace", watched)
    yield s
    assert all(got == want for got, want in seen if want is not None)
    assert any(want is not None for _, want in seen) or getattr(s, "no_workspace", False)
    torch.cuda.synchronize()


def same(got, want, s):
    s.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g, w) and stream_of(g) == s.cuda_stream


def test_linear(side, busy):
    x, w, b, r = linear_inputs(600, 500, 4000, BF, 11)
    want = vf.linear(x, w, b, residual=r, activation="gelu", save=True)
    back = vf.linear_backward(r, x, w, z=want[1], activation="gelu")
    torch.cuda.synchronize()
    late(side, busy, x, w, b, r)
    got = vf.linear(x, w, b, residual=r, activation="gelu", save=True, stream=side)
    same(got, want, side)
    late(side, busy, x, w, r)
    same(vf.linear_backward(r, x, w, z=want[1], activation="gelu", stream=side), back, side)


def test_layer_norm(side, busy):
    x, w, b, dy = norm_inputs(500, 768, BF, 9)
    want = vf.layer_norm(x, w, b, save=True)
    back = vf.layer_norm_backward(dy, x, *want[1:], w)
    torch.cuda.synchronize()
    late(side, busy, x, w, b)
    same(vf.layer_norm(x, w, b, save=True, stream=side), want, side)
    late(side, busy, x, w, dy)
    same(vf.layer_norm_backward(dy, x, *want[1:], w, stream=side), back, side)


def test_log_probs(side, busy):
    x, t = make(50, 9000, BF, 9)
    d = torch.randn(50, device="cuda")
    want = vf.log_probs(x, t, top=4)
    grad = vf.log_probs_backward(x, want[2], t, d)
    torch.cuda.synchronize()
    late(side, busy, x, t)
    same(vf.log_probs(x, t, top=4, stream=side), want, side)
    late(side, busy, x, t, d)
    same([vf.log_probs_backward(x, want[2], t, d, stream=side)], [grad], side)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw(side, busy, bits):
    side.no_workspace = True
    p, g = torch.randn(3000, device="cuda"), torch.randn(3000, device="cuda")
    states = [vf.adamw_state(p, bits) for _ in range(2)]
    params = [p.clone(), p.clone()]
    outs = []
    for i, stream in enumerate((None, side)):
        st = states[i]
        if stream is not None:
            torch.cuda.synchronize()
            late(side, busy, g)
        scales = dict(m_scales=[st[2]], v_scales=[st[3]]) if bits == 8 else {}
        vf.adamw_step([params[i]], [g], [st[0]], [st[1]], step=1, lr=0.1, stream=stream, **scales)
        outs.append(vf.adamw_moments([st[0]], [st[1]], stream=stream, **scales))
    same([outs[1][0][0], outs[1][1][0]], [outs[0][0][0], outs[0][1][0]], side)
    assert torch.equal(params[0], params[1]) and torch.isfinite(params[1]).all()

"""CPU-side checks of the gated encoder's operators: bad arguments are refused before a GPU is touched, workspaces are stated, empty work needs
no device."""
import ctypes as C
import os
import re

import pytest

from paper_2506_00812_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P, Q, R = 1 << 30, 1 << 31, 1 << 32        # addresses that are never looked at, far from each other: validation fails first
F32, BF16 = binding.VF_F32, binding.VF_BF16


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2506_00812_amd.build import build
        build(verbose=False)
    return binding.load_library()


def caller(fn, **defaults):
    return lambda **kw: fn(*{**defaults, **kw}.values())


def test_constants_match_the_header():
    hdr = open(os.path.join(ROOT, "include", "vecflow.h")).read()
    for name, value in dict(VF_Q8_BLOCK=binding.Q8_BLOCK, VF_DISTILL_MAX_TOP=binding.DISTILL_MAX_TOP).items():
        assert int(re.search(r"#define %s (\d+)" % name, hdr).group(1)) == value


def test_gated_linear_refusals(lib):
    fwd = caller(lib.vf_gated_linear, dt=F32, m=4, n=8, k=16, x=P, ldx=16, w=Q, ldw=16, b=None, act=3, y=R, ldy=8, z=None, ldz=16, ws=None, nws=0, s=None)
    for kw in (dict(dt=0), dict(m=-1), dict(n=(1 << 24) + 1), dict(k=-2), dict(x=None), dict(w=None), dict(y=None), dict(ldx=15), dict(ldw=3), dict(ldy=7),
               dict(z=P + (1 << 20), ldz=15), dict(act=9), dict(m=1 << 32), dict(y=P), dict(y=Q + 8), dict(z=R), dict(b=R)):
        assert fwd(**kw) == -1, kw
        assert b"gated linear" in lib.vf_last_error()
    assert fwd(m=0) == 0 and fwd(n=0) == 0
    n = C.c_size_t(99)
    assert lib.vf_gated_linear_workspace(F32, 4, 8, 16, 3, 0, None) == -1
    assert lib.vf_gated_linear_workspace(F32, 0, 8, 16, 3, 0, C.byref(n)) == 0 and n.value == 0
    assert lib.vf_gated_linear_workspace(BF16, 2000, 512, 256, 3, 1, C.byref(n)) == 0 and n.value >= 2000 * 1024 * 2
    back = caller(lib.vf_gated_linear_backward, dt=BF16, m=2000, n=512, k=256, dy=P, lddy=512, x=Q, ldx=256, w=R, ldw=256, z=R + Q, ldz=1024, act=3, dx=2 * R,
                  lddx=256, dw=3 * R, lddw=256, db=4 * R, ws=5 * R, nws=n.value, s=None)
    for kw in (dict(dy=None), dict(z=None), dict(lddy=511), dict(ldz=1023), dict(w=None), dict(x=None), dict(lddx=255), dict(lddw=255), dict(ws=None), dict(nws=1000),
               dict(act=-1), dict(dt=0), dict(dx=P), dict(dw=Q), dict(db=P), dict(dx=3 * R), dict(ws=5 * R + 8)):
        assert back(**kw) == -1, kw


def test_too_many_tiles_are_refused(lib):
    """2^31 rows of 2^24 outputs are 2^40 elements of 128 x 128 tiles, before any work."""
    assert lib.vf_gated_linear(BF16, (1 << 31) - 1, 1 << 24, 8, P, 8, Q, 8, None, 3, R, 1 << 24, None, 0, None, 0, None) == -1
    assert b"tiles" in lib.vf_last_error()
    n = C.c_size_t(0)
    assert lib.vf_linear_quantized_workspace(BF16, (1 << 31) - 1, 1 << 24, 128, 0, 0, C.byref(n)) == 0
    assert lib.vf_linear_quantized(BF16, (1 << 31) - 1, 1 << 24, 128, P, 128, Q, 4, 1 << 45, 128, 1 << 46, 4, None, 0, 0, None, 0, 1 << 50, 1 << 24, None, 0, None, 0,
                            1 << 60, n.value, None) == -1
    assert b"tiles" in lib.vf_last_error()


def test_q8_refusals(lib):
    q = caller(lib.vf_quantize, dt=F32, m=3, d=200, x=P, ldx=200, c=Q, ld=256, sc=R, lds=4, s=None)
    for kw in (dict(dt=0), dict(m=-1), dict(d=(1 << 25) + 1), dict(x=None), dict(ldx=199), dict(c=None), dict(sc=None), dict(ld=200), dict(ld=264), dict(lds=1), dict(lds=6),
               dict(c=Q + 8), dict(sc=R + 2), dict(c=P), dict(sc=Q)):
        assert q(**kw) == -1, kw
    d = caller(lib.vf_dequantize, dt=F32, m=3, d=200, c=Q, ld=256, sc=R, lds=4, y=P, ldy=200, s=None)
    for kw in (dict(dt=9), dict(m=-1), dict(y=None), dict(ldy=199), dict(c=None), dict(ld=192), dict(y=Q), dict(y=R)):
        assert d(**kw) == -1, kw
    assert q(m=0) == 0 and d(m=0) == 0 and q(d=0) == 0
    n = C.c_size_t(0)
    assert lib.vf_linear_quantized_workspace(BF16, 300, 100, 200, 0, 0, None) == -1 and lib.vf_linear_quantized_workspace(BF16, 300, 100, 200, 0, 0, C.byref(n)) == 0
    p = caller(lib.vf_linear_quantized, dt=BF16, m=300, n=100, k=200, x=P, ldx=256, xs=P + (1 << 24), ldxs=4, w=Q, ldw=256, ws_=Q + (1 << 24), ldws=4, b=None, act=0, gated=0,
               r=None, ldr=100, y=R, ldy=100, yc=None, ldyc=0, ys=None, ldys=0, ws=3 * R, nws=n.value, s=None)
    for kw in (dict(dt=0), dict(m=-1), dict(n=(1 << 24) + 1), dict(k=-1), dict(x=None), dict(xs=None), dict(w=None), dict(ws_=None), dict(ldx=240), dict(ldw=255), dict(ldxs=2),
               dict(act=7), dict(gated=2), dict(y=None), dict(ldy=99), dict(r=2 * R, ldr=99), dict(yc=2 * R, ys=2 * R + Q, ldyc=128, ldys=4), dict(y=None, yc=2 * R, ldyc=128),
               dict(y=None, yc=2 * R, ys=2 * R + Q, ldyc=100, ldys=4), dict(y=P), dict(y=Q), dict(r=R + 2), dict(y=None, yc=P, ldyc=128, ys=2 * R, ldys=4),
               dict(y=None, yc=2 * R, ldyc=128, ys=2 * R, ldys=4)):
        assert p(**kw) == -1, kw
        assert b"8 bits" in lib.vf_last_error()
    if n.value:
        assert p(nws=n.value - 1) == -1 and p(ws=None) == -1
    assert p(m=0) == 0 and p(n=0) == 0


def test_rms_norm_refusals(lib):
    f = caller(lib.vf_rms_norm, dt=F32, m=3, d=8, x=P, ldx=8, r=None, ldr=8, w=None, eps=1e-6, y=Q, ldy=8, yc=None, ldyc=0, ys=None, ldys=0, t=None, ldt=8, rstd=None, s=None)
    for kw in (dict(dt=0), dict(m=-1), dict(d=0), dict(d=(1 << 24) + 1, ldx=1 << 25, ldy=1 << 25), dict(x=None), dict(y=None), dict(ldx=7), dict(ldy=7), dict(eps=-1.0),
               dict(eps=float("nan")), dict(r=R), dict(t=R), dict(r=R, t=2 * R, ldr=7), dict(r=R, t=2 * R, ldt=7), dict(yc=R, ys=2 * R, ldyc=128, ldys=4), dict(y=None, yc=R, ldyc=128),
               dict(y=None, yc=R, ys=2 * R, ldyc=8, ldys=4), dict(r=R, t=2 * R, y=P), dict(r=R, t=P + 4), dict(r=R, t=R + 4), dict(rstd=P), dict(rstd=Q), dict(w=Q)):
        assert f(**kw) == -1, kw
        assert b"rms norm" in lib.vf_last_error()
    assert f(m=0) == 0
    n = C.c_size_t(0)
    assert lib.vf_rms_norm_workspace(F32, 100, 64, C.byref(n)) == 0 and n.value > 0 and lib.vf_rms_norm_workspace(F32, 100, 0, C.byref(n)) == -1
    need = 7 * 64 * 4
    b = caller(lib.vf_rms_norm_backward, dt=F32, m=100, d=64, dy=P, lddy=64, t=Q, ldt=64, rstd=R, w=None, dt_=None, lddt=64, dx=2 * R, lddx=64, dw=3 * R, ws=4 * R, nws=need, s=None)
    for kw in (dict(dy=None), dict(t=None), dict(rstd=None), dict(lddx=63), dict(dt_=5 * R, lddt=63), dict(ws=None), dict(nws=need - 1), dict(dx=Q), dict(dx=P + 4), dict(dw=P),
               dict(dw=2 * R)):
        assert b(**kw) == -1, kw


def test_distill_refusals(lib):
    f = caller(lib.vf_distill, dt=F32, m=3, v=50, x=P, ld=50, ids=Q, t=R, top=4, temp=2.0, loss=2 * R, lse=3 * R, ws=None, nws=0, s=None)
    nan, inf = float("nan"), float("inf")
    for kw in (dict(dt=0), dict(m=-1), dict(v=0), dict(x=None), dict(ids=None), dict(t=None), dict(ld=49), dict(loss=None), dict(top=0), dict(top=257), dict(temp=0.0),
               dict(temp=-2.0), dict(temp=nan), dict(temp=inf), dict(temp=1e-9), dict(loss=P), dict(lse=2 * R), dict(lse=Q), dict(v=200_000, ld=200_000)):
        assert f(**kw) == -1, kw
        assert b"distill" in lib.vf_last_error()
    assert f(m=0) == 0
    n = C.c_size_t(0)
    assert lib.vf_distill_workspace(F32, 1, 200_000, C.byref(n)) == 0 and n.value > 0
    assert lib.vf_distill_workspace(F32, 100_000, 1000, C.byref(n)) == 0 and n.value == 0
    b = caller(lib.vf_distill_backward, dt=F32, m=3, v=50, x=P, ld=50, lse=Q, ids=R, t=2 * R, top=4, temp=2.0, d=3 * R, dx=4 * R, ldd=50, s=None)
    for kw in (dict(x=None), dict(lse=None), dict(ids=None), dict(t=None), dict(d=None), dict(dx=None), dict(ldd=49), dict(top=300), dict(dx=P + 4), dict(dx=Q), dict(dx=2 * R)):
        assert b(**kw) == -1, kw

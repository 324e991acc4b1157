"""CPU-side checks of the encoder operators' entry points: structures match the header, bad arguments are refused before a
GPU is touched, workspaces are stated, empty work needs no device."""
import ctypes as C
import os
import re

import pytest

from paper_2506_00812_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20        # an address that is never looked at: validation fails first
F32, BF16 = binding.VF_F32, binding.VF_BF16


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2506_00812_amd.build import build
        build(verbose=False)
    return binding.load_library()


def test_structs_and_constants_match_the_header():
    hdr = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "vecflow.h")).read(), flags=re.S)
    for name, cls in (("vf_adamw_tensor", binding.VfAdamwTensor), ("vf_adamw_params", binding.VfAdamwParams)):
        body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), hdr, re.S).group(1)
        names = [re.sub(r"[*\s]", "", n.split()[-1]) for line in body.split(";") if line.strip() for n in line.split(",")]
        assert names == [n for n, _ in cls._fields_]
    assert binding._ADAMW_ITEM.size == C.sizeof(binding.VfAdamwTensor) == 88
    for name, value in dict(VF_BF16=binding.VF_BF16, VF_F16=binding.VF_F16, VF_ADAMW_BLOCK=binding.ADAMW_BLOCK,
                            VF_LOG_PROBS_MAX_TOP=binding.LOG_PROBS_MAX_TOP).items():
        assert int(re.search(r"#define %s (\d+)" % name, hdr).group(1)) == value
    for name, value in binding.ACTIVATIONS.items():
        assert int(re.search(r"#define VF_ACT_%s (\d+)" % name.upper(), hdr).group(1)) == value


def linear(lib, dtype=F32, m=4, n=8, k=16, x=P, ldx=16, w=P, ldw=16, act=0, r=None, ldr=8, y=P, ldy=8, z=None, ldz=8, ws=None, nws=0):
    return lib.vf_linear(dtype, m, n, k, x, ldx, w, ldw, None, act, r, ldr, y, ldy, z, ldz, ws, nws, None)


def test_linear_refusals(lib):
    for kw in (dict(dtype=0), dict(dtype=7), dict(m=-1), dict(n=1 << 26), dict(k=-2), dict(x=None), dict(w=None), dict(y=None), dict(ldx=15),
               dict(ldw=3), dict(ldy=7), dict(r=P, ldr=7), dict(z=P, ldz=7), dict(act=9), dict(m=1 << 32)):
        assert linear(lib, **kw) == -1, kw
        assert b"linear" in lib.vf_last_error()
    assert linear(lib, m=0) == 0 and linear(lib, n=0) == 0
    n = C.c_size_t(99)
    assert lib.vf_linear_workspace(F32, 4, 8, 16, 0, 0, None) == -1
    assert lib.vf_linear_workspace(F32, 0, 8, 16, 0, 0, C.byref(n)) == 0 and n.value == 0
    assert lib.vf_linear_workspace(BF16, 2000, 512, 256, 2, 1, C.byref(n)) == 0 and n.value >= 2000 * 512 * 2
    need = n.value
    back = lambda **kw: lib.vf_linear_backward(*[{**dict(dt=BF16, m=2000, n=512, k=256, dy=P, lddy=512, x=P, ldx=256, w=P, ldw=256, z=P, ldz=512, act=2,   # noqa: E731
                                                       dx=P, lddx=256, dw=P, lddw=256, db=P, ws=P, nws=need), **kw}[a] for a in
                                                  "dt m n k dy lddy x ldx w ldw z ldz act dx lddx dw lddw db ws nws".split()], None)
    for kw in (dict(dy=None), dict(z=None), dict(lddy=511), dict(w=None), dict(x=None), dict(lddx=255), dict(lddw=255), dict(ws=None), dict(nws=1000),
               dict(act=-1), dict(dt=0)):
        assert back(**kw) == -1, kw


def test_layer_norm_refusals(lib):
    def fwd(dt=F32, m=3, d=8, x=P, ldx=8, eps=1e-5, y=P, ldy=8):
        return lib.vf_layer_norm(dt, m, d, x, ldx, None, None, eps, y, ldy, None, None, None)
    for kw in (dict(dt=0), dict(m=-1), dict(d=0), dict(d=(1 << 24) + 1, ldx=1 << 25, ldy=1 << 25), dict(x=None), dict(y=None), dict(ldx=7), dict(ldy=7),
               dict(eps=-1.0), dict(eps=float("nan"))):
        assert fwd(**kw) == -1, kw
    assert fwd(m=0) == 0
    n = C.c_size_t(0)
    assert lib.vf_layer_norm_workspace(F32, 100, 64, C.byref(n)) == 0 and n.value > 0

    def back(dy=P, x=P, mu=P, rs=P, dx=P, ldo=64, dw=P, db=P, ws=P, nws=n.value):
        return lib.vf_layer_norm_backward(F32, 100, 64, dy, 64, x, 64, mu, rs, None, dx, ldo, dw, db, ws, nws, None)
    for kw in (dict(dy=None), dict(x=None), dict(mu=None), dict(rs=None), dict(ldo=63), dict(ws=None), dict(nws=n.value - 1)):
        assert back(**kw) == -1, kw


def test_log_probs_refusals(lib):
    def fwd(dt=F32, m=3, v=50, x=P, ld=50, t=P, top=4, lp=P, h=P, lse=P, ids=P, tl=P, ws=None, nws=0):
        return lib.vf_log_probs(dt, m, v, x, ld, t, top, lp, h, lse, ids, tl, ws, nws, None)
    for kw in (dict(dt=0), dict(m=-1), dict(v=0), dict(x=None), dict(ld=49), dict(lp=None), dict(top=65), dict(top=-1), dict(ids=None), dict(tl=None),
               dict(v=200_000, ld=200_000)):
        assert fwd(**kw) == -1, kw
    assert fwd(m=0) == 0
    n = C.c_size_t(0)
    assert lib.vf_log_probs_workspace(F32, 1, 200_000, 8, C.byref(n)) == 0 and n.value > 0
    assert lib.vf_log_probs_workspace(F32, 100_000, 1000, 8, C.byref(n)) == 0 and n.value == 0

    def back(x=P, lse=P, t=P, dl=P, h=None, dh=None, out=P, ldd=50):
        return lib.vf_log_probs_backward(F32, 3, 50, x, 50, lse, t, dl, h, dh, out, ldd, None)
    for kw in (dict(x=None), dict(lse=None), dict(t=None), dict(dl=None), dict(h=P), dict(dh=P), dict(out=None), dict(ldd=49)):
        assert back(**kw) == -1, kw


def test_adamw_refusals(lib):
    def step(params=None, n_tensors=1, **kw):
        f = {**dict(param=P, grad=P, master=0, m=P, v=P, ms=0, vs=0, n=10, decay=0.0, pt=F32, gt=F32, bits=32, reserved=0), **kw}
        item = binding._ADAMW_ITEM.pack(*f.values())
        h = binding.VfAdamwParams(*({**dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, grad_scale=1.0, step=1), **(params or {})}).values())
        return lib.vf_adamw_step(item, n_tensors, C.byref(h), None, None)
    inf, nan = float("inf"), float("nan")
    for kw in (dict(param=0), dict(grad=0), dict(m=0), dict(v=0), dict(n=-1), dict(n=1 << 62), dict(pt=0), dict(gt=9), dict(bits=16), dict(bits=8),
               dict(reserved=1), dict(decay=nan), dict(n_tensors=-1)):
        assert step(**kw) == -1, kw
    for p in (dict(step=0), dict(beta1=1.0), dict(beta2=-0.1), dict(lr=nan), dict(eps=-1.0), dict(eps=inf), dict(grad_scale=inf)):
        assert step(params=p) == -1, p
    assert b"adamw" in lib.vf_last_error()
    assert lib.vf_adamw_step(None, 1, None, None, None) == -1 and lib.vf_adamw_moments(None, 1, None, None, None) == -1
    assert step(n=0, param=0, grad=0, m=0, v=0) == 0        # nothing to do: no launch

"""Outputs of the encoder operators that lie over what the call still reads are refused; without a GPU (no address is looked at)."""
import ctypes as C
import random

import pytest

from paper_2506_00812_amd import binding
from .test_abi_ops import F32, lib  # noqa: F401

K, W, B, R, Y, Z, X = (i << 24 for i in range(1, 8))     # far apart


def refused(rc, lib):  # noqa: F811
    return rc == -1 and b"overlap" in lib.vf_last_error()


def test_linear(lib):  # noqa: F811
    m, n, k = 6, 8, 16

    def call(x=X, ldx=16, w=W, b=B, r=R, ldr=8, y=Y, ldy=8, z=Z, ldz=8):
        return lib.vf_linear(F32, m, n, k, x, ldx, w, 16, b, 0, r, ldr, y, ldy, z, ldz, None, 0, None)
    for kw in (dict(y=X), dict(y=X + 4), dict(y=X + 6 * 64 - 4), dict(y=X - 6 * 32 + 4), dict(y=W + 4), dict(y=B + 28), dict(y=R + 4), dict(y=R, ldy=9),
               dict(z=Y), dict(z=R), dict(z=X), dict(z=W), dict(z=B), dict(x=X, ldx=100, y=X + 15 * 4, ldy=100), dict(x=X, ldx=100, y=X + 93 * 4, ldy=100),
               dict(x=X, ldx=100, y=X - 99 * 4, ldy=100)):
        assert refused(call(**kw), lib), kw


def test_linear_backward(lib):  # noqa: F811
    m, n, k = 6, 8, 16

    def call(dy=Y, x=X, w=W, z=None, act=0, dx=K, dw=R, db=B):
        return lib.vf_linear_backward(F32, m, n, k, dy, n, x, k, w, k, z, n, act, dx, k, dw, k, db, 1 << 32, 1 << 30, None)
    for kw in (dict(dx=Y), dict(dx=X), dict(dx=W), dict(dw=Y), dict(dw=X), dict(dw=W), dict(db=Y), dict(db=X), dict(db=W), dict(dx=R), dict(db=R), dict(db=K),
               dict(z=Z, act=2, db=Z)):
        assert refused(call(**kw), lib), kw


def test_layer_norm(lib):  # noqa: F811
    m, d = 6, 16

    def fwd(x=X, ldx=16, w=W, b=B, y=Y, ldy=16, mu=K, rs=R):
        return lib.vf_layer_norm(F32, m, d, x, ldx, w, b, 1e-5, y, ldy, mu, rs, None)
    for kw in (dict(y=X + 4), dict(y=X, ldy=17), dict(y=W), dict(y=B), dict(mu=X), dict(rs=X), dict(mu=Y), dict(rs=Y), dict(mu=R), dict(mu=W), dict(rs=B)):
        assert refused(fwd(**kw), lib), kw

    def back(dy=Y, ld=16, x=X, mu=K, rs=R, w=W, dx=Z, ldx=16, dw=8 << 24, db=9 << 24):
        return lib.vf_layer_norm_backward(F32, m, d, dy, ld, x, 16, mu, rs, w, dx, ldx, dw, db, 1 << 32, 1 << 30, None)
    for kw in (dict(dx=Y + 4), dict(dx=Y, ldx=17), dict(dx=X), dict(dx=K), dict(dx=R), dict(dx=W), dict(dw=Z), dict(db=Z), dict(db=8 << 24), dict(dw=W), dict(db=Y),
               dict(dw=X)):
        assert refused(back(**kw), lib), kw


def test_log_probs_backward(lib):  # noqa: F811
    m, v = 6, 50

    def back(x=X, ld=50, lse=K, t=W, dl=B, h=R, dh=Y, out=Z, ldd=50):
        return lib.vf_log_probs_backward(F32, m, v, x, ld, lse, t, dl, h, dh, out, ldd, None)
    for kw in (dict(out=X + 4), dict(out=X, ldd=51), dict(out=K), dict(out=W), dict(out=B), dict(out=R), dict(out=Y)):
        assert refused(back(**kw), lib), kw


def test_against_the_bytes_themselves(lib):  # noqa: F811
    """Random places and row distances: refused exactly where x and y share a byte (of slices with unlike distances: only there)."""
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("an accepted call would run, on addresses that are not there")
    rng = random.Random(1)
    seen = set()
    for _ in range(4000):
        m, d = rng.randint(1, 4), rng.randint(1, 6)
        ldx, ldy = [d + rng.choice([0, 0, 1, 3, 9]) for _ in range(2)]
        if rng.random() < 0.5:
            ldy = ldx
        at = rng.randint(-60, 60)
        cells = [{a + i * ld + j for i in range(m) for j in range(d)} for a, ld in ((0, ldx), (at, ldy))]
        rc = lib.vf_layer_norm(F32, m, d, X, ldx, None, None, 1e-5, X + 4 * at, ldy, None, None, None)
        in_place = at == 0 and (ldx == ldy or m == 1)
        shared = bool(cells[0] & cells[1]) and not in_place
        alike = ldx == ldy or m == 1 or d in (ldx, ldy)
        assert refused(rc, lib) == shared or (shared and not alike), (m, d, ldx, ldy, at)
        seen.add((shared, alike, in_place))
    assert len(seen) >= 5
    # an input that is not read may lie under an output: w where only dw is asked for, z where there is no activation
    m, n, k = 6, 8, 16
    back = lambda dx, dw, w, x, z: lib.vf_linear_backward(F32, m, n, k, Y, n, x, k, w, k, z, n, 0, dx, k, dw, k, None, 1 << 32, 1 << 30, None)   # noqa: E731
    assert not refused(back(None, W, W, X, None), lib) and not refused(back(X, None, W, X, None), lib) and not refused(back(K, R, W, X, R), lib)

"""RMS norm and rotary positions without a GPU: refusals of the C entry points, which
come before anything touches a device, and of the binding."""
import ctypes
import os

import pytest

from paper_2602_01219_amd import mita

pytestmark = pytest.mark.skipif(not os.path.exists(mita.LIB_PATH), reason="libmita.so not built")
# addresses that are never read: every call below is refused before a launch
A = [0x10000000 * (i + 1) for i in range(12)]
MAX_C = 65536
BAD, NOT = mita.MITA_ERR_INVALID_ARG, mita.MITA_ERR_UNSUPPORTED


def test_rms_configurations():
    ok = lambda **kw: mita.rms_check(mita.RmsConfig(**{**dict(rows=(10,), C=64), **kw}))
    assert ok() == mita.MITA_OK and ok(out="e4m3") == mita.MITA_OK and ok(out="e4m3", group=128) == mita.MITA_OK
    assert ok(C=0) == BAD and ok(rows=(0,)) == BAD and ok(eps=0.0) == BAD and ok(eps=float("inf")) == BAD
    assert ok(C=MAX_C + 1) == NOT and ok(out="e4m3", group=64) == NOT and ok(group=128) == NOT
    assert ok(rows=(2 ** 30 + 1,)) == NOT and ok(rows=(2 ** 15, 2 ** 15, 2)) == NOT
    for kw in (dict(out="f16"), dict(dtype="f16"), dict(wdtype="e4m3"), dict(rows=(1, 2, 3, 4)), dict(rows=(2 ** 32,)),
               dict(C=2 ** 32 + 64), dict(eps=1e-60)):
        with pytest.raises(ValueError):
            ok(**kw)
    assert mita.rms_workspace_size(mita.RmsConfig((10,), 64)) > 0
    assert mita.rms_workspace_size(mita.RmsConfig((10,), 70000)) == 0
    lib = mita.load_library()
    assert lib.mita_rms_check(None) == BAD and lib.mita_rms_workspace_size(None) == 0


def test_rms_calls():
    lib = mita.load_library()
    same = mita.RmsConfig((10,), 64).struct()
    e4m3 = mita.RmsConfig((10,), 64, out="e4m3").struct()

    def fwd(x=A[0], res=A[1], w=A[2], h=A[3], y=A[4], scales=None, rstd=A[6], c=same):
        return lib.mita_rms_forward(ctypes.byref(c), x, res, w, h, y, scales, rstd, None)

    def bwd(h=A[0], w=A[1], rstd=A[2], dy=A[3], dh=A[4], dx=A[5], dw=A[6], ws=A[7], n=1 << 20):
        return lib.mita_rms_backward(ctypes.byref(same), h, w, rstd, dy, dh, dx, dw, ws, n, None)

    assert fwd(x=None) == BAD and fwd(y=None) == BAD and fwd(x=A[0] + 1) == BAD and fwd(res=A[1] + 1) == BAD
    assert fwd(w=A[2] + 2) == BAD and fwd(h=A[3] + 1) == BAD and fwd(rstd=A[6] + 2) == BAD
    assert fwd(h=A[0] + 2) == BAD and fwd(y=A[1] + 128) == BAD and fwd(h=A[4]) == BAD and fwd(y=A[2]) == BAD
    assert fwd(rstd=A[0]) == BAD and fwd(rstd=A[4]) == BAD and fwd(scales=A[5]) == BAD
    assert fwd(c=e4m3, scales=None) == BAD and fwd(c=e4m3, scales=A[5] + 1) == BAD
    assert fwd(c=e4m3, scales=A[5], y=A[0]) == BAD and fwd(c=e4m3, scales=A[4]) == BAD and fwd(c=e4m3, scales=A[1]) == BAD
    assert fwd(c=mita.RmsConfig((10,), 70000).struct()) == NOT
    assert bwd(h=None) == BAD and bwd(rstd=None) == BAD and bwd(dy=None) == BAD and bwd(dx=None, dw=None) == BAD
    assert bwd(dx=A[0]) == BAD and bwd(dx=A[3] + 2) == BAD and bwd(dx=A[4] + 2) == BAD and bwd(dw=A[3]) == BAD
    assert bwd(dw=A[5]) == BAD and bwd(ws=A[4]) == BAD and bwd(ws=A[7] + 16) == BAD and bwd(dw=A[6] + 2) == BAD
    assert bwd(ws=None) == mita.MITA_ERR_WORKSPACE and bwd(n=8) == mita.MITA_ERR_WORKSPACE


def test_rope_configurations():
    ok = lambda **kw: mita.rope_check(mita.RopeConfig(**{**dict(B=1, H=2, N=3, d=64), **kw}))
    assert ok() == mita.MITA_OK and ok(rot=2) == mita.MITA_OK and ok(d=7, rot=4) == mita.MITA_OK
    assert ok(rot=3) == BAD and ok(rot=66) == BAD and ok(d=7) == BAD and ok(d=1) == BAD and ok(B=0) == BAD
    assert ok(d=258) == NOT and ok(H=5000) == NOT and ok(B=2 ** 25, N=1) == NOT and ok(B=2 ** 25 - 8, N=1) == mita.MITA_OK
    assert ok(base=1.0) == BAD and ok(base=float("nan")) == BAD and ok(base=float("inf")) == BAD
    assert ok(scale=-1.0) == BAD and ok(scale=float("nan")) == BAD
    assert ok(scaling="linear", factor=0.5) == BAD and ok(scaling="linear", factor=float("inf")) == BAD
    assert ok(scaling="base", rot=2, factor=2.0) == mita.MITA_OK
    assert ok(scaling="parts", factor=2.0) == BAD and ok(scaling="parts", factor=2.0, trained=10) == mita.MITA_OK
    assert ok(scaling="parts", trained=10, slow=2.0, fast=2.0) == BAD and ok(scaling="parts", trained=10, slow=-1.0) == BAD
    for kw in (dict(scaling="ntk"), dict(dtype="f16"), dict(first=2 ** 31 + 1), dict(N=2 ** 32), dict(scale=1e-60),
               dict(rot=2 ** 32 + 2)):
        with pytest.raises(ValueError):
            ok(**kw)
    assert mita.load_library().mita_rope_check(None) == BAD


def test_rope_calls():
    lib = mita.load_library()
    cfg = mita.RopeConfig(2, 4, 10, 64, H_kv=2).struct()

    def call(q=A[0], k=A[1], pos=None, qo=A[2], ko=A[3], c=cfg, fn=lib.mita_rope_forward):
        return fn(ctypes.byref(c), q, k, pos, qo, ko, None)

    for fn in (lib.mita_rope_forward, lib.mita_rope_backward):
        assert call(q=None, fn=fn) == BAD and call(qo=None, fn=fn) == BAD and call(ko=None, fn=fn) == BAD
        assert call(k=None, fn=fn) == BAD and call(q=A[0] + 1, fn=fn) == BAD and call(pos=A[4] + 2, fn=fn) == BAD
        assert call(qo=A[0] + 2, fn=fn) == BAD and call(qo=A[1], fn=fn) == BAD and call(ko=A[0], fn=fn) == BAD
        assert call(ko=A[2], fn=fn) == BAD and call(pos=A[2], fn=fn) == BAD and call(pos=A[3] + 64, fn=fn) == BAD
    bad = mita.RopeConfig(2, 4, 10, 64, H_kv=2).struct(7)
    assert call(c=bad) == BAD and "pos_b" in lib.mita_last_error().decode()
    bad = mita.RopeConfig(2, 4, 10, 64, H_kv=2).struct()
    bad.qo = mita.StridesStruct(0, 640, 64)  # both sequences written to one place
    assert call(c=bad) == BAD

"""Dense attention and layer norm without a GPU: the header-only validation and
plans in a host program, and refusals of the C entry points, which come before
anything touches a device."""
import ctypes
import os
import subprocess

import pytest

from paper_2602_01219_amd import mita

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("sanitize", [False, True], ids=["plain", "asan_ubsan"])
def test_layer_check_host_program(tmp_path, sanitize):
    exe = tmp_path / "test_layer_check"
    flags = ["-std=c++17", "-O1", "-Wall", "-g"]
    if sanitize:
        flags += ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer"]
    r = subprocess.run(["g++", *flags, "-I", os.path.join(ROOT, "include"),
                        os.path.join(ROOT, "tests", "host", "test_layer_check.cpp"), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "layer checks ok" in r.stdout


needs_lib = pytest.mark.skipif(not os.path.exists(mita.LIB_PATH), reason="libmita.so not built")
# addresses that are never read: every call below is refused before a launch
A = [0x10000000 * (i + 1) for i in range(12)]


def _forward(cfg, q=A[0], k=A[1], v=A[2], q_len=None, k_len=None, o=A[3], lse=A[4], ws=A[5], nws=1 << 27):
    lib = mita.load_library()
    return lib.mita_dense_forward(ctypes.byref(cfg), q, k, v, q_len, k_len, o, lse, ws, nws, None)


def _backward(cfg, dq=A[6], dk=A[7], dv=A[8], lse=A[4], ws=A[9], nws=1 << 27):
    lib = mita.load_library()
    return lib.mita_dense_backward(ctypes.byref(cfg), A[0], A[1], A[2], A[3], lse, A[5], None, None, dq, dk, dv, ws,
                                   nws, None)


@needs_lib
def test_dense_refusals():
    cfg = mita.DenseConfig(1, 2, 1, 64, N_k=8192).struct()
    bad = mita.MITA_ERR_INVALID_ARG
    assert _forward(mita.DenseConfig(1, 2, 1, 80).struct()) == mita.MITA_ERR_UNSUPPORTED
    assert _forward(cfg, q=None) == bad
    assert _forward(cfg, k=A[1] + 8) == bad
    assert _forward(cfg, k_len=A[9] + 2) == bad
    assert _forward(cfg, o=A[0]) == bad
    assert _forward(cfg, o=A[2] + 64 * 2) == bad
    assert _forward(cfg, lse=A[1] + 4) == bad
    assert _forward(cfg, ws=A[1]) == bad
    assert _forward(cfg, ws=A[5] + 16) == bad
    assert _forward(cfg, ws=None) == mita.MITA_ERR_WORKSPACE
    assert _forward(cfg, nws=64) == mita.MITA_ERR_WORKSPACE
    assert "workspace needs" in mita.load_library().mita_last_error().decode()
    assert _backward(cfg, dk=None) == bad
    assert _backward(cfg, lse=None) == bad
    assert _backward(cfg, dq=A[0]) == bad
    assert _backward(cfg, dk=A[6]) == bad
    assert _backward(cfg, dv=A[7] + 64 * 2 * 100) == bad
    assert _backward(cfg, dv=A[4]) == bad
    assert _backward(cfg, nws=0) == mita.MITA_ERR_WORKSPACE
    with pytest.raises(ValueError):
        mita.DenseConfig(1, 2, 1, 64, dtype="f16").struct()


@needs_lib
def test_norm_refusals():
    lib = mita.load_library()
    cfg = mita.NormConfig((10,), 64).struct()
    bad = mita.MITA_ERR_INVALID_ARG

    def fwd(x=A[0], w=A[1], b=A[2], y=A[3], mean=A[4], rstd=A[5], c=cfg):
        return lib.mita_norm_forward(ctypes.byref(c), x, w, b, y, mean, rstd, None)

    def bwd(x=A[0], w=A[1], mean=A[4], rstd=A[5], dy=A[6], dx=A[7], dw=A[8], db=A[9], ws=A[10], n=1 << 20):
        return lib.mita_norm_backward(ctypes.byref(cfg), x, w, mean, rstd, dy, dx, dw, db, ws, n, None)

    assert fwd(x=None) == bad and fwd(x=A[0] + 1) == bad and fwd(w=A[1] + 2) == bad and fwd(y=A[0] + 2) == bad
    assert fwd(mean=A[3]) == bad and fwd(rstd=A[4]) == bad and fwd(y=A[1]) == bad
    assert fwd(c=mita.NormConfig((10,), 70000).struct()) == mita.MITA_ERR_UNSUPPORTED
    assert fwd(c=mita.NormConfig((10,), 64, eps=0.0).struct()) == bad
    assert bwd(dx=None, dw=None, db=None) == bad and bwd(dx=A[0]) == bad and bwd(dw=A[9]) == bad
    assert bwd(mean=None) == bad and bwd(db=A[6]) == bad and bwd(ws=A[6]) == bad
    assert bwd(ws=None) == mita.MITA_ERR_WORKSPACE and bwd(n=8) == mita.MITA_ERR_WORKSPACE
    with pytest.raises(ValueError):
        mita.NormConfig((1, 2, 3, 4), 64).struct()


@needs_lib
def test_sizes_past_a_launch():
    lib = mita.load_library()
    # workgroups of 256 threads, one per 32 rows (or keys) of a slice, of which a launch has less than 2^32 / 256
    assert mita.dense_check(mita.DenseConfig(2 ** 21, 4, 32, 64)) == mita.MITA_OK
    assert mita.dense_check(mita.DenseConfig(2 ** 21, 8, 32, 64)) == mita.MITA_ERR_UNSUPPORTED
    assert mita.dense_check(mita.DenseConfig(2 ** 20, 8, 1, 64, N_k=64)) == mita.MITA_ERR_UNSUPPORTED
    for rows in ((2 ** 30 + 1,), (2 ** 15, 2 ** 15, 2)):
        cfg = mita.NormConfig(rows, 9)
        assert mita.norm_check(cfg) == mita.MITA_ERR_UNSUPPORTED
        assert lib.mita_norm_forward(ctypes.byref(cfg.struct()), A[0], None, None, A[0], None, None,
                                     None) == mita.MITA_ERR_UNSUPPORTED
    assert mita.norm_check(mita.NormConfig((2 ** 30,), 9)) == mita.MITA_OK

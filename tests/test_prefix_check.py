"""Attention over shared prefixes without a GPU: refusals, which come before anything
touches a device, and the launch plans that the GPU tests' calls meet."""
import ctypes
import os
import subprocess

import pytest

from paper_2602_01219_amd import mita
from tests.prefix_cases import CASES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = [0x10000000 * (i + 1) for i in range(12)]
BAD, NOT = mita.MITA_ERR_INVALID_ARG, mita.MITA_ERR_UNSUPPORTED
needs_lib = pytest.mark.skipif(not os.path.exists(mita.LIB_PATH), reason="libmita.so not built")


@needs_lib
def test_configurations():
    ok = lambda **kw: mita.prefix_check(mita.PrefixConfig(**{**dict(B=4, H=4, N=1, P=100, d=64, Bp=2, H_kv=2, N_k=7), **kw}))
    assert ok() == mita.MITA_OK and ok(N_k=0) == mita.MITA_OK
    for kw in (dict(Bp=3), dict(Bp=0), dict(H_kv=3), dict(B=0), dict(N=0), dict(P=0), dict(N_k=-1), dict(left=-2),
               dict(right=-2), dict(scale=-1.0), dict(scale=float("nan"))):
        assert ok(**kw) == BAD, kw
    for kw in (dict(d=96), dict(P=2 ** 20 + 1), dict(N_k=2 ** 20 + 1), dict(N=2 ** 20 + 1), dict(H=8192, H_kv=8192),
               dict(B=2 ** 10, Bp=1, N=2 ** 16, H=8), dict(B=2 ** 23, Bp=2 ** 22, H=2, H_kv=2)):
        assert ok(**kw) == NOT, kw
    for kw in (dict(dtype="f16"), dict(B=2 ** 32 + 4), dict(left=2 ** 32), dict(scale=1e-60)):
        with pytest.raises(ValueError):
            ok(**kw)
    lib = mita.load_library()
    assert lib.mita_prefix_check(None) == BAD and lib.mita_prefix_workspace_size(None) == 0
    c = mita.PrefixConfig(4, 4, 1, 100, 64, Bp=2, H_kv=2, N_k=7).struct()
    for name in ("q", "kp", "vp", "k", "v", "o"):
        for s in ((400, 64, 68), (64, 100, 64), (-64, 64, 64), (6400, 64, 2 ** 22 + 8)):
            x = mita.PrefixCfgStruct.from_buffer_copy(c)
            if name in "qo" and s[2] != 64:
                continue  # one token: its distance is not used
            setattr(x, name, mita.StridesStruct(*s))
            assert lib.mita_prefix_check(ctypes.byref(x)) == BAD, (name, s)
    x = mita.PrefixCfgStruct.from_buffer_copy(c)
    x.o = mita.StridesStruct(256, 0, 64)
    assert lib.mita_prefix_check(ctypes.byref(x)) == BAD


@needs_lib
def test_calls():
    lib = mita.load_library()
    cfg = mita.PrefixConfig(4, 4, 1, 1000, 64, Bp=2, H_kv=2, N_k=70).struct()

    def call(q=A[0], kp=A[1], vp=A[2], k=A[3], v=A[4], q_len=None, p_len=None, k_len=None, o=A[5], lse=A[6], ws=A[7],
             n=1 << 27):
        return lib.mita_prefix_forward(ctypes.byref(cfg), q, kp, vp, k, v, q_len, p_len, k_len, o, lse, ws, n, None)

    for name in ("q", "kp", "vp", "k", "v", "o"):
        assert call(**{name: None}) == BAD and call(**{name: A[8] + 8}) == BAD, name
    for name in ("q_len", "p_len", "k_len", "lse"):
        assert call(**{name: A[9] + 2}) == BAD, name
    for at in A[:5]:
        assert call(o=at) == BAD and call(lse=at + 4) == BAD and call(ws=at) == BAD
    assert call(p_len=A[5] + 4) == BAD and call(lse=A[5] + 64) == BAD and call(ws=A[7] + 16) == BAD
    assert call(ws=None) == mita.MITA_ERR_WORKSPACE and call(n=64) == mita.MITA_ERR_WORKSPACE


PROGRAM = """
#include <cstdio>
#include "paper_2602_01219_amd/csrc/layer_check.hpp"
using namespace mita;
int main() {
  mita_prefix_cfg_t c{};
  while (scanf("%d %d %d %d %d %d %d %d %d", &c.B, &c.Bp, &c.H, &c.H_kv, &c.N, &c.P, &c.N_k, &c.left, &c.right) == 9) {
    c.d = 64, c.dtype = MITA_BF16;
    if (check_prefix(&c, nullptr) != MITA_OK) return 1;
    const PrefixPlan p = prefix_plan(c);
    const int64_t rows = p.shared ? shared_rows(c) : dense_rows(c), per = p.few ? DENSE_FEW : DENSE_TQ;
    if (p.tiles * per < rows || (p.tiles - 1) * per >= rows || p.splits < 1 || p.splits > PREFIX_MAX_SPLITS) return 2;
    if (p.shared && c.N_k && (p.otiles * DENSE_FEW < dense_rows(c) || p.osplits < 1)) return 3;
    if (p.slots != p.splits + (p.shared ? p.osplits : 0)) return 4;
    const PrefixLayout L = prefix_layout(c);
    const size_t parts = (size_t)slices(c) * dense_rows(c) * p.slots;
    if (p.slots > 1 && (L.part_lse < parts * 64 * 4 || L.total < L.part_lse + parts * 4)) return 5;
    if (p.blocks + p.oblocks >= (1 << 24)) return 6;
    printf("%d %d %d %d %d\\n", p.shared, p.few, p.splits > 1, p.osplits > 1, p.once);
  }
  return 0;
}
"""


def plans(tmp_path, calls):
    src, exe = tmp_path / "plans.cpp", tmp_path / "plans"
    src.write_text(PROGRAM)
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", os.path.join(ROOT, "include"), "-I", ROOT, str(src),
                        "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in calls), capture_output=True, text=True)
    assert r.returncode == 0, r.returncode
    return [tuple(map(int, l.split())) for l in r.stdout.splitlines()]


def test_the_gpu_tests_meet_every_way(tmp_path):
    got = plans(tmp_path, [c[:7] + c[8:10] for c in CASES])
    assert len(got) == len(CASES)
    ways = {(shared, few, split) for shared, few, split, _, _ in got}
    assert ways == {(s, f, p) for s in (0, 1) for f in (0, 1) for p in (0, 1)}
    assert {own for shared, _, _, own, _ in got if shared} == {0, 1}
    assert {(shared, few) for shared, few, _, _, once in got if once} == {(1, 1), (1, 0), (0, 1)}


def test_plans_hold_over_the_range(tmp_path):
    calls = [(B * S, B, Hk * G, Hk, N, P, Nk, left, 0) for B in (1, 3) for S in (1, 2, 64, 1000) for Hk in (1, 12)
             for G in (1, 8) for N in (1, 17, 300) for P in (1, 200, 70000) for Nk in (0, 1, 5000) for left in (-1, 30)]
    assert len(plans(tmp_path, calls)) == len(calls)

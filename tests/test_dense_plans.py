"""The GPU tests of the dense attention reach every forward kernel: the launch
plans of their calls, from the header that makes them."""
import os
import subprocess

import pytest

from paper_2602_01219_amd import mita
from tests.dense_tile_cases import TILE_CASES
from tests.test_gpu_dense import SHAPES
from tests.test_gpu_dense_values import PLANS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    exe = tmp_path_factory.mktemp("plans") / "dense_plans"
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", os.path.join(ROOT, "include"),
                        os.path.join(ROOT, "tests", "host", "dense_plans.cpp"), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def of(calls, d, dtype):
        code = mita.MITA_F32 if dtype == "f32" else mita.MITA_BF16
        text = "\n".join(f"{B} {H} {Hk} {N} {Nk} {d} {code} {left} {right}" for B, H, Hk, N, Nk, left, right in calls)
        r = subprocess.run([str(exe)], input=text, capture_output=True, text=True)
        assert r.returncode == 0
        out = [dict(zip(("few", "tiles", "splits", "qtiles", "qsplits", "ktiles", "ksplits"), map(int, l.split())))
               for l in r.stdout.splitlines()]
        assert len(out) == len(calls)
        return out

    return of


def call(case):
    B, H, Hk, N, Nk, _, left, right = case[:8]
    return B, H, Hk, N, Nk, left, right


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_every_kernel_and_split_is_reached(plans, d, dtype):
    tiles = plans([call(c) for c in TILE_CASES], d, dtype)
    assert all(not p["few"] for p in tiles)
    assert {p["splits"] > 1 for p in tiles} == {False, True}
    small = plans([call(c) for c in SHAPES], d, dtype)
    assert all(p["few"] for p in small) and {p["splits"] > 1 for p in small} == {False, True}
    for part in ("qsplits", "ksplits"):
        assert {p[part] > 1 for p in small + tiles} == {False, True}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_values_that_are_not_finite_meet_every_kernel(plans, d, dtype):
    got = plans([(B, H, H, N, Nk, -1, 0) for B, H, N, Nk in PLANS.values()], d, dtype)
    assert [(p["few"], p["splits"] > 1) for p in got] == [(1, False), (1, True), (0, False), (0, True)]

"""No C++ exception leaves the C entry points of the dense attention and the layer norm."""
import os
import subprocess

import pytest

from paper_2602_01219_amd import mita

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(not os.path.exists(mita.LIB_PATH), reason="libmita.so not built")
def test_out_of_memory_for_a_message(tmp_path):
    exe = tmp_path / "test_no_throw"
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-rdynamic", "-I", os.path.join(ROOT, "include"),
                        os.path.join(ROOT, "tests", "host", "test_no_throw.cpp"), "-o", str(exe), "-ldl"],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe), mita.LIB_PATH], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "no throw ok" in r.stdout

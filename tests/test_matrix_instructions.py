"""Kernels use matrix instructions of at most 32 cycles: a longer one still reads
its third operand when an LDS read behind it writes those registers."""
import os
import subprocess

import pytest

from paper_2602_01219_amd import build, mita

needs_hipcc = pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="no hipcc")


@pytest.mark.skipif(not os.path.exists(mita.LIB_PATH), reason="libmita.so not built")
def test_library():
    names = build.matrix_instructions(mita.LIB_PATH)
    assert names  # the library's code was read
    assert names <= build.MFMA
    build.check_matrix_instructions(mita.LIB_PATH)


@needs_hipcc
def test_a_longer_one_is_refused(tmp_path):
    src, obj = tmp_path / "k.hip", tmp_path / "k.o"
    src.write_text("""#include <hip/hip_runtime.h>
typedef __attribute__((ext_vector_type(16))) float f32x16;
__global__ void k(const float *x, f32x16 *y) {
  y[threadIdx.x] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[threadIdx.x], x[threadIdx.x + 64], y[threadIdx.x], 0, 0, 0);
}
""")
    r = subprocess.run([build.HIPCC, *build.FLAGS, "-c", str(src), "-o", str(obj)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert build.matrix_instructions(str(obj)) == {"v_mfma_f32_32x32x2_f32"}
    with pytest.raises(RuntimeError, match="32x32x2_f32"):
        build.check_matrix_instructions(str(obj))


def test_a_library_without_device_code_is_refused(tmp_path):
    empty = tmp_path / "empty.so"
    empty.write_bytes(b"no code objects")
    with pytest.raises(RuntimeError, match="no gfx950"):
        build.check_matrix_instructions(str(empty))

"""Layer norm paths that only many rows take, against float64 (the bounds of
tests/test_gpu_norm.py): several rows per thread, and rows too wide for
registers that a workgroup takes one after the other."""
from __future__ import annotations

import pytest
import torch

from tests.test_gpu_norm import check

pytestmark = pytest.mark.gpu


# enough rows for eight workgroups per CU at four (C = 64, 128) and two rows per thread group, none a multiple of them
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["bhnd", "bnhd", "qkv"])
@pytest.mark.parametrize("C", [64, 128])
def test_four_rows_per_thread_group(C, layout, dtype):
    check((3, 8, 10925), C, dtype, layout=layout)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C,rows", [(384, 65549), (1024, 32781)])
def test_two_rows_per_thread_group(C, rows, dtype):
    check((1, 1, rows), C, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["bhnd", "padded"])
def test_wide_rows_one_after_the_other(layout, dtype):
    check((1, 2, 1061), 16385, dtype, layout=layout)

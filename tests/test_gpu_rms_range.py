"""RMS norm at the end of its range: a row's mean of squares has to be finite in fp32, the
sum of its squares need not be. Bounds as in tests/test_gpu_rms.py."""
from __future__ import annotations

import pytest
import torch

from paper_2602_01219_amd import mita
from tests.gpu_helpers import log
from tests.test_gpu_norm import gen
from tests.test_gpu_rms import backward_errors, forward_errors

pytestmark = pytest.mark.gpu
MOST = 3.4e38 ** 0.5  # root mean square whose square fp32 just holds


def rows(C, dtype, seed):
    """Rows of root mean square 2^-8 to 0.97 times the largest: of normal values, of one size, of one element."""
    g = gen(seed)
    z = torch.randn((6, C), device="cuda", generator=g, dtype=torch.float64)
    z[3] = 1
    z[4] = 0
    z[4, C // 3] = 1
    z = z * z.square().mean(-1, keepdim=True).rsqrt()
    size = torch.tensor([2.0 ** -8, 2.0 ** -3, 0.9, 0.97, 0.97, 0.5], device="cuda", dtype=torch.float64)
    return (z * MOST * size[:, None]).to(dtype)


@pytest.mark.parametrize("out", [("same", 0), ("e4m3", 0), ("e4m3", 128)], ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [1, 3, 16, 17, 64, 333, 768, 1025, 4096, 20001, 65536])
def test_sums_of_squares_past_fp32(C, dtype, out):
    cfg = mita.RmsConfig((6,), C, dtype=dtype, out=out[0], group=out[1])
    x = rows(C, cfg.torch_dtype, C)
    # bf16 rounds each element by up to 2^-8 of itself, the mean of squares by twice that: still finite
    assert float(x.double().square().mean(-1).max()) < 3.4e38
    w = 1 + 0.2 * torch.randn(C, device="cuda", generator=gen(2))
    got = mita.rms_forward(cfg, x, w)
    e = forward_errors(cfg, x, None, w, got)
    res = torch.randn((6, C), device="cuda", generator=gen(3)).to(cfg.torch_dtype)
    both = mita.rms_forward(cfg, x, w, res)
    e.update({n + "+": v for n, v in forward_errors(cfg, x, res, w, both).items()})
    dy = torch.randn((6, C), device="cuda", generator=gen(4)).to(cfg.torch_dtype)
    dx, dw = mita.rms_backward(cfg, x, got[3], dy, w, want_weight=True)
    e.update(backward_errors(cfg, x, got[3], dy, w, None, dx, dw))
    log(f"[rms range] {cfg}: " + " ".join(f"{k} {v:.3f}" for k, v in e.items()))
    assert max(e.values()) <= 1.0, e


@pytest.mark.parametrize("C", [17, 4096, 20001])
def test_the_smallest_rows(C):
    # squares of 1e-30 and below beside eps = 1e-30: eps counts alone, or both do
    cfg = mita.RmsConfig((4,), C, dtype="f32", eps=1e-30)
    x = torch.randn((4, C), device="cuda", generator=gen(5)) * torch.tensor([[1e-14], [1e-15], [1e-16], [1e-20]],
                                                                            device="cuda")
    e = forward_errors(cfg, x, None, None, mita.rms_forward(cfg, x))
    assert max(e.values()) <= 1.0, e

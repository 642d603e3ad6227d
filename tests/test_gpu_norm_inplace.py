"""Layer norm gradients written in dy's place: the same bits as beside it."""
from __future__ import annotations

import pytest
import torch

from paper_2602_01219_amd import mita

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [64, 384, 768, 1021])
def test_a_last_row_whose_dx_overflows(C, dtype):
    """Lanes past the last row read its dy again, where dx may have been written
    by then: infinite there, it must not reach the sums of dw and db."""
    rows = 33  # no multiple of the rows that a workgroup takes
    cfg = mita.NormConfig((rows,), C, dtype=dtype)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    # rstd about 300, and dy of 1e37 and alternating sign: dx overflows, dy h and dy do not
    x = (1e-3 * torch.randn((rows, C), device="cuda", generator=g)).to(cfg.torch_dtype)
    dy = torch.randn((rows, C), device="cuda", generator=g)
    dy[-1] = 1e37 * (1.0 - 2.0 * (torch.arange(C, device="cuda") % 2))
    dy = dy.to(cfg.torch_dtype)
    _, mean, rstd = mita.norm_forward(cfg, x)
    dx, dw, db = mita.norm_backward(cfg, x, mean, rstd, dy)
    assert bool(torch.isinf(dx[-1].float()).any())
    assert bool(torch.isfinite(dw).all()) and bool(torch.isfinite(db).all())
    for _ in range(50):
        z = dy.clone()
        _, dw2, db2 = mita.norm_backward(cfg, x, mean, rstd, z, dx=z)
        assert torch.equal(z.nan_to_num(7.0), dx.nan_to_num(7.0))
        assert torch.equal(dw2, dw) and torch.equal(db2, db)

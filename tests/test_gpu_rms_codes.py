"""Codes of the RMS norm's 8-bit output are y / scale rounded to nearest even, also where the
quotient lies at or next to the middle between two codes. Rows of ones with eps = 1e-30
have rstd = 1 exactly (C a power of two), so that y is the weights, whatever the order
of the sum; scale and quotient are single fp32 operations, and the codes are compared bit for
bit with the host's."""
from __future__ import annotations

import pytest
import torch

from paper_2602_01219_amd import mita

E4M3 = torch.float8_e4m3fn


def middles():
    """The numbers half way between two neighbouring codes, from the smallest on, up to 224."""
    codes = torch.arange(0, 127, dtype=torch.uint8).view(E4M3).float()
    codes = codes[codes <= 224]
    return (codes[1:] + codes[:-1]) / 2


def weights(C, group, seed):
    """[C] fp32: in each group a zero, one largest value, and multiples of its scale by the middles, moved by up to two
    steps."""
    g = torch.Generator().manual_seed(seed)
    width, w = group or C, torch.empty(C)
    m = middles()
    for at in range(0, C, width):
        n = min(width, C - at)
        top = torch.rand(1, generator=g) + 0.5
        t = m[torch.randint(len(m), (n,), generator=g)] * (top / 448)
        step = torch.randint(-2, 3, (n,), generator=g, dtype=torch.int32)
        t = (t.view(torch.int32) + step).view(torch.float32)
        t = torch.where(torch.rand(n, generator=g) < 0.5, -t, t)
        t[0] = 0.0
        t[1 + torch.randint(n - 1, (1,), generator=g)] = top
        w[at:at + n] = t
    return w


def expected(w, group):
    """(codes as bytes, scales) of y = w, and the bytes that the product with the scale's reciprocal gives."""
    parts = w.split(group or len(w))
    scales = torch.stack([p.abs().max() / 448 for p in parts])
    codes = torch.cat([p / s for p, s in zip(parts, scales)]).to(E4M3).view(torch.uint8)
    product = torch.cat([p * (1 / s) for p, s in zip(parts, scales)]).to(E4M3).view(torch.uint8)
    return codes, scales, product


SIZES = [(128, 128), (128, 0), (64, 0), (1024, 128), (4096, 128), (4096, 0), (32768, 128), (32768, 0)]


@pytest.mark.parametrize("C,group", SIZES)
def test_the_middles_tell_the_quotient_from_the_product(C, group):
    # without a GPU: the inputs below have codes that a product with the reciprocal gets wrong
    wrong = 0
    for seed in range(6):
        codes, _, product = expected(weights(C, group, seed), group)
        wrong += int((codes != product).sum())
    assert wrong > 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C,group", SIZES)
def test_codes_are_the_quotients(C, group, dtype):
    cfg = mita.RmsConfig((6,), C, dtype=dtype, out="e4m3", group=group, eps=1e-30)
    one = torch.ones((6, C), device="cuda").to(cfg.torch_dtype)
    one[1::2] = -1
    for seed in range(6):
        w = weights(C, group, seed)
        codes, scales, _ = expected(w, group)
        y, s, _, rstd = mita.rms_forward(cfg, one, w.cuda())
        assert (rstd == 1).all()
        y, s = y.view(torch.uint8).cpu(), s.cpu()
        assert torch.equal(s, scales.expand(6, -1))
        assert torch.equal(y[::2], codes.expand(3, -1)), int((y[0] != codes).sum())
        assert torch.equal(y[1::2], codes.expand(3, -1) ^ 0x80)


@pytest.mark.gpu
@pytest.mark.parametrize("off", [0, 1, 2])
def test_codes_of_rows_at_any_alignment(off):
    # pieces of 16 bytes, of two elements and of one
    C = 1024
    cfg = mita.RmsConfig((5,), C, out="e4m3", group=128, eps=1e-30)
    x = torch.ones((5, C + 8), device="cuda", dtype=torch.bfloat16)[:, off:off + C]
    w = weights(C, 128, 11)
    codes, scales, _ = expected(w, 128)
    y, s, _, _ = mita.rms_forward(cfg, x, w.cuda())
    assert torch.equal(s.cpu(), scales.expand(5, -1)) and torch.equal(y.view(torch.uint8).cpu(), codes.expand(5, -1))


@pytest.mark.gpu
@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("C", [1024, 32768])
def test_a_group_past_fp32(C, off):
    # one y beyond the largest fp32 number: its group's scale is infinite and its codes 0, but for its own, NaN
    x = torch.ones((3, C + 8), device="cuda", dtype=torch.bfloat16)[:, off:off + C]
    x[:, 300] = 2.0
    w = weights(C, 128, 12)
    w[300] = 3e38
    y, s, _, _ = mita.rms_forward(mita.RmsConfig((3,), C, out="e4m3", group=128, eps=1e-30), x, w.cuda())
    y = y.float().cpu()
    assert torch.isinf(s[:, 2]).all() and torch.isfinite(s[:, :2]).all() and torch.isfinite(s[:, 3:]).all()
    assert torch.isnan(y[:, 300]).all()
    assert (y[:, 256:300] == 0).all() and (y[:, 301:384] == 0).all()
    assert torch.isfinite(y[:, :256]).all() and torch.isfinite(y[:, 384:]).all()

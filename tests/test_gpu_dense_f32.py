"""fp32 products of the dense attention, formed from three bf16 numbers per operand:
scores are not low or high on average, and the largest fp32 numbers stay finite."""
from __future__ import annotations

import math

import pytest
import torch

from paper_2602_01219_amd import mita

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
LARGEST = torch.finfo(torch.float32).max


def rand(g, *shape):
    return torch.rand(shape, device="cuda", generator=g)


@pytest.mark.parametrize("d", [64, 128])
def test_scores_have_no_bias(d):
    """One key, so lse is the score: its relative error, averaged over rows of
    positive numbers. Parts cut off on both sides would make every product low,
    by 3.7e-8 on average."""
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    B, H, N = 64, 16, 256
    q, k, v = 1 + rand(g, B, H, N, d), 1 + rand(g, B, H, 1, d), rand(g, B, H, 1, d)
    cfg = mita.DenseConfig(B, H, N, d, N_k=1, dtype="f32", scale=0.125)
    _, lse = mita.dense_forward(cfg, q, k, v)
    z = 0.125 * (q.double() @ k.double().transpose(-1, -2))[..., 0]
    # the two constants as they are rounded: scale log2(e) and log(2)
    f = lambda x: float(torch.tensor(x, dtype=torch.float32))
    fixed = f(0.125 * f(math.log2(math.e))) * f(math.log(2.0)) / 0.125 - 1.0
    mean = float(((lse.double() - z) / z).mean()) - fixed
    # six products per 16 dimensions and four more operations, each rounded by at most u of the sum, either way:
    # four standard deviations of the mean of the 2^18 rows
    assert abs(mean) <= 4 * (6 * d / 16 + 4) * U / math.sqrt(B * H * N)


@pytest.mark.parametrize("d", [64, 128])
def test_the_largest_numbers_stay_finite(d):
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    q, k, v, dO = (rand(g, 1, 2, n, d) for n in (40, 50, 50, 40))
    cfg = mita.DenseConfig(1, 2, 40, d, N_k=50, dtype="f32")
    # a column of q that meets zeros of k, and the other way round: products of 0, whatever the size
    k[..., 0] = 0.0
    q[..., 1] = 0.0
    def run(top):
        q[..., 0], k[..., 1] = top, -top
        o, lse = mita.dense_forward(cfg, q, k, v)
        return (o, lse, *mita.dense_backward(cfg, q, k, v, o, lse, dO))
    o, lse, dq, dk, dv = run(LARGEST)
    o0, lse0, dq0, dk0, dv0 = run(0.0)
    assert torch.equal(o, o0) and torch.equal(lse, lse0) and torch.equal(dv, dv0)
    assert torch.equal(dq[..., 2:], dq0[..., 2:]) and torch.equal(dk[..., 2:], dk0[..., 2:])
    # values, against gradients of 0
    one = mita.DenseConfig(1, 2, 40, d, N_k=1, dtype="f32")
    k, v = k[:, :, :1].contiguous() * 0, v[:, :, :1].contiguous()
    v[..., 5], dO[..., 5] = LARGEST, 0.0
    o, lse = mita.dense_forward(one, q * 0, k, v)
    assert torch.equal(o, v.expand_as(o))
    for x in mita.dense_backward(one, q * 0, k, v, o, lse, dO):
        assert bool(torch.isfinite(x).all())

"""What dense attention makes of scores that are not finite or larger than it
supports (2^27 log 2): rows that see one have o and lse NaN, whichever kernel and
split a call takes, and rows that see none of them are as if they were not there."""
from __future__ import annotations

import math

import pytest
import torch

from paper_2602_01219_amd import mita

pytestmark = pytest.mark.gpu

# B, H, N, N_k: 32-row tiles whole and split, 128-row tiles whole and split
PLANS = {"few": (1, 2, 40, 200), "few_split": (1, 2, 20, 3000), "tiles": (8, 16, 140, 200), "tiles_split": (8, 16, 140, 1100)}


def inputs(plan, d, dtype, seed=1):
    B, H, N, N_k = PLANS[plan]
    cfg = mita.DenseConfig(B, H, N, d, N_k=N_k, dtype=dtype, right=0)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    q, k, v = (torch.randn((B, H, n, d), device="cuda", generator=g).to(cfg.torch_dtype) for n in (N, N_k, N_k))
    return cfg, q, k, v


def all_nan(x):
    return bool(torch.isnan(x).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("plan", list(PLANS))
@pytest.mark.parametrize("what", ["nan", "overflow"])
def test_rows_that_see_a_score_that_is_not_finite(what, plan, d, dtype):
    cfg, q, k, v = inputs(plan, d, dtype)
    o, lse = mita.dense_forward(cfg, q, k, v)
    N, N_k = cfg.N, cfg.N_k
    bad = N_k - N // 2  # seen by the last N // 2 queries
    first = bad - (N_k - N)
    if what == "overflow":
        q[0, 0, :, 0] = 1e20  # 1e20 * 1e20 overflows; with other keys the dots are finite, but past what is supported
        o3, lse3 = mita.dense_forward(cfg, q, k, v)
        assert all_nan(o3[0, 0]) and all_nan(lse3[0, 0])
        q[0, 0, :first, 0] = 1.0
        o, lse = mita.dense_forward(cfg, q, k, v)
        k[0, 0, bad, 0] = 1e20
    else:
        k[0, 0, bad, 3] = math.nan
    o2, lse2 = mita.dense_forward(cfg, q, k, v)
    assert all_nan(o2[0, 0, first:]) and all_nan(lse2[0, 0, first:])
    for x, y in ((o, o2), (lse, lse2)):
        assert torch.equal(x[0, 0, :first], y[0, 0, :first])
        assert torch.equal(x[0, 1:], y[0, 1:]) and torch.equal(x[1:], y[1:])
    # and the gradients of those rows say so
    dO = torch.ones_like(q)
    dq, dk, dv = mita.dense_backward(cfg, q, k, v, o2, lse2, dO)
    assert all_nan(dq[0, 0, first:]) and all_nan(dv[0, 0, bad]) and all_nan(dk[0, 0, bad])
    assert bool(torch.isfinite(dq[0, 1:]).all()) and bool(torch.isfinite(dk[0, 1:]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("plan", list(PLANS))
def test_rows_whose_every_score_is_minus_infinity(plan, dtype):
    # 0 / 0, not the 0 of a row that sees no key
    cfg, q, k, v = inputs(plan, 64, dtype)
    q[0, 1, 7, 0] = 1e20
    k[0, 1, :, 0] = -1e20
    o, lse = mita.dense_forward(cfg, q, k, v)
    assert all_nan(o[0, 1, 7]) and all_nan(lse[0, 1, 7])
    assert bool(torch.isfinite(o[0, 0]).all()) and bool(torch.isfinite(lse[0, 0]).all())
    # the other rows' scores are -1e20 q: none of a size that is supported
    assert all_nan(o[0, 1])
    # rows without keys stay 0 and -infinity
    n = torch.zeros(cfg.B, dtype=torch.int32, device="cuda")
    o, lse = mita.dense_forward(cfg, q, k, v, k_len=n)
    assert bool((o == 0).all()) and bool(torch.isneginf(lse).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("plan", list(PLANS))
def test_scores_of_the_lowest_values_weigh_nothing(plan, dtype):
    # the first keys of a sequence blanked by scores far below every other (and below what is supported)
    cfg, q, k, v = inputs(plan, 64, dtype)
    q[..., 0] = 1.0
    blank = cfg.N_k - cfg.N - 9
    k[:, :, :blank, 0] = -3e38 if dtype == "f32" else -1e30
    o, lse = mita.dense_forward(cfg, q, k, v)
    assert bool(torch.isfinite(o).all()) and bool(torch.isfinite(lse).all())
    k[:, :, :blank] = 0  # the same, with the window instead
    z = (q.double() @ k.double().transpose(-1, -2)) / 8.0
    i, j = torch.arange(cfg.N, device="cuda")[:, None], torch.arange(cfg.N_k, device="cuda")[None]
    z = z.masked_fill((j < blank) | (j > i + cfg.N_k - cfg.N), -math.inf)
    want = torch.softmax(z, -1) @ v.double()
    # |z| < 16, |v| < 6: 64-term fp32 dots and the exponents are off by 1e-4, bf16 weights and o by 2^-8 each
    bound = 6 * (2e-4 + (2 * 2.0 ** -8 if dtype == "bf16" else 0))
    assert float((o.double() - want).abs().max()) <= bound
    assert float((lse.double() - torch.logsumexp(z, -1)).abs().max()) <= 1e-3


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("plan", list(PLANS))
def test_large_scores_that_are_supported(plan, sign):
    # scores near 2^26 in size, multiples of 2^20: the first key has all the weight of every row
    cfg, q, k, v = inputs(plan, 64, "f32")
    q.zero_()
    k.zero_()
    q[..., 0] = 8.0
    step = 1 + torch.randperm(cfg.N_k, generator=torch.Generator().manual_seed(2)).cuda() % 50
    step[0] = 0
    k[..., 0] = sign * 2.0 ** 26 - step * 2.0 ** 20
    o, lse = mita.dense_forward(cfg, q, k, v)
    # one weight, divided by itself and multiplied as three bf16 numbers: exact but for their sum's rounding
    assert float((o - v[:, :, :1]).abs().max()) <= 2.0 ** -23 * float(v.abs().max())
    # fp32 numbers of that size (9.7e7 in log2 units) are 8 apart: half of it in each of three roundings
    assert float((lse.double() - sign * 2.0 ** 26).abs().max()) <= 12


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("plan", list(PLANS))
def test_gradients_beside_scores_of_the_lowest_values(plan, dtype):
    # keys without weight get no gradient and give none: as if a length had left them out
    cfg, q, k, v = inputs(plan, 64, dtype)
    q[..., 0] = 1.0
    blank = cfg.N_k - cfg.N - 9
    k[:, :, :blank, 0] = -3e38 if dtype == "f32" else -1e30
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    dO = torch.randn(q.shape, device="cuda", generator=g).to(q.dtype)
    o, lse = mita.dense_forward(cfg, q, k, v)
    dq, dk, dv = mita.dense_backward(cfg, q, k, v, o, lse, dO)
    assert bool((dk[:, :, :blank] == 0).all()) and bool((dv[:, :, :blank] == 0).all())
    short = mita.DenseConfig(cfg.B, cfg.H, cfg.N, 64, N_k=cfg.N_k - blank, dtype=dtype, right=0)
    cut = [t[:, :, blank:] for t in (k, v)]
    want = mita.dense_backward(short, q, *cut, o, lse, dO)
    # the same terms in sums of another order or split: at most a few hundred of them, fp32, then one rounding
    for x, y in zip((dq, dk[:, :, blank:], dv[:, :, blank:]), want):
        bound = 256 * 2.0 ** -24 * float(y.abs().max()) + 2 * (2.0 ** -8 if dtype == "bf16" else 0) * y.abs().double()
        assert bool(((x.double() - y.double()).abs() <= bound + 1e-30).all())

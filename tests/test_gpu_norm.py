"""Layer norm forward and backward on the GPU against float64.

Bounds, with u = 2^-24 and r = 2^-8 (half a step of bf16) or 0: the mean of C
fp32 values is off by C u mean|x|, a centred value by em = that + u |x|; the
variance's relative error is below 2 mean(|c|) em / var + (C + 4) u, rstd's half
of it, =: ev; y is off by |w| rstd em + |h w| (ev + 4 u) + u |b| + r |y|. In the
backward mean and rstd are inputs: h is off by 4 u (|x| + |mean|) rstd =: eh, the
row means by C u times the means of the absolute terms plus their factors'
errors, a column sum over n rows by n u times the sum of the absolute terms.
Every bound is doubled for second-order terms."""
from __future__ import annotations

import pytest
import torch

from paper_2602_01219_amd import mita
from tests.dense_reference import U, worst
from tests.gpu_helpers import log

pytestmark = pytest.mark.gpu
F64 = torch.float64


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rows_of(g, rows, C, dtype, layout, mean=0.5, std=1.0):
    x = torch.randn((*rows, C), device="cuda", generator=g) * std + mean * torch.randn(C, device="cuda", generator=g)
    x = x.to(dtype)
    if layout == "bnhd":
        x = x.transpose(1, 2).contiguous().transpose(1, 2)
    elif layout == "padded":  # rows further apart than their width, not 16-byte aligned
        buf = torch.empty((*rows, C + 3), dtype=dtype, device="cuda")
        buf[..., 1:1 + C] = x
        x = buf[..., 1:1 + C]
    elif layout == "qkv":
        buf = torch.empty((rows[0], rows[2], 3, rows[1], C), dtype=dtype, device="cuda")
        buf[:, :, 1] = x.transpose(1, 2)
        x = buf[:, :, 1].transpose(1, 2)
    return x


def half_step(dtype):
    return 2.0 ** -8 if dtype == "bf16" else U


def check(rows, C, dtype, wdtype="f32", layout="bhnd", affine=True, mean=0.5, seed=1):
    cfg = mita.NormConfig(rows, C, dtype=dtype, wdtype=wdtype)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    wt = torch.float32 if wdtype == "f32" else torch.bfloat16
    g = gen(seed)
    x, dy = (rows_of(g, rows, C, dt, layout, m) for m in (mean, 0.1))
    w = (1 + 0.2 * torch.randn(C, device="cuda", generator=g)).to(wt) if affine else None
    b = (0.3 * torch.randn(C, device="cuda", generator=g)).to(wt) if affine else None
    y = rows_of(g, rows, C, dt, layout).fill_(float("nan"))
    y, mu, rs = mita.norm_forward(cfg, x, w, b, y=y)
    X = x.to(F64)
    W = w.to(F64) if affine else torch.ones(C, dtype=F64, device="cuda")
    Bv = b.to(F64) if affine else torch.zeros(C, dtype=F64, device="cuda")
    M = X.mean(-1, keepdim=True)
    c = X - M
    var = (c * c).mean(-1, keepdim=True) + cfg.eps
    rstd = var ** -0.5
    r = half_step(dtype)
    emean = (C + 2) * U * X.abs().mean(-1, keepdim=True)
    em = emean + U * X.abs()
    ev = (c.abs() * em).mean(-1, keepdim=True) / var + (C + 8) * U
    Y = c * rstd * W + Bv
    ey = 2 * (W.abs() * rstd * em + (c * rstd * W).abs() * (ev + 4 * U) + U * Bv.abs() + r * Y.abs())
    e = dict(y=worst(y, Y, ey), mean=worst(mu, M[..., 0], 2 * emean[..., 0]),
             rstd=worst(rs, rstd[..., 0], 2 * (rstd * ev)[..., 0]))
    # backward from the stored statistics
    dx = rows_of(g, rows, C, dt, layout).fill_(float("nan"))
    ws = torch.full((max(1, mita.norm_workspace_size(cfg)),), 0xFF, dtype=torch.uint8, device="cuda")
    dx, dw, db = mita.norm_backward(cfg, x, mu, rs, dy, w, dx=dx, ws=ws)
    m1, r1 = mu.to(F64)[..., None], rs.to(F64)[..., None]
    h = (X - m1) * r1
    eh = 4 * U * (X.abs() + m1.abs()) * r1
    DY = dy.to(F64)
    gw = DY * W
    s1, s2 = gw.mean(-1, keepdim=True), (gw * h).mean(-1, keepdim=True)
    es1 = (C + 2) * U * gw.abs().mean(-1, keepdim=True)
    es2 = (C + 4) * U * (gw * h).abs().mean(-1, keepdim=True) + (gw.abs() * eh).mean(-1, keepdim=True)
    DX = r1 * (gw - s1 - h * s2)
    ex = 2 * (r1 * (es1 + h.abs() * es2 + eh * s2.abs() + 4 * U * (gw.abs() + s1.abs() + (h * s2).abs())) + r * DX.abs())
    n, rw = X[..., 0].numel(), half_step(wdtype)
    flat = lambda t: t.expand(X.shape).reshape(-1, C)
    DW, DB = flat(DY * h).sum(0), flat(DY).sum(0)
    ew = 2 * (flat((n + 2) * U * (DY * h).abs() + DY.abs() * eh).sum(0) + rw * DW.abs())
    eb = 2 * ((n + 2) * U * flat(DY.abs()).sum(0) + rw * DB.abs())
    e.update(dx=worst(dx, DX, ex), dw=worst(dw, DW, ew), db=worst(db, DB, eb))
    log(f"[norm] {cfg} {layout}: " + " ".join(f"{k} {v:.3f}" for k, v in e.items()))
    assert max(e.values()) <= 1.0, e
    again = mita.norm_backward(cfg, x, mu, rs, dy, w, ws=ws)
    assert all(torch.equal(p, q) for p, q in zip((dx, dw, db), again))


WIDTHS = [1, 2, 7, 8, 33, 64, 65, 128, 200, 256, 384, 512, 513, 768, 1021, 1024, 1500, 2048, 2056, 4096, 4097, 5000, 8192,
          8200, 16384, 20001]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", WIDTHS)
def test_widths(C, dtype):
    check((1, 1, 37), C, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [(1, 1, 1), (1, 1, 5), (3, 1, 7), (2, 3, 1100), (1, 1, 9001)], ids=str)
def test_rows(rows, dtype):
    check(rows, 64, dtype)
    check(rows, 72, dtype, wdtype="bf16" if dtype == "bf16" else "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["bnhd", "qkv", "padded"])
@pytest.mark.parametrize("C", [64, 100, 768])
def test_strides(C, layout, dtype):
    check((2, 5, 77), C, dtype, layout=layout)


def test_without_weights_and_far_from_zero():
    check((1, 2, 50), 256, "f32", affine=False)
    check((1, 2, 50), 256, "bf16", affine=False)
    # a mean 1000 standard deviations away: the variance is summed about the mean
    check((1, 1, 64), 512, "f32", mean=0.0, seed=3)
    g = gen(4)
    cfg = mita.NormConfig((64,), 512, dtype="f32")
    x = 1000.0 + torch.randn((64, 512), device="cuda", generator=g)
    _, mean, rstd = mita.norm_forward(cfg, x)
    X = x.to(F64)
    var = ((X - X.mean(-1, keepdim=True)) ** 2).mean(-1) + cfg.eps
    # each centred value is off by at most u |x| 514 (the mean) + u |x|, about 0.03: the variance, quadratic in
    # the mean's error and linear in the values' own (which average out over 512), by 1e-3 and C u
    assert float((rstd.double() * var.sqrt() - 1).abs().max()) <= 2e-3
    # equal values: y is the bias, rstd 1 / sqrt(eps)
    x = torch.full((64, 512), 3.0, device="cuda")
    y, mean, rstd = mita.norm_forward(cfg, x)
    assert (y == 0).all() and (mean == 3).all()
    assert float((rstd.double() * cfg.eps ** 0.5 - 1).abs().max()) <= 4 * U


def test_more_rows_than_one_grid_dimension():
    """2^27 + 5 rows of 9, a wave each, two rows per wave: 2^32 threads and more."""
    g = gen(12)
    R, C = 2 ** 27 + 5, 9
    cfg = mita.NormConfig((R,), C)
    x = torch.randn((R, C), device="cuda", generator=g, dtype=torch.bfloat16)
    y = torch.full_like(x, float("nan"))
    y, mu, rs = mita.norm_forward(cfg, x, y=y)
    dx, _, _ = mita.norm_backward(cfg, x, mu, rs, x, dx=torch.full_like(x, float("nan")), want_weights=False)
    # workgroup 2^21, the first of the second row of the grid, takes row 2^24
    for at in (0, 2 ** 24 - 500, 2 ** 26, R - 1000):
        X = x[at:at + 1000].to(F64)
        c = X - X.mean(-1, keepdim=True)
        var = (c * c).mean(-1, keepdim=True) + cfg.eps
        Y = c * var ** -0.5
        # |x| < 6 and 9 elements: fp32 mean and x - mean are off by 11 U 6 + 6 U < 5e-6; with that, rstd by
        # 5e-6 rstd of itself, so y by 5e-6 rstd (1 + |y|), |y| < 3, and by the rounding of bf16; twice all of it
        err = 2 * (5e-6 * var ** -0.5 * 4 + half_step("bf16") * Y.abs())
        assert worst(y[at:at + 1000], Y, err) <= 1.0
        G = (X * Y).mean(-1, keepdim=True)
        D = var ** -0.5 * (c - Y * G)
        # dy = x: c, Y and G (|G| = |mean(x y)| < 6) each carry the errors above
        ed = 2 * (var ** -0.5 * (5e-6 + 5e-6 * var ** -0.5 * 4 * (6 + 2 * Y.abs() * 6)
                                 + 5e-6 * var ** -0.5 * (c.abs() + (Y * G).abs()) + 12 * U * (c.abs() + 6 * Y.abs()))
                  + half_step("bf16") * D.abs())
        assert worst(dx[at:at + 1000], D, ed) <= 1.0
    assert all(bool(torch.isfinite(t).all()) for t in (y, mu, rs, dx))


def test_one_dimensional_rows_in_place_and_parts():
    cfg = mita.NormConfig((300,), 384, dtype="bf16")
    g = gen(5)
    x, dy = (torch.randn((300, 384), device="cuda", generator=g).bfloat16() for _ in range(2))
    w, b = (torch.randn(384, device="cuda", generator=g) for _ in range(2))
    y, mean, rstd = mita.norm_forward(cfg, x, w, b)
    dx, dw, db = mita.norm_backward(cfg, x, mean, rstd, dy, w)
    z = x.clone()
    mita.norm_forward(cfg, z, w, b, y=z, want_stats=False)
    assert torch.equal(z, y)
    z = dy.clone()
    _, dw2, db2 = mita.norm_backward(cfg, x, mean, rstd, z, w, dx=z)
    assert torch.equal(z, dx) and torch.equal(dw, dw2) and torch.equal(db, db2)
    only, n1, n2 = mita.norm_backward(cfg, x, mean, rstd, dy, w, want_weights=False)
    assert torch.equal(only, dx) and n1 is None and n2 is None
    n0, dw3, db3 = mita.norm_backward(cfg, x, mean, rstd, dy, w, want_dx=False)
    assert n0 is None and torch.equal(dw, dw3) and torch.equal(db, db3)
    # wide rows in place
    cfg = mita.NormConfig((9,), 20001, dtype="f32")
    x, dy = (torch.randn((9, 20001), device="cuda", generator=g) for _ in range(2))
    y, mean, rstd = mita.norm_forward(cfg, x)
    dx, dw, db = mita.norm_backward(cfg, x, mean, rstd, dy)
    z = dy.clone()
    _, dw2, db2 = mita.norm_backward(cfg, x, mean, rstd, z, dx=z)
    assert torch.equal(z, dx) and torch.equal(dw, dw2) and torch.equal(db, db2)
    z = x.clone()
    mita.norm_forward(cfg, z, y=z)
    assert torch.equal(z, y)


def test_gradient_against_differences():
    cfg = mita.NormConfig((1, 2, 9), 40, dtype="f32")
    g = gen(6)
    x, dy = (torch.randn((1, 2, 9, 40), device="cuda", generator=g) for _ in range(2))
    w, b = (torch.randn(40, device="cuda", generator=g) for _ in range(2))
    y, mean, rstd = mita.norm_forward(cfg, x, w, b)
    grads = mita.norm_backward(cfg, x, mean, rstd, dy, w)

    def f(x, w, b):
        c = x - x.mean(-1, keepdim=True)
        return float(((c * ((c * c).mean(-1, keepdim=True) + cfg.eps).rsqrt() * w + b) * dy.double()).sum())

    at = [t.double() for t in (x, w, b)]
    for i, grad in enumerate(grads):
        way = torch.randn(grad.shape, device="cuda", generator=g, dtype=F64)
        hi, lo = ([t + (s * 1e-4 * way if j == i else 0) for j, t in enumerate(at)] for s in (1, -1))
        # truncation: 1e-8 / 6 of a third derivative of the order of the sums' size, about 1e3
        assert abs(float((grad.double() * way).sum()) - (f(*hi) - f(*lo)) / 2e-4) <= 1e-4


def test_captured_with_eager_calls_in_between():
    cfg = mita.NormConfig((2, 3, 500), 64, dtype="bf16")
    g = gen(7)
    x, dy = (torch.randn((2, 3, 500, 64), device="cuda", generator=g).bfloat16() for _ in range(2))
    w, b = (torch.randn(64, device="cuda", generator=g) for _ in range(2))
    ws = torch.empty(mita.norm_workspace_size(cfg), dtype=torch.uint8, device="cuda")

    def both():
        y, m, r = mita.norm_forward(cfg, x, w, b)
        return (y, m, r) + mita.norm_backward(cfg, x, m, r, dy, w, ws=ws)

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for seed in (1, 2, 3):
        g = gen(seed)
        for t in (x, dy):
            t.copy_(torch.randn(t.shape, device="cuda", generator=g))
        eager = both()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(eager, out))


def test_refusals():
    g = gen(8)
    x = torch.randn((4, 64), device="cuda", generator=g)
    cfg = mita.NormConfig((4,), 64, dtype="f32")
    bad = lambda *a, **kw: pytest.raises(ValueError, mita.norm_forward, cfg, *a, **kw)
    bad(x.cpu())
    bad(x.bfloat16())
    bad(x[:3])
    bad(x, torch.ones(63, device="cuda"))
    bad(x, torch.ones(64, device="cuda").bfloat16())
    bad(x.t().contiguous().t())
    y, mean, rstd = mita.norm_forward(cfg, x)
    buf = torch.randn((5, 64), device="cuda", generator=g)
    for a, b in ((buf[:4], buf[1:]), (buf[1:], buf[:4])):
        with pytest.raises(mita.MitaError) as e:
            mita.norm_forward(cfg, a, y=b)
        assert e.value.status == mita.MITA_ERR_INVALID_ARG
    with pytest.raises(mita.MitaError):
        mita.norm_backward(cfg, x, mean, rstd, y, dx=x)
    with pytest.raises(mita.MitaError):
        mita.norm_backward(cfg, x, mean, rstd, y, want_dx=False, want_weights=False)
    with pytest.raises(mita.MitaError) as e:
        mita.norm_backward(cfg, x, mean, rstd, y, ws=torch.empty(8, dtype=torch.uint8, device="cuda"))
    assert e.value.status == mita.MITA_ERR_WORKSPACE


@pytest.mark.parametrize("attention", ["mita", "dense"])
def test_normalised_queries_and_keys(attention):
    """A layer as it is used: queries and keys normalised per head, attention,
    and back through both, against float64 autograd (MiTA: with one landmark
    per token and every key selected, which makes its choices certain)."""
    g = gen(9)
    B, H, N, d = 2, 3, 64, 64
    q, k, v, dO = (torch.randn((B, H, N, d), device="cuda", generator=g) for _ in range(4))
    wq, bq, wk, bk = (s + 0.1 * torch.randn(d, device="cuda", generator=g) for s in (1.0, 0.0, 1.0, 0.0))
    ncfg = mita.NormConfig((B, H, N), d, dtype="f32")
    qn, mq, rq = mita.norm_forward(ncfg, q, wq, bq)
    kn, mk, rk = mita.norm_forward(ncfg, k, wk, bk)
    if attention == "dense":
        cfg = mita.DenseConfig(B, H, N, d, dtype="f32")
        o, lse = mita.dense_forward(cfg, qn, kn, v)
        dqn, dkn, dv = mita.dense_backward(cfg, qn, kn, v, o, lse, dO)
    else:
        cfg = mita.Config(B=B, H=H, N=N, d=d, grid_h=8, grid_w=8, M=1, lm_h=1, lm_w=1, k=N, dtype="f32", use_shared=0)
        o = mita.forward(cfg, qn, kn, v)
        dqn, dkn, dv = mita.backward(cfg, qn, kn, v, o, dO)
    dq, dwq, dbq = mita.norm_backward(ncfg, q, mq, rq, dqn, wq)
    dk, dwk, dbk = mita.norm_backward(ncfg, k, mk, rk, dkn, wk)
    leaf = [t.double().cpu().requires_grad_() for t in (q, k, v, wq, bq, wk, bk)]
    Q, K, V, Wq, Bq, Wk, Bk = leaf

    def norm(x, w, b):
        c = x - x.mean(-1, keepdim=True)
        return c * ((c * c).mean(-1, keepdim=True) + 1e-5).rsqrt() * w + b

    z = norm(Q, Wq, Bq) @ norm(K, Wk, Bk).transpose(-1, -2) / d ** 0.5
    out = torch.softmax(z, -1) @ V
    out.backward(dO.double().cpu())
    # fp32 throughout: scores up to about 30 in size carry 64 products' roundings (30 * 68 u = 1.2e-4 at the very
    # worst), so weights, o and the gradients are within 2e-4 of their largest element
    for name, got, ref in zip("o dq dk dv dwq dbq dwk dbk".split(), (o, dq, dk, dv, dwq, dbq, dwk, dbk),
                              (out.detach(), Q.grad, K.grad, V.grad, Wq.grad, Bq.grad, Wk.grad, Bk.grad)):
        err = float((got.double().cpu() - ref).abs().max() / ref.abs().max())
        # the key bias' gradient is zero but for rounding (a shift of every key leaves the softmax as it is)
        if name == "dbk":
            err = float((got.double().cpu() - ref).abs().max() / dkn.double().abs().sum((0, 1, 2)).max().cpu())
        assert err <= 2e-4, (name, err)

"""RMS norm with the residual's addition, forward (also to 8 bits) and backward, on
the GPU against float64.

Bounds, with u = 2^-24 and r = 2^-8 (half a step of bf16) or 0: the sum v = x + res
is off by u |v|, its mean of squares over C by (C + 6) u of itself, rstd by half
of that and 6 u for the addition of eps, root and quotient, =: er; y by (er + 4 u + r)
|y|, h by (u + r) |h|. An 8-bit group's scale is off by that of its largest |y| and
2 u, a code (whose quotient adds 2 u) by half a step: 2^-4 of it, or 2^-10 of the scale
where that is more. In the backward rstd is an input: u_i = h rstd and the products carry
4 u, the row mean s is off by (C + 6) u mean|g u|, a column sum over n rows by
(n + 6) u times the sum of the absolute terms. Bounds but for the half steps of 8 bits
are doubled for second-order terms."""
from __future__ import annotations

import pytest
import torch

from paper_2602_01219_amd import mita
from tests.dense_reference import U, worst
from tests.gpu_helpers import log
from tests.test_gpu_norm import gen, half_step, rows_of

pytestmark = pytest.mark.gpu
F64 = torch.float64


def inputs(rows, C, dtype, wdtype, layout, seed, residual=True, affine=True):
    g = gen(seed)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    wt = torch.float32 if wdtype == "f32" else torch.bfloat16
    x, res, dy, dh = (rows_of(g, rows, C, dt, layout, 0.2, s) for s in (0.5, 1.5, 1.0, 1.0))
    w = (1 + 0.2 * torch.randn(C, device="cuda", generator=g)).to(wt) if affine else None
    return x, res if residual else None, w, dy, dh if residual else None


def forward_errors(cfg, x, res, w, got):
    y, scales, h, rstd = got
    C = cfg.C
    r = half_step(cfg.dtype)
    V = x.to(F64) + (res.to(F64) if res is not None else 0)
    W = w.to(F64) if w is not None else torch.ones(C, dtype=F64, device="cuda")
    R = ((V * V).mean(-1, keepdim=True) + cfg.eps) ** -0.5
    er = (C / 2 + 10) * U
    Y = V * R * W
    e = {}
    if rstd is not None:
        e["rstd"] = worst(rstd, R[..., 0], 2 * er * R[..., 0])
    if h is not None:
        e["h"] = worst(h, V, 2 * (U + r) * V.abs())
    if cfg.out == "same":
        e["y"] = worst(y, Y, 2 * (er + 4 * U + r) * Y.abs())
        return e
    n = scales.shape[-1]
    width = cfg.group or C
    full = torch.zeros((*Y.shape[:-1], n * width), dtype=F64, device="cuda")
    full[..., :C] = Y
    S = full.unflatten(-1, (n, width)).abs().amax(-1).clamp(min=2.0 ** -117) / 448
    e["scales"] = worst(scales, S, 2 * (er + 6 * U) * S)
    each = scales.to(F64).repeat_interleave(width, -1)[..., :C]
    value = y.to(F64) * each
    slack = 2 * (2 * er + 12 * U) * Y.abs()
    e["codes"] = worst(value, Y, torch.maximum(2.0 ** -4 * (Y.abs() + slack), 2.0 ** -10 * each) + slack)
    assert float(y.to(F64).abs().max()) <= 448
    return e


def backward_errors(cfg, h, rstd, dy, w, dh, dx, dw):
    C = cfg.C
    r, rw = half_step(cfg.dtype), half_step(cfg.wdtype)
    Hh, R, DY = h.to(F64), rstd.to(F64)[..., None], dy.to(F64)
    W = w.to(F64) if w is not None else torch.ones(C, dtype=F64, device="cuda")
    u, g = Hh * R, DY * W
    s = (g * u).mean(-1, keepdim=True)
    es = (C + 6) * U * (g * u).abs().mean(-1, keepdim=True)
    D = R * (g - u * s) + (dh.to(F64) if dh is not None else 0)
    ed = R * (u.abs() * es + 6 * U * (g.abs() + (u * s).abs())) + (2 * U + r) * D.abs()
    e = {}
    if dx is not None:
        e["dx"] = worst(dx, D, 2 * ed)
    if dw is not None:
        flat = (DY * u).reshape(-1, C)
        e["dw"] = worst(dw, flat.sum(0), 2 * ((len(flat) + 6) * U * flat.abs().sum(0) + rw * flat.sum(0).abs()))
    return e


def check(rows, C, dtype, wdtype="f32", layout="bhnd", residual=True, affine=True, out="same", group=0, seed=1,
          backward=True):
    cfg = mita.RmsConfig(rows, C, dtype=dtype, wdtype=wdtype, out=out, group=group)
    x, res, w, dy, dh = inputs(rows, C, dtype, wdtype, layout, seed, residual, affine)
    y = torch.full(cfg.shape, float("nan"), device="cuda").to(cfg.torch_ydtype) if layout == "bhnd" else None
    got = mita.rms_forward(cfg, x, w, res, y=y)
    e = forward_errors(cfg, x, res, w, got)
    if backward:
        h, rstd = got[2] if residual else x, got[3]
        dx = rows_of(gen(2), rows, C, cfg.torch_dtype, layout).fill_(float("nan"))
        ws = torch.full((max(1, mita.rms_workspace_size(cfg)),), 0xFF, dtype=torch.uint8, device="cuda")
        dx, dw = mita.rms_backward(cfg, h, rstd, dy, w, dh, dx=dx, ws=ws)
        e.update(backward_errors(cfg, h, rstd, dy, w, dh, dx, dw))
        again = mita.rms_backward(cfg, h, rstd, dy, w, dh, ws=ws)
        assert all(torch.equal(p, q) for p, q in zip((dx, dw), again))
    log(f"[rms] {cfg} {layout}: " + " ".join(f"{k} {v:.3f}" for k, v in e.items()))
    assert max(e.values()) <= 1.0, e


OUTS = [("same", 0), ("e4m3", 0), ("e4m3", 128)]
WIDTHS = [1, 2, 7, 8, 33, 64, 65, 120, 128, 130, 200, 256, 257, 384, 510, 512, 513, 768, 1021, 1024, 1500, 2048, 2056,
          4096, 4097, 5000, 8192, 8200, 16384, 20001]


@pytest.mark.parametrize("out", OUTS, ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", WIDTHS)
def test_widths(C, dtype, out):
    check((1, 1, 37), C, dtype, out=out[0], group=out[1], backward=out[0] == "same", residual=C % 3 != 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [(1, 1, 1), (1, 1, 5), (3, 1, 7), (2, 3, 1100), (1, 1, 9001)], ids=str)
def test_rows(rows, dtype):
    check(rows, 64, dtype)
    check(rows, 72, dtype, wdtype="bf16" if dtype == "bf16" else "f32", residual=False, out="e4m3")
    check(rows, 200, dtype, affine=False, out="e4m3", group=128)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C,many", [(64, 70000), (384, 20000), (768, 17000), (333, 9000)])
def test_several_rows_per_thread_group(C, many, dtype):
    check((many,), C, dtype, out="e4m3", group=128)
    check((many,), C, dtype, backward=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [768, 4096, 8192])
def test_inputs_of_128_mb_and_more(C, dtype):
    rows = 2 ** 27 // (C * (2 if dtype == "bf16" else 4)) + 3
    check((rows,), C, dtype, residual=False, out="e4m3", group=128)
    check((rows // 2 + 1,), C, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["bnhd", "qkv", "padded"])
@pytest.mark.parametrize("C", [64, 100, 768])
def test_strides(C, layout, dtype):
    check((2, 5, 77), C, dtype, layout=layout)
    check((2, 5, 77), C, dtype, layout=layout, out="e4m3", group=128)


def test_inputs_of_different_strides_and_alignments():
    g = gen(3)
    C = 96
    for off in (0, 1, 2, 8):
        cfg = mita.RmsConfig((50,), C, out="e4m3", group=128)
        x = torch.randn((50, C), device="cuda", generator=g).bfloat16()
        res = torch.randn((50, C + 16), device="cuda", generator=g).bfloat16()[:, off:off + C]
        y = torch.zeros((50, C + 9), dtype=torch.uint8, device="cuda")
        h = torch.zeros((50, 2 * C), dtype=torch.bfloat16, device="cuda")
        got = mita.rms_forward(cfg, x, res=res, h=h[:, off:off + C], y=y.view(torch.float8_e4m3fn)[:, off:off + C])
        assert max(forward_errors(cfg, x, res, None, got).values()) <= 1.0
        # nothing beside the rows was written
        assert (y[:, :off] == 0).all() and (y[:, off + C:] == 0).all()
        assert (h[:, :off] == 0).all() and (h[:, off + C:] == 0).all()


@pytest.mark.parametrize("C", [384, 20001])
def test_outputs_in_their_inputs_places(C):
    cfg = mita.RmsConfig((40,), C)
    x, res, w, dy, dh = inputs((40,), C, "bf16", "f32", "bhnd", 5)
    y, _, h, rstd = mita.rms_forward(cfg, x, w, res)
    for swap in (False, True):
        a, b = x.clone(), res.clone()
        to = dict(y=a, h=b) if not swap else dict(y=b, h=a)
        mita.rms_forward(cfg, a, w, b, **to)
        assert torch.equal(to["y"], y) and torch.equal(to["h"], h)
    dx, dw = mita.rms_backward(cfg, h, rstd, dy, w, dh)
    for t in ("dy", "dh"):
        z = dict(dy=dy.clone(), dh=dh.clone())
        _, dw2 = mita.rms_backward(cfg, h, rstd, z["dy"], w, z["dh"], dx=z[t])
        assert torch.equal(z[t], dx) and torch.equal(dw2, dw)
    only, none = mita.rms_backward(cfg, h, rstd, dy, w, dh, want_weight=False)
    assert torch.equal(only, dx) and none is None
    none, dw3 = mita.rms_backward(cfg, h, rstd, dy, w, dh, want_dx=False)
    assert none is None and torch.equal(dw3, dw)
    # without the sum or the statistics; the sum of x alone is x
    y2, _, n1, n2 = mita.rms_forward(cfg, x, w, res, want_h=False, want_rstd=False)
    assert torch.equal(y2, y) and n1 is None and n2 is None
    _, _, same, _ = mita.rms_forward(cfg, x, w, h=torch.empty_like(x))
    assert torch.equal(same, x)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C,group", [(320, 0), (320, 128), (333, 128), (20001, 0), (20001, 128)])
def test_values_at_the_ends_of_eight_bits(C, group, dtype):
    cfg = mita.RmsConfig((9,), C, dtype=dtype, out="e4m3", group=group, eps=1e-30)
    g = gen(6)
    x = torch.randn((9, C), device="cuda", generator=g).to(cfg.torch_dtype)
    x[0] = 0                    # a row without values: codes 0, the smallest scale
    x[1] = 1                    # equal values: every code the largest
    x[2] = -x[2].abs()
    x[3] *= 1e-6                # values near the type's smallest steps beside one large one
    x[3, 3] = 1
    x[4] *= 1e-4                # eps far below
    x[5, : C // 2] = 0          # a group without values beside others
    got = mita.rms_forward(cfg, x)
    y, scales, _, _ = got
    e = forward_errors(cfg, x, None, None, got)
    log(f"[rms] ends {cfg}: {e}")
    assert max(e.values()) <= 1.0
    assert (y[0].float() == 0).all() and (scales[0] == torch.tensor(2.0 ** -117) / 448).all()
    assert (y[1].float() == 448).all()
    assert torch.isfinite(y.float()).all() and torch.isfinite(scales).all() and (scales > 0).all()


def test_a_row_that_is_not_finite_stays_alone():
    for kw in (dict(), dict(out="e4m3"), dict(out="e4m3", group=128)):
        cfg = mita.RmsConfig((50,), 256, **kw)
        g = gen(7)
        x = torch.randn((50, 256), device="cuda", generator=g).bfloat16()
        ok = mita.rms_forward(cfg, x)
        bad = x.clone()
        bad[7, 3], bad[20, 200] = float("nan"), float("inf")
        got = mita.rms_forward(cfg, bad)
        keep = [i for i in range(50) if i not in (7, 20)]
        for a, b in zip(ok, got):
            if a is not None:
                assert torch.equal(a[keep].float(), b[keep].float())
        assert torch.isnan(got[0][7].float()).all() and torch.isnan(got[3][7])


def test_more_rows_than_one_grid_dimension():
    """2^27 + 5 rows of 9, a wave each, two rows per wave: 2^32 threads and more."""
    g = gen(12)
    R, C = 2 ** 27 + 5, 9
    cfg = mita.RmsConfig((R,), C)
    x = torch.randn((R, C), device="cuda", generator=g, dtype=torch.bfloat16)
    y, _, _, rstd = mita.rms_forward(cfg, x, y=torch.full_like(x, float("nan")))
    dx, _ = mita.rms_backward(cfg, x, rstd, x, dx=torch.full_like(x, float("nan")), want_weight=False)
    for at in (0, 2 ** 24 - 500, 2 ** 26, R - 1000):
        part = mita.RmsConfig((1000,), C)
        i = slice(at, at + 1000)
        e = forward_errors(part, x[i], None, None, (y[i], None, None, rstd[i]))
        e.update(backward_errors(part, x[i], rstd[i], x[i], None, None, dx[i], None))
        assert max(e.values()) <= 1.0, e
    assert all(bool(torch.isfinite(t).all()) for t in (y, rstd, dx))


def test_gradient_against_differences():
    cfg = mita.RmsConfig((2, 9), 40, dtype="f32")
    x, res, w, dy, dh = inputs((2, 9), 40, "f32", "f32", "bhnd", 8)
    y, _, h, rstd = mita.rms_forward(cfg, x, w, res)
    dx, dw = mita.rms_backward(cfg, h, rstd, dy, w, dh)

    def f(x, res, w):
        v = x + res
        return float((v * ((v * v).mean(-1, keepdim=True) + cfg.eps).rsqrt() * w * dy.double()).sum()
                     + (v * dh.double()).sum())

    at = [t.double() for t in (x, res, w)]
    g = gen(9)
    for i, grad in enumerate((dx, dx, dw)):  # the residual's gradient is x's
        way = torch.randn(grad.shape, device="cuda", generator=g, dtype=F64)
        hi, lo = ([t + (s * 1e-4 * way if j == i else 0) for j, t in enumerate(at)] for s in (1, -1))
        # truncation: 1e-8 / 6 of a third derivative of the order of the sums' size, about 1e3
        assert abs(float((grad.double() * way).sum()) - (f(*hi) - f(*lo)) / 2e-4) <= 1e-4


def test_streams_and_a_graph_with_eager_calls_in_between():
    cfg = mita.RmsConfig((2, 300), 768, out="e4m3", group=128)
    x, res, w, dy, dh = inputs((2, 300), 768, "bf16", "f32", "bhnd", 10)
    ws = torch.empty(mita.rms_workspace_size(cfg), dtype=torch.uint8, device="cuda")

    def both(ws=None, stream=None):
        y, s, h, r = mita.rms_forward(cfg, x, w, res, stream=stream)
        return (y.view(torch.uint8), s, h, r) + mita.rms_backward(cfg, h, r, dy, w, dh, ws=ws, stream=stream)

    first = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [both(stream=side) for _ in range(5)]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for o in got for p, q in zip(first, o))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both(ws)
    for seed in (1, 2, 3):
        g = gen(seed)
        for t in (x, res, dy, dh):
            t.copy_(torch.randn(t.shape, device="cuda", generator=g))
        eager = both(ws)
        for t in out:
            t.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(eager, out))


def test_refusals():
    g = gen(11)
    x, res = (torch.randn((4, 64), device="cuda", generator=g).bfloat16() for _ in range(2))
    cfg, e4 = mita.RmsConfig((4,), 64), mita.RmsConfig((4,), 64, out="e4m3", group=128)
    bad = lambda c, *a, **kw: pytest.raises(ValueError, mita.rms_forward, c, *a, **kw)
    bad(cfg, x.cpu())
    bad(cfg, x.float())
    bad(cfg, x[:3])
    bad(cfg, x, torch.ones(63, device="cuda"))
    bad(cfg, x, torch.ones(64, device="cuda").bfloat16())
    bad(cfg, x, res=res.float())
    bad(cfg, x, res=res[:, ::2])
    bad(cfg, x, scales=torch.empty((4, 1), device="cuda"))
    bad(cfg, x, y=torch.empty((4, 64), device="cuda"))
    bad(e4, x, y=torch.empty_like(x))
    bad(e4, x, scales=torch.empty((4, 2), device="cuda"))
    buf = torch.randn((5, 64), device="cuda", generator=g).bfloat16()
    for kw in (dict(y=buf[1:]), dict(h=buf[1:]), dict(res=buf[1:], h=buf[:4], y=buf[:4])):
        with pytest.raises(mita.MitaError) as e:
            mita.rms_forward(cfg, buf[:4], **kw)
        assert e.value.status == mita.MITA_ERR_INVALID_ARG
    y, _, h, rstd = mita.rms_forward(cfg, x, res=res)
    for kw in (dict(dx=h), dict(want_dx=False, want_weight=False)):
        with pytest.raises(mita.MitaError) as e:
            mita.rms_backward(cfg, h, rstd, y, **kw)
        assert e.value.status == mita.MITA_ERR_INVALID_ARG
    with pytest.raises(mita.MitaError) as e:
        mita.rms_backward(cfg, h, rstd, y, ws=torch.empty(8, dtype=torch.uint8, device="cuda"))
    assert e.value.status == mita.MITA_ERR_WORKSPACE

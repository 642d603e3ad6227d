"""Rotary positions and their gradients on the GPU against float64.

Bounds, with u = 2^-24 and r = 2^-8 (half a step of bf16) or 0: an angle of t turns,
formed and reduced in 64 bits, is off by 2^-50 |t| turns; the eighth of a turn that is
left (0.79 at most) by 3 u of itself; the sine's and cosine's sums by 2 u; so they are
off by 5 u and 2^-47 |t|, times the scale (one more u) by 6 u in all. A product adds
u, their difference u of the larger: |dy| <= s (|a| + |b|) (10 u + 2^-47 |t|) + r |y|,
the rounding to bf16 taken of the value as it is (2^-8 of it more)."""
from __future__ import annotations

import math

import pytest
import torch

from paper_2602_01219_amd import mita
from tests.dense_reference import U, worst
from tests.gpu_helpers import log
from tests.test_gpu_norm import gen, half_step

pytestmark = pytest.mark.gpu
F64 = torch.float64


def rates(cfg):
    """Radians per position of each pair."""
    rot, base = cfg.rot or cfg.d, cfg.base
    if cfg.scaling == "base" and rot > 2:
        base *= cfg.factor ** (rot / (rot - 2))
    out = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        if cfg.scaling == "linear":
            f /= cfg.factor
        if cfg.scaling == "parts":
            t = cfg.trained * f / (2 * math.pi)
            c = min(1.0, max(0.0, (t - cfg.slow) / (cfg.fast - cfg.slow)))
            f = c * f + (1 - c) * f / cfg.factor
        out.append(f)
    return torch.tensor(out, dtype=F64, device="cuda")


def pairs(cfg):
    rot = cfg.rot or cfg.d
    i = torch.arange(rot // 2)
    return (2 * i, 2 * i + 1) if cfg.interleaved else (i, i + rot // 2)


def reference(cfg, x, pos, back=False):
    """The rotated x and its bound."""
    p = torch.arange(cfg.N, device="cuda") + cfg.first if pos is None else pos
    p = p.to(F64) if p.dim() == 2 else p.to(F64)[None]
    a = (p[..., None] * rates(cfg))[:, None]
    s = cfg.scale or 1.0
    c, sn = torch.cos(a) * s, torch.sin(a) * (-s if back else s)
    i, j = pairs(cfg)
    X = x.to(F64)
    Y, E = X.clone(), torch.zeros_like(X)
    Y[..., i] = X[..., i] * c - X[..., j] * sn
    Y[..., j] = X[..., j] * c + X[..., i] * sn
    e = s * (X[..., i].abs() + X[..., j].abs()) * (10 * U + 2.0 ** -47 * a.abs() / (2 * math.pi))
    r = half_step(cfg.dtype)
    E[..., i] = e + r * (1 + 2.0 ** -8) * (Y[..., i].abs() + e)
    E[..., j] = e + r * (1 + 2.0 ** -8) * (Y[..., j].abs() + e)
    return Y, E


def heads(g, B, H, N, d, dtype, layout):
    if layout == "bnhd":
        return torch.randn((B, N, H, d), device="cuda", generator=g).to(dtype).transpose(1, 2)
    if layout.startswith("off"):  # rows further apart, off by so many elements
        k = int(layout[3:])
        return torch.randn((B, H, N, d + 16), device="cuda", generator=g).to(dtype)[..., k:k + d]
    return torch.randn((B, H, N, d), device="cuda", generator=g).to(dtype)


def check(cfg, layout="bhnd", pos="count", seed=1):
    g = gen(seed)
    B, H, N, d = cfg.q_shape
    Hk = cfg.k_shape[1]
    dt = cfg.torch_dtype
    if layout == "qkv":
        x = torch.randn((B, N, 3, H, d), device="cuda", generator=g).to(dt)
        q, k = (x[:, :, i].transpose(1, 2) for i in range(2))
    else:
        q, k = (heads(g, B, h, N, d, dt, layout) for h in (H, Hk))
    p = None
    if pos == "shared":
        p = torch.randint(-1000, 1 << 20, (N,), device="cuda", generator=g, dtype=torch.int32)
    elif pos == "own":
        p = torch.randint(0, 1 << 20, (B, N), device="cuda", generator=g, dtype=torch.int32)
    e = {}
    for fn, back in ((mita.rope_forward, False), (mita.rope_backward, True)):
        qo, ko = fn(cfg, q, k, p)
        for name, x, y in (("q", q, qo), ("k", k, ko)):
            Y, E = reference(cfg, x, p, back)
            e[name + "_back" * back] = worst(y, Y, E)
            rot = cfg.rot or d
            assert torch.equal(y[..., rot:], x[..., rot:])
        # in place, and queries alone
        q2, k2 = (torch.empty_strided(t.shape, t.stride(), dtype=dt, device="cuda").copy_(t) for t in (q, k))
        fn(cfg, q2, k2, p, q2, k2)
        assert torch.equal(q2, qo) and torch.equal(k2, ko)
        q2 = torch.empty_strided(q.shape, q.stride(), dtype=dt, device="cuda").copy_(q)
        k2 = torch.full_like(k, float("nan"))
        fn(cfg, q2, k, p, q2, k2)  # one of them in place
        assert torch.equal(q2, qo) and torch.equal(k2, ko)
        only, none = fn(cfg, q, pos=p)
        assert torch.equal(only, qo) and none is None
    log(f"[rope] {cfg} {layout} {pos}: " + " ".join(f"{n} {v:.3f}" for n, v in e.items()))
    assert max(e.values()) <= 1.0, e


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "inter"])
@pytest.mark.parametrize("d,rot", [(64, 0), (128, 0), (64, 32), (128, 24), (80, 20), (64, 2), (96, 90), (6, 4), (2, 2),
                                   (7, 4), (33, 32), (256, 0), (256, 66)])
def test_parts_of_the_head(d, rot, interleaved, dtype):
    for layout, pos in (("bhnd", "count"), ("bnhd", "own"), ("qkv", "shared")):
        check(mita.RopeConfig(2, 3, 37, d, rot=rot, dtype=dtype, interleaved=interleaved), layout, pos)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "inter"])
@pytest.mark.parametrize("layout", ["off1", "off2", "off4", "off8"])
def test_alignments(layout, interleaved, dtype):
    check(mita.RopeConfig(2, 4, 33, 64, H_kv=2, dtype=dtype, interleaved=interleaved), layout, "own")
    check(mita.RopeConfig(1, 4, 33, 64, H_kv=1, rot=40, dtype=dtype, interleaved=interleaved), layout)


@pytest.mark.parametrize("shape", [(1, 1, 1, 1), (24, 32, 8, 1), (1, 8, 2, 5000), (3, 5, 7, 129), (300, 1, 1, 3)], ids=str)
def test_sizes(shape):
    B, H, Hk, N = shape
    check(mita.RopeConfig(B, H, N, 128, H_kv=Hk), "bnhd", "own")
    check(mita.RopeConfig(B, H, N, 64, H_kv=Hk, dtype="f32", interleaved=True, first=70000), "bhnd")


@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "inter"])
@pytest.mark.parametrize("dtype,N,rot", [("bf16", 16390, 0), ("bf16", 16390, 48), ("f32", 8200, 0)])
def test_inputs_of_128_mb_and_more(dtype, N, rot, interleaved):
    check(mita.RopeConfig(2, 12, N, 128, H_kv=4, rot=rot, dtype=dtype, interleaved=interleaved), "bnhd")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scaling", ["linear", "base", "parts"])
def test_long_contexts(scaling, dtype):
    more = dict(trained=4096, slow=1.0, fast=32.0, scale=1.3) if scaling == "parts" else {}
    for d, rot in ((64, 0), (128, 64), (64, 2), (64, 4)):
        check(mita.RopeConfig(1, 2, 700, d, rot=rot, dtype=dtype, scaling=scaling, factor=8.0, first=100000, **more))


def test_scalings_that_change_nothing():
    g = gen(2)
    q = torch.randn((1, 2, 90, 64), device="cuda", generator=g)
    plain, _ = mita.rope_forward(mita.RopeConfig(1, 2, 90, 64, dtype="f32"), q)
    for kw in (dict(scaling="linear"), dict(scaling="base"), dict(scaling="parts", trained=100, fast=2.0)):
        y, _ = mita.rope_forward(mita.RopeConfig(1, 2, 90, 64, dtype="f32", **kw), q)
        # the rates agree to 64-bit roundings, far below an fp32 step of the angle: sums may round apart once
        assert float((y - plain).abs().max()) <= 4 * U * float(q.abs().max())


def test_positions_at_the_ends_of_32_bits():
    # one sequence's positions are far from the other's, the same angles as in 64 bits
    cfg = mita.RopeConfig(2, 2, 3, 64, dtype="f32")
    g = gen(3)
    q = torch.randn((2, 2, 3, 64), device="cuda", generator=g)
    pos = torch.tensor([[2 ** 31 - 1, -2 ** 31, 0], [2 ** 30 + 1, -1, 1]], dtype=torch.int32, device="cuda")
    y, _ = mita.rope_forward(cfg, q, pos=pos)
    Y, E = reference(cfg, q, pos)
    assert worst(y, Y, E) <= 1.0
    for first in (2 ** 31, -2 ** 31):
        cfg = mita.RopeConfig(2, 2, 3, 64, dtype="f32", first=first)
        y, _ = mita.rope_forward(cfg, q)
        Y, E = reference(cfg, q, None)
        assert worst(y, Y, E) <= 1.0


def test_there_and_back():
    # the rotation's transpose is its inverse, times the scale twice
    cfg = mita.RopeConfig(2, 3, 50, 128, dtype="f32", rot=96, scale=1.5)
    g = gen(4)
    q = torch.randn((2, 3, 50, 128), device="cuda", generator=g)
    y, _ = mita.rope_forward(cfg, q)
    z, _ = mita.rope_backward(cfg, y)
    want = torch.cat((q[..., :96] * 2.25, q[..., 96:]), -1)
    # two passes: (|a| + |b|) (10 u) s s, and the second's of |y| <= s (|a| + |b|); twice each
    assert float((z - want).abs().max()) <= 4 * 2.25 * 10 * U * 2 * float(q.abs().max()) * 2


def test_gradient_against_differences():
    cfg = mita.RopeConfig(1, 2, 9, 64, H_kv=1, dtype="f32", rot=32, interleaved=True, scale=0.7, first=12345)
    g = gen(5)
    q, dq = (torch.randn((1, 2, 9, 64), device="cuda", generator=g) for _ in range(2))
    k, dk = (torch.randn((1, 1, 9, 64), device="cuda", generator=g) for _ in range(2))
    grads = mita.rope_backward(cfg, dq, dk)
    for x, dy, grad in zip((q, k), (dq, dk), grads):
        f = lambda z: float((reference(cfg, z, None)[0] * dy.double()).sum())
        way = torch.randn(x.shape, device="cuda", generator=g, dtype=F64)
        diff = (f(x.double() + 1e-3 * way) - f(x.double() - 1e-3 * way)) / 2e-3  # linear: no truncation
        # fp32 gradients of size 5 in 1152 elements, each off by 10 u (|a| + |b|)
        assert abs(float((grad.double() * way).sum()) - diff) <= 1152 * 10 * U * 10 * 4


def test_inputs_that_repeat():
    cfg = mita.RopeConfig(3, 4, 40, 64)
    g = gen(6)
    one = torch.randn((1, 1, 40, 64), device="cuda", generator=g).bfloat16()
    pos = torch.arange(40, device="cuda", dtype=torch.int32)
    y, z = mita.rope_forward(cfg, one.expand(3, 4, 40, 64), one.expand(3, 4, 40, 64), pos)
    a, _ = mita.rope_forward(mita.RopeConfig(1, 1, 40, 64), one)
    assert all(torch.equal(t, a.expand(3, 4, 40, 64)) for t in (y, z))
    token = torch.randn((3, 4, 1, 64), device="cuda", generator=g).bfloat16()
    y, _ = mita.rope_forward(cfg, token.expand(3, 4, 40, 64), pos=pos)
    b, _ = mita.rope_forward(cfg, token.expand(3, 4, 40, 64).contiguous(), pos=pos)
    assert torch.equal(y, b)


def test_only_the_tensors_are_written():
    # queries and keys rotated inside a fused projection's buffer: values and padding stay
    g = gen(7)
    x = torch.randn((2, 30, 3, 4, 64), device="cuda", generator=g).bfloat16()
    before = x.clone()
    q, k = (x[:, 1:25, i].transpose(1, 2) for i in range(2))
    cfg = mita.RopeConfig(2, 4, 24, 64, rot=32)
    want = mita.rope_forward(cfg, q, k)
    mita.rope_forward(cfg, q, k, qo=q, ko=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    keep = torch.ones(x.shape, dtype=torch.bool)
    keep[:, 1:25, :2, :, :32] = False
    assert torch.equal(x.cpu()[keep], before.cpu()[keep])


def test_grouped_heads_in_place_in_a_fused_projection():
    # 6 query heads, 2 key heads and 2 value heads of a token side by side
    g = gen(11)
    x = torch.randn((2, 30, 10, 64), device="cuda", generator=g).bfloat16()
    before = x.clone()
    q, k = x[:, :, :6].transpose(1, 2), x[:, :, 6:8].transpose(1, 2)
    cfg = mita.RopeConfig(2, 6, 30, 64, H_kv=2)
    want = mita.rope_forward(cfg, q, k)
    mita.rope_forward(cfg, q, k, qo=q, ko=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(x[:, :, 8:], before[:, :, 8:])
    with pytest.raises(mita.MitaError):  # the keys' output one head into the queries
        mita.rope_forward(cfg, q, k, qo=q, ko=x[:, :, 5:7].transpose(1, 2))


def test_values_that_are_not_finite():
    # a NaN or an infinity stays in its pair; what does not turn is copied bit for bit
    cfg = mita.RopeConfig(2, 2, 30, 64, rot=32)
    g = gen(10)
    q = torch.randn((2, 2, 30, 64), device="cuda", generator=g).bfloat16()
    ok, _ = mita.rope_forward(cfg, q)
    bad = q.clone()
    bad[0, 1, 7, 3], bad[1, 0, 9, 20] = float("nan"), float("inf")
    bad.view(torch.int16)[..., 40:] = torch.randint(-2 ** 15, 2 ** 15, (2, 2, 30, 24), device="cuda", generator=g).short()
    y, _ = mita.rope_forward(cfg, bad)
    keep = torch.ones(q.shape, dtype=torch.bool, device="cuda")
    keep[0, 1, 7, [3, 19]] = keep[1, 0, 9, [4, 20]] = False
    keep[..., 40:] = False
    assert torch.equal(y[keep], ok[keep]) and not torch.isfinite(y[0, 1, 7, [3, 19]]).any()
    assert torch.equal(y[..., 32:].view(torch.int16), bad[..., 32:].view(torch.int16))


def test_offsets_past_32_bits():
    N, H = 70000, 256
    cfg = mita.RopeConfig(1, 1, N, 128)
    g = gen(8)
    x = torch.randn((1, 1, N, 128), device="cuda", generator=g).bfloat16()
    far = torch.empty((1, N, H, 128), dtype=torch.bfloat16, device="cuda").transpose(1, 2)[:, H - 1:]
    far.copy_(x)
    y, _ = mita.rope_forward(cfg, x)
    assert torch.equal(mita.rope_forward(cfg, far, qo=torch.empty_like(x))[0], y)
    mita.rope_forward(cfg, x, qo=far)
    assert torch.equal(far, y)


def test_streams_and_a_graph_with_eager_calls_in_between():
    cfg = mita.RopeConfig(4, 8, 100, 64, H_kv=2)
    g = gen(9)
    q, k = (torch.randn((4, h, 100, 64), device="cuda", generator=g).bfloat16() for h in (8, 2))
    pos = torch.randint(0, 5000, (4, 100), device="cuda", generator=g, dtype=torch.int32)
    first = mita.rope_forward(cfg, q, k, pos)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [mita.rope_forward(cfg, q, k, pos, stream=side) for _ in range(5)]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for o in got for a, b in zip(first, o))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = mita.rope_forward(cfg, q, k, pos)
    for step in (1, 2, 3):  # the next token's positions, as a captured decoding step moves on
        pos += 1
        q.copy_(torch.randn(q.shape, device="cuda", generator=g))
        eager = mita.rope_forward(cfg, q, k, pos)
        for t in out:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, out))


def test_refusals():
    cfg = mita.RopeConfig(2, 4, 10, 64, H_kv=2)
    q, k = (torch.zeros((2, h, 10, 64), dtype=torch.bfloat16, device="cuda") for h in (4, 2))
    bad = lambda *a, **kw: pytest.raises(ValueError, mita.rope_forward, cfg, *a, **kw)
    bad(q.cpu(), k)
    bad(q.float(), k)
    bad(q, q)
    bad(q, k.transpose(2, 3).contiguous().transpose(2, 3))
    bad(q, k, torch.zeros((2, 10), dtype=torch.int64, device="cuda"))
    bad(q, k, torch.zeros((2, 9), dtype=torch.int32, device="cuda"))
    bad(q, k, torch.zeros((2, 20), dtype=torch.int32, device="cuda")[:, ::2])
    bad(q, ko=k)
    buf = torch.zeros((3, 4, 10, 64), dtype=torch.bfloat16, device="cuda")
    other = torch.empty_like(q)
    for kw in (dict(qo=buf[1:]), dict(k=buf[1:, :2], qo=other, ko=buf[:2, :2]),
               dict(k=k, qo=other, ko=other[:, :2]), dict(k=k, qo=other, ko=buf[:2, :2])):
        with pytest.raises(mita.MitaError) as e:
            mita.rope_forward(cfg, buf[:2], **kw)
        assert e.value.status == mita.MITA_ERR_INVALID_ARG

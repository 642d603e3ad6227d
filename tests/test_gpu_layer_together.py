"""The operators around attention as a decoder layer uses them: the sum with the
residual and its norm, projections (torch's products), rotary positions of queries
and keys, attention behind a shared prefix, and back."""
from __future__ import annotations

import pytest
import torch

from paper_2602_01219_amd import mita
from tests.test_gpu_norm import gen
from tests.test_gpu_rope import rates

pytestmark = pytest.mark.gpu
F64 = torch.float64

B, H, HK, D, C = 6, 4, 2, 64, 384  # sequences, heads, head size, width of the residual stream


def weights(g, dtype):
    w = {n: torch.randn((C, h * D), device="cuda", generator=g) * C ** -0.5 for n, h in (("q", H), ("k", HK), ("v", HK))}
    w["norm"] = 1 + 0.1 * torch.randn(C, device="cuda", generator=g)
    return {n: t if n == "norm" else t.to(dtype) for n, t in w.items()}


def project(y, w, heads):
    """[.., N, C] tokens to [.., heads, N, d], as the product writes it."""
    return (y @ w).unflatten(-1, (heads, D)).transpose(-2, -3)


def reference(x, res, w, first, N):
    """What one layer computes up to its attention's inputs, in float64 on tokens x + res at positions first .."""
    h = x + res
    y = h * (h.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * w["norm"]
    q, k, v = ((y @ w[n]).unflatten(-1, (z, D)).transpose(-2, -3) for n, z in (("q", H), ("k", HK), ("v", HK)))
    r = rates(mita.RopeConfig(1, 1, 1, D)).to(x.device)
    a = ((torch.arange(N, dtype=F64, device=x.device) + first)[:, None] * r)

    def turn(t):
        u, z = t[..., :D // 2], t[..., D // 2:]
        return torch.cat((u * a.cos() - z * a.sin(), z * a.cos() + u * a.sin()), -1)

    return h, turn(q), turn(k), v


def softmax(q, k, v, causal_from):
    """Attention of q over k, v; query i sees the keys up to causal_from + i."""
    k, v = (t.repeat_interleave(H // HK, -3) for t in (k, v))
    z = q @ k.transpose(-1, -2) / D ** 0.5
    j, i = torch.arange(k.shape[-2], device=q.device), torch.arange(q.shape[-2], device=q.device)
    return torch.softmax(z.masked_fill(j > causal_from + i[:, None], float("-inf")), -1) @ v


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_serving_a_prompt_and_single_tokens(dtype):
    """A prefix once, then each sequence's own question behind it, then single tokens that
    are appended to the sequences' caches, against the whole computed in float64 from the
    same (rounded) projections' inputs."""
    g = gen(1)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    w = weights(g, dt)
    P, N, STEPS = 210, 37, 3
    tokens = lambda *s: (torch.randn((*s, C), device="cuda", generator=g).to(dt) for _ in range(2))

    def layer(x, res, pos):
        """Queries, keys and values of tokens x + res at positions pos [B, N]."""
        b, n = x.shape[:2]
        y, _, h, _ = mita.rms_forward(mita.RmsConfig((b, n), C, dtype=dtype), x, w["norm"], res)
        q, k, v = (project(y, w[t], z) for t, z in (("q", H), ("k", HK), ("v", HK)))
        return (h, *mita.rope_forward(mita.RopeConfig(b, H, n, D, H_kv=HK, dtype=dtype), q, k, pos), v)

    at = lambda first, n: (first + torch.arange(n, device="cuda", dtype=torch.int32))
    xp, rp = tokens(1, P)
    _, _, kp, vp = layer(xp, rp, at(0, P))
    x, res = tokens(B, N + STEPS)
    ks, vs = (torch.full((B, HK, N + STEPS, D), float("nan"), device="cuda").to(dt) for _ in range(2))
    o = torch.empty((B, H, N + STEPS, D), device="cuda", dtype=dt)
    _, q, k, v = layer(x[:, :N], res[:, :N], at(P, N))
    ks[:, :, :N], vs[:, :, :N] = k, v
    cfg = mita.PrefixConfig(B, H, N, P, D, H_kv=HK, N_k=N + STEPS, dtype=dtype, right=0)
    lens = torch.full((B,), N, device="cuda", dtype=torch.int32)
    o[:, :, :N] = mita.prefix_forward(cfg, q, kp, vp, ks, vs, k_len=lens)[0]
    one = mita.PrefixConfig(B, H, 1, P, D, H_kv=HK, N_k=N + STEPS, dtype=dtype, right=0)
    for s in range(STEPS):
        t = N + s
        _, q, k, v = layer(x[:, t:t + 1], res[:, t:t + 1], lens[:, None] + P)
        ks[:, :, t:t + 1], vs[:, :, t:t + 1] = k, v
        lens += 1
        o[:, :, t:t + 1] = mita.prefix_forward(one, q, kp, vp, ks, vs, k_len=lens)[0]
    W = {n: t.to(F64) for n, t in w.items()}
    _, _, Kp, Vp = reference(xp.to(F64), rp.to(F64), W, 0, P)
    _, Q, K, V = reference(x.to(F64), res.to(F64), W, P, N + STEPS)
    R = softmax(Q, torch.cat((Kp.expand(B, -1, -1, -1), K), 2), torch.cat((Vp.expand(B, -1, -1, -1), V), 2), P)
    # every element of q, k and v is rounded at most four times on the way (norm, product, rotation, weights): a
    # score of size |q||k| / 8, at most 15 here, is off by 8 half steps of itself at most, and so is its weight
    # relatively; o by that and its values' and its own roundings. In fp32 the products' sums over 384 terms
    # count instead (386 u, each score 3 times): both with the sizes of the largest elements
    step = 2.0 ** -8 if dtype == "bf16" else 400 * 2.0 ** -24
    size = float((Q.norm(dim=-1).max() * torch.cat((Kp.expand(B, -1, -1, -1), K), 2).norm(dim=-1).max()) / 8)
    err = float((o.double() - R).abs().max())
    assert size < 25 and err <= (2 * 8 * step * size + 4 * step) * float(V.abs().max()), (err, size)


def test_training_gradients_against_autograd():
    """Norm, rotation and dense attention forward and backward in fp32, with the residual's
    path around them, against float64 autograd."""
    g = gen(2)
    N = 50
    w = weights(g, torch.float32)
    x, res = (torch.randn((B, N, C), device="cuda", generator=g) for _ in range(2))
    dO = torch.randn((B, H, N, D), device="cuda", generator=g)
    dh = torch.randn((B, N, C), device="cuda", generator=g)
    rms = mita.RmsConfig((B, N), C, dtype="f32")
    rope = mita.RopeConfig(B, H, N, D, H_kv=HK, dtype="f32", first=7)
    dense = mita.DenseConfig(B, H, N, D, H_kv=HK, dtype="f32", right=0)
    y, _, h, rstd = mita.rms_forward(rms, x, w["norm"], res)
    q, k, v = (project(y, w[t], z) for t, z in (("q", H), ("k", HK), ("v", HK)))
    qo, ko = mita.rope_forward(rope, q, k)
    o, lse = mita.dense_forward(dense, qo, ko, v)
    dqo, dko, dv = mita.dense_backward(dense, qo, ko, v, o, lse, dO)
    dq, dk = mita.rope_backward(rope, dqo, dko)
    dy = sum(t.transpose(1, 2).flatten(2) @ w[n].t() for n, t in (("q", dq), ("k", dk), ("v", dv)))
    dx, dw = mita.rms_backward(rms, h, rstd, dy, w["norm"], dh)

    leaf = [t.double().cpu().requires_grad_() for t in (x, res, w["norm"])]
    W = {n: t.double().cpu() for n, t in w.items()} | {"norm": leaf[2]}
    Hs, Q, K, V = reference(leaf[0], leaf[1], W, 7, N)
    O = softmax(Q, K, V, 0)
    torch.autograd.backward([O, Hs], [dO.double().cpu(), dh.double().cpu()])
    # fp32 throughout: sums of up to 384 products, scores up to about 25 in size (25 * 400 u = 6e-4 at the very
    # worst in a weight), so outputs and gradients are within 1e-3 of their largest element
    for name, got, ref in (("o", o, O.detach()), ("h", h, Hs.detach()), ("dx", dx, leaf[0].grad),
                           ("dres", dx, leaf[1].grad), ("dw", dw, leaf[2].grad)):
        err = float((got.double().cpu() - ref).abs().max() / ref.abs().max())
        assert err <= 1e-3, (name, err)


def test_eight_bit_output_in_a_product():
    """The norm's 8-bit output as a projection takes it: codes times scales, in groups of
    128 columns, against the product of the unrounded norm."""
    g = gen(3)
    x, res = (torch.randn((64, C), device="cuda", generator=g).bfloat16() for _ in range(2))
    w = weights(g, torch.float32)
    cfg = mita.RmsConfig((64,), C, out="e4m3", group=128)
    y, s, h, rstd = mita.rms_forward(cfg, x, w["norm"], res)
    got = sum((y[:, i * 128:(i + 1) * 128].double() * s[:, i:i + 1].double()) @ w["q"][i * 128:(i + 1) * 128].double()
              for i in range(3))
    full = x.double() + res.double()
    Y = full * (full.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * w["norm"].double()
    # a code is off by half a step at most: 2^-4 of its value, or 2^-10 of the scale; the sum by the sum of those
    # times |w|, and 1e-4 of it for the fp32 norm (C / 2 u = 1.1e-5 and the scales' roundings)
    half = torch.maximum(2.0 ** -4 * Y.abs(), 2.0 ** -10 * s.double().repeat_interleave(128, 1))
    bound = (half * (1 + 1e-4) + 1e-4 * Y.abs()) @ w["q"].double().abs()
    assert float(((got - Y @ w["q"].double()).abs() / bound).max()) <= 1.0

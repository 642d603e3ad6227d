"""A decoder layer as it serves: a shared prefix once, each sequence's own question behind it,
then single tokens that are appended to the sequences' caches. The outputs are compared
with the whole computed in float64 by their root mean square, which wrong compositions miss by
far (shown without a GPU), and every call with float64 on its own inputs by its own bounds.

Bound of the whole, r = 2^-8, a bf16 rounding being 0.58 r (rms) of an element: a query's, key's
or value's element passes three (norm, product, rotation; a value two), 1.0 r of it (0.8 r); a
score q.k / 8 of vectors of |q| = |k| = 8 is off by sqrt(2) 1.0 r |q||k| / (8 * 8) = 1.4 r, and
that is its weight's relative error; with the weight's and the output's own rounding o is off by
sqrt(1.4^2 + 0.8^2 + 2 * 0.58^2) r = 1.8 r of its size: 4 r is allowed. In fp32, u = 2^-24, a
product's 384 terms and a row's norm are off by about 8 u and 20 u, a score by some 40 u with
them, the sums over up to 250 keys by 10 u: about 80 u, and 400 u are allowed."""
from __future__ import annotations

import math

import pytest
import torch

from paper_2602_01219_amd import mita

F64 = torch.float64
B, H, HK, D, C = 6, 4, 2, 64, 384  # sequences, heads, head size, width of the residual stream
P, N, STEPS = 210, 37, 3           # prefix, question and single tokens
BOUND = {"bf16": 4 * 2.0 ** -8, "f32": 400 * 2.0 ** -24}


def inputs(seed, dtype):
    g = torch.Generator().manual_seed(seed)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    new = lambda *s: torch.randn(s, generator=g)
    s = {n: (new(C, h * D) * C ** -0.5).to(dt) for n, h in (("q", H), ("k", HK), ("v", HK))}
    s["norm"] = 1 + 0.1 * new(C)
    s.update({n: new(*b, C).to(dt) for n, b in (("xp", (1, P)), ("rp", (1, P)), ("x", (B, N + STEPS)), ("r", (B, N + STEPS)))})
    return s


class Host:
    """The layer's operators on the host in float64, each output rounded to `to`."""

    def __init__(self, to=F64):
        self.to = to

    def norm(self, x, res, w):
        h = x.to(F64) + res.to(F64)
        return (h * (h.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * w.to(F64)).to(self.to)

    def project(self, y, w, heads):
        return (y.to(F64) @ w.to(F64)).to(self.to).unflatten(-1, (heads, D)).transpose(-2, -3)

    def turn(self, q, k, pos):
        a = pos.to(F64)[:, None, :, None] * 10000.0 ** (-torch.arange(0, D, 2, dtype=F64) / D)

        def one(t):
            u, z = t.to(F64).chunk(2, -1)
            return torch.cat((u * a.cos() - z * a.sin(), z * a.cos() + u * a.sin()), -1).to(self.to)

        return one(q), one(k)

    def attend(self, q, kp, vp, k, v, n, drop=()):
        """Of queries at the ends of n own keys; keys of `drop` are left out."""
        n = int(n[0])
        K, V = (torch.cat((a.to(F64).expand(B, -1, -1, -1), b[:, :, :n].to(F64)), 2).repeat_interleave(H // HK, 1)
                for a, b in ((kp, k), (vp, v)))
        z = q.to(F64) @ K.transpose(-1, -2) / math.sqrt(D)
        j, i = torch.arange(P + n), torch.arange(q.shape[2]) + P + n - q.shape[2]
        hidden = j > i[:, None]
        if "prefix" in drop:
            hidden = hidden | (j < P)
        if "own" in drop:
            hidden = hidden | (j >= P)
        if "newest" in drop:
            hidden = hidden | (j == i[:, None])
        return (torch.softmax(z.masked_fill(hidden, -math.inf), -1).to(self.to).to(F64) @ V).to(self.to)


class Framework:
    """The same by the framework's calls, each compared with float64 on its own inputs."""

    def __init__(self, dtype):
        self.dtype = dtype

    def norm(self, x, res, w):
        from tests.test_gpu_rms import forward_errors
        cfg = mita.RmsConfig(x.shape[:2], C, dtype=self.dtype)
        got = mita.rms_forward(cfg, x, w, res)
        assert max(forward_errors(cfg, x, res, w, got).values()) <= 1.0
        return got[0]

    def project(self, y, w, heads):
        return (y @ w).unflatten(-1, (heads, D)).transpose(-2, -3)

    def turn(self, q, k, pos):
        from tests.dense_reference import worst
        from tests.test_gpu_rope import reference
        b, _, n, _ = q.shape
        cfg = mita.RopeConfig(b, H, n, D, H_kv=HK, dtype=self.dtype)
        got = mita.rope_forward(cfg, q, k, pos.contiguous())
        assert max(worst(y, *reference(cfg, x, pos)) for x, y in zip((q, k), got)) <= 1.0
        return got

    def attend(self, q, kp, vp, k, v, n):
        from tests.dense_reference import worst
        from tests.test_gpu_prefix import expected
        cfg = mita.PrefixConfig(B, H, q.shape[2], P, D, H_kv=HK, N_k=N + STEPS, dtype=self.dtype, right=0)
        o, lse = mita.prefix_forward(cfg, q, kp, vp, k, v, k_len=n)
        R = expected(cfg, (q, kp, vp, k, v), None, None, n.tolist())
        assert max(worst(o, R.o, R.eo), worst(lse, R.lse, R.elz)) <= 1.0
        return o


def serve(op, s, later=0, stale=False, **how):
    """o of the question's tokens and of each single token. Wrong on purpose: positions that are `later`, tokens that
    the caches miss (`stale`), keys that the attention drops."""
    dev = s["x"].device

    def layer(x, res, pos):
        y = op.norm(x, res, s["norm"])
        q, k, v = (op.project(y, s[t], z) for t, z in (("q", H), ("k", HK), ("v", HK)))
        return (*op.turn(q, k, pos), v)

    at = lambda first, n, b: (first + torch.arange(n, device=dev, dtype=torch.int32)).expand(b, n)
    _, kp, vp = layer(s["xp"], s["rp"], at(0, P, 1))
    ks, vs = (torch.full((B, HK, N + STEPS, D), float("nan"), device=dev, dtype=kp.dtype) for _ in range(2))
    q, k, v = layer(s["x"][:, :N], s["r"][:, :N], at(P + later, N, B))
    ks[:, :, :N], vs[:, :, :N] = k, v
    lens = torch.full((B,), N, device=dev, dtype=torch.int32)
    out = [op.attend(q, kp, vp, ks, vs, lens, **how)]
    for t in range(N, N + STEPS):
        q, k, v = layer(s["x"][:, t:t + 1], s["r"][:, t:t + 1], at(P + later + t, 1, B))
        if stale:
            k, v = ks[:, :, t - 1:t], vs[:, :, t - 1:t]
        ks[:, :, t:t + 1], vs[:, :, t:t + 1] = k, v
        lens += 1
        out.append(op.attend(q, kp, vp, ks, vs, lens, **how))
    return out


def off(got, ref):
    """Root mean square of each part's error, relative to that of the part."""
    return [float((a.double().cpu() - b).norm() / b.norm()) for a, b in zip(got, ref)]


@pytest.mark.parametrize("seed", [1, 2])
def test_wrong_layers_miss_the_bound(seed):
    s = inputs(seed, "bf16")
    ref = serve(Host(), s)
    wrong = dict(zeros=[torch.zeros_like(t) for t in ref], later=serve(Host(), s, later=1),
                 prefix=serve(Host(), s, drop=("prefix",)), own=serve(Host(), s, drop=("own",)),
                 newest=serve(Host(), s, drop=("newest",)))
    for name, o in wrong.items():
        assert min(off(o, ref)) > 2 * BOUND["bf16"], name
    assert min(off(serve(Host(), s, stale=True), ref)[1:]) > 2 * BOUND["bf16"]
    assert max(off(serve(Host(torch.bfloat16), s), ref)) <= BOUND["bf16"]
    s = inputs(seed, "f32")
    assert max(off(serve(Host(torch.float32), s), serve(Host(), s))) <= BOUND["f32"]


@pytest.mark.gpu
@pytest.mark.parametrize("seed", [1, 2])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_serving(dtype, seed):
    from tests.gpu_helpers import log
    s = inputs(seed, dtype)
    e = off(serve(Framework(dtype), {n: t.cuda() for n, t in s.items()}), serve(Host(), s))
    log(f"[serving] {dtype} {seed}: " + " ".join(f"{x / BOUND[dtype]:.3f}" for x in e))
    assert max(e) <= BOUND[dtype]

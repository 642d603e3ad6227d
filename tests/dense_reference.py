"""Dense attention and its gradients in float64 from the definitions, with a
bound on what the kernels' roundings may change, element by element.

u = 2^-24 is half a step of fp32; r = 2^-8 half a step of bf16 (0 in fp32),
the rounding of the weights, of dS and of the outputs. To first order:
 - a score is a d-term fp32 dot (|dz| <= scale (d + 4) u |q|.|k|), and the
   exponent z - m (or z - lse) adds 8 u (|z| + |lse| + 1) in all: ez;
 - a weight is off by its exponent's error and r; o is a ratio of two sums of
   weights over at most n keys: |do| <= sum P (ez + r + n u) (|v| + |o|) + r |o|;
 - dP - D: (d + 4) u (|dO|.|v| + |dO|.|o|) =: ep; dS = P (dP - D) is off by
   |dS| (ez + r) + P ep; sums over n terms add n u.
Every bound is doubled for the second-order terms."""
import math

import torch

U = 2.0 ** -24


class Ref:
    """o, lse, dq, dk, dv (float64, laid out like the kernels' outputs) and the
    bounds eo, else, edq, edk, edv."""


def visible(n, m, left, right, device):
    i = torch.arange(n, device=device)[:, None] + (m - n)
    j = torch.arange(m, device=device)[None, :]
    ok = torch.ones((n, m), dtype=torch.bool, device=device)
    if left >= 0:
        ok &= j >= i - left
    if right >= 0:
        ok &= j <= i + right
    return ok


def reference(cfg, q, k, v, q_len=None, k_len=None, dO=None, o=None, lse=None):
    """With dO: the gradients too, for the forward's given outputs o and lse."""
    dev, f64 = q.device, torch.float64
    B, H, N, d = cfg.q_shape
    Hk, Nk = cfg.k_shape[1:3]
    G = H // Hk
    r = 2.0 ** -8 if cfg.dtype == "bf16" else 0.0
    scale = cfg.scale or 1.0 / math.sqrt(d)
    R = Ref()
    zq = lambda: torch.zeros((B, H, N, d), dtype=f64, device=dev)
    zk = lambda: torch.zeros((B, Hk, Nk, d), dtype=f64, device=dev)
    R.o, R.eo = zq(), zq()
    R.lse = torch.full((B, H, N), -math.inf, dtype=f64, device=dev)
    R.elz = torch.zeros((B, H, N), dtype=f64, device=dev)
    R.dq, R.edq, R.dk, R.edk, R.dv, R.edv = zq(), zq(), zk(), zk(), zk(), zk()
    for b in range(B):
        n = N if q_len is None else int(q_len[b])
        m = Nk if k_len is None else int(k_len[b])
        if n == 0 or m == 0:
            continue
        ok = visible(n, m, cfg.left, cfg.right, dev)
        some = ok.any(1)
        for h in range(H):
            Q, K, V = q[b, h, :n].to(f64), k[b, h // G, :m].to(f64), v[b, h // G, :m].to(f64)
            z = scale * (Q @ K.T)
            zm = z.masked_fill(~ok, -math.inf)
            t = torch.logsumexp(zm, 1)
            t0 = torch.where(some, t, torch.zeros_like(t))
            P = torch.exp(zm - t0[:, None])
            ez = scale * (d + 4) * U * (Q.abs() @ K.abs().T) + 8 * U * (z.abs() + t0.abs()[:, None] + 1)
            w = P * (ez + r + m * U)
            O = P @ V
            R.o[b, h, :n] = O
            R.lse[b, h, :n] = t
            R.eo[b, h, :n] = 2 * (w @ V.abs() + w.sum(1, keepdim=True) * O.abs() + r * O.abs())
            R.elz[b, h, :n] = 2 * (P * (ez + m * U)).sum(1) + 4 * U * t0.abs()
            if dO is None:
                continue
            g, oo = dO[b, h, :n].to(f64), o[b, h, :n].to(f64)
            tl = lse[b, h, :n].to(f64)
            P = torch.exp(zm - torch.where(some, tl, torch.zeros_like(tl))[:, None])
            D = (g * oo).sum(1, keepdim=True)
            S = P * (g @ V.T - D)
            ep = (d + 4) * U * (g.abs() @ V.abs().T + (g * oo).abs().sum(1, keepdim=True))
            eS = S.abs() * (ez + r) + P * ep
            eP = P * (ez + r)
            R.dq[b, h, :n] = scale * (S @ K)
            R.edq[b, h, :n] = 2 * scale * ((eS + m * U * S.abs()) @ K.abs()) + 2 * r * R.dq[b, h, :n].abs()
            R.dk[b, h // G, :m] += scale * (S.T @ Q)
            R.dv[b, h // G, :m] += P.T @ g
            R.edk[b, h // G, :m] += 2 * scale * ((eS + G * n * U * S.abs()).T @ Q.abs())
            R.edv[b, h // G, :m] += 2 * ((eP + G * n * U * P).T @ g.abs())
    R.edk += 2 * r * R.dk.abs()
    R.edv += 2 * r * R.dv.abs()
    return R


def worst(got, ref, bound, tiny=1e-30):
    """Largest |got - ref| / bound; infinite where got is not finite and ref is."""
    got = got.to(torch.float64)
    same = torch.isinf(ref) & (got == ref)
    x = torch.where(same, torch.zeros_like(got), (got - ref).abs() / (bound + tiny))
    x = torch.where(torch.isnan(x), torch.full_like(x, math.inf), x)
    return float(x.max()) if x.numel() else 0.0

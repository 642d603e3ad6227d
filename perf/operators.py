"""Performance cases of the operators beside MiTA that a layer is built from:
dense attention (forward, single tokens against long key sequences, and the
backward pass) and the layer norm of queries, keys and tokens (forward and
backward).

A case is one call that a program makes, on device tensors it already holds:

  op "attend"           o and the rows' log-sum-exps
  op "attend_backward"  dq, dk, dv from the forward's o and log-sum-exps
  op "norm"             y and the rows' mean and 1 / standard deviation
  op "norm_backward"    dx and the weight's and bias's gradients

Layouts: "bhnd" contiguous heads, "bnhd" the [B, N, H, d] that a projection
writes, seen as [B, H, N, d], "qkv" the slices of one fused projection
[B, N, 3, H, d]. With "ragged" every sequence of the batch has its own length
(the last one none at all with "empty"); rows and keys behind a sequence's end
are padding. left and right bound how far a query at position p sees (-1: no
bound; right = 0 is causal); a sequence's last query stands at its last key.

With own = False, run() uses elementary torch operations in 32 bits; exact()
follows the definitions in 64 bits and shares nothing with them but the inputs.
"""
import math

import torch

own = False


def _attn(name, op, B, H, H_kv, N, N_k, d, dtype, layout="bhnd", ragged=False, empty=False, left=-1, right=-1):
    c = dict(op=op, B=B, H=H, H_kv=H_kv, N=N, N_k=N_k, d=d, dtype=dtype, layout=layout, ragged=ragged, empty=empty,
             left=left, right=right)
    if name:
        c["name"] = name
    return c


def _norm(name, op, n0, n1, n2, C, dtype, wdtype="f32", layout="bhnd"):
    c = dict(op=op, n0=n0, n1=n1, n2=n2, C=C, dtype=dtype, wdtype=wdtype, layout=layout)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one query token over the 196 tokens of one image in fp32: the smallest call, all latency
        _attn("pool_token_f32", "attend", 1, 6, 6, 1, 196, 64, "f32"),
        # a batch of images through a dense ViT-S layer, straight from its fused projection
        _attn("vit_bf16", "attend", 64, 6, 6, 196, 196, 64, "bf16", "qkv"),
        # 16384 tokens, head dimension 128: what the top-k experts are compared with
        _attn("long_bf16", "attend", 1, 16, 16, 16384, 16384, 128, "bf16"),
        # a padded batch of causal sequences, three query heads to a key head, no tile divides the length
        _attn("ragged_causal_bf16", "attend", 5, 12, 4, 2039, 2039, 128, "bf16", "bnhd", ragged=True, right=0),
        # serving: a token of each of 24 sequences against its keys and values, four query heads to a key head
        _attn("decode_bf16", "attend", 24, 32, 8, 1, 16384, 128, "bf16", "bnhd", ragged=True, right=0),
        # training: the ViT-S layer's backward pass
        _attn("vit_backward_bf16", "attend_backward", 64, 6, 6, 196, 196, 64, "bf16", "qkv"),
        # training: dense prediction on 128x128 tokens, the benchmark's default shape
        _attn("dense_pred_backward_bf16", "attend_backward", 2, 12, 12, 16384, 16384, 64, "bf16"),
        # fp32 training on padded 33x41 grids as causal sequences with a window, three query heads to a key head
        _attn("ragged_window_backward_f32", "attend_backward", 3, 6, 2, 1353, 1353, 64, "f32", "bnhd", ragged=True,
              left=500, right=0),
        # one image's tokens before a block, fp32: all latency
        _norm("image_norm_f32", "norm", 1, 1, 196, 384, "f32"),
        # the queries of every head before attention, as the projection wrote them
        _norm("head_norm_bf16", "norm", 2, 12, 16384, 64, "bf16", layout="bnhd"),
        # the tokens of eight 64x64 images before a ViT-B block
        _norm("block_norm_backward_bf16", "norm_backward", 1, 1, 32768, 768, "bf16"),
        # a width that no vector divides, weights in the tokens' type
        _norm("odd_norm_backward_bf16", "norm_backward", 1, 1, 4099, 1021, "bf16", wdtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend_backward", "attend_backward", "norm", "norm_backward"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if op in ("norm", "norm_backward"):
        wdtype = "bf16" if dtype == "bf16" and rng.random() < 0.3 else "f32"
        if rng.random() < 0.4:  # queries or keys of every head
            B, H, n = _log_int(rng, 1, 64), rng.choice([1, 2, 3, 6, 8, 12, 16]), _log_int(rng, 1, 16384)
            n = max(1, min(n, (1 << 19) // (B * H)))
            return _norm(None, op, B, H, n, rng.choice([64, 128]), dtype, wdtype, rng.choice(["bhnd", "bnhd", "qkv"]))
        C = _log_int(rng, 33, 8192)
        if rng.random() < 0.7:
            C = (C + 7) // 8 * 8
        return _norm(None, op, 1, 1, max(1, min(_log_int(rng, 1, 65536), 25_000_000 // C)), C, dtype, wdtype)
    d = rng.choice([64, 64, 128])
    H_kv = rng.choice([1, 2, 3, 4, 6, 8, 12, 16])
    H = H_kv * rng.choice([1, 1, 1, 2, 3, 4, 8])
    right = rng.choice([-1, -1, 0])
    layout = rng.choice(["bhnd", "bnhd"])
    ragged = rng.random() < 0.4
    B = _log_int(rng, 1, 48)
    if op == "attend" and rng.random() < 0.35:  # a few new tokens against the keys so far
        N, N_k = rng.choice([1, 1, 1, 2, 5, 16]), _log_int(rng, 100, 60000)
        left = rng.choice([-1, -1, -1, _log_int(rng, 64, 4096)])
        B = max(1, min(B, int(4.0e8 / (H_kv * N_k * d)), int(2.0e11 / (H * N * N_k * d))))
        return _attn(None, op, B, H, H_kv, N, N_k, d, dtype, layout, ragged, ragged and B > 2 and rng.random() < 0.3,
                     left, right)
    N = _log_int(rng, 30, 3000 if dtype == "f32" else 12000)
    N_k = N if rng.random() < 0.8 else _log_int(rng, 30, 3000 if dtype == "f32" else 12000)
    if N_k == N and H == H_kv and rng.random() < 0.3:
        layout = "qkv"
    left = _log_int(rng, 16, 2048) if rng.random() < 0.2 else -1
    most = 1.5e11 if op == "attend" else 7.0e10  # products, below the largest listed cases
    if dtype == "f32":
        most /= 8
    B = max(1, min(B, int(most / (H * N * N_k * d)), int(1.0e8 / (H * max(N, N_k) * d))))
    return _attn(None, op, B, H, H_kv, N, N_k, d, dtype, layout, ragged, ragged and B > 2 and rng.random() < 0.3, left,
                 right)


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _lengths(case):
    """(q_len, k_len) of the batch's sequences, as lists."""
    B, N, N_k = case["B"], case["N"], case["N_k"]
    if not case["ragged"]:
        return [N] * B, [N_k] * B
    k_len = [max(1, N_k - b * N_k * 5 // (8 * B)) for b in range(B)]
    q_len = [min(N, x) if N == N_k else N for x in k_len]
    if case["empty"]:
        k_len[-1] = 0
        q_len[-1] = 0 if N == N_k else N
    return q_len, k_len


def _reach(case):
    """How many keys each query sees, added up."""
    total = 0
    for n, m in zip(*_lengths(case)):
        p = torch.arange(n, dtype=torch.int64) + (m - n)
        lo = torch.clamp(p - case["left"], min=0) if case["left"] >= 0 else torch.zeros_like(p)
        hi = torch.clamp(p + case["right"] + 1, min=0, max=m) if case["right"] >= 0 else torch.full_like(p, m)
        total += int(torch.clamp(hi - lo, min=0).sum())
    return total


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] in ("norm", "norm_backward"):
        rows, C, ew = case["n0"] * case["n1"] * case["n2"], case["C"], 4 if case["wdtype"] == "f32" else 2
        if case["op"] == "norm":  # x, w, b in; y and the statistics out
            return {"bytes": 2 * rows * C * e + 2 * C * ew + 8 * rows, "flops": 8 * rows * C}
        # x, dy, w and the statistics in; dx, dw, db out
        return {"bytes": 3 * rows * C * e + 3 * C * ew + 8 * rows, "flops": 14 * rows * C}
    H, d = case["H"], case["d"]
    q_len, k_len = _lengths(case)
    q = H * sum(q_len) * d * e
    kv = 2 * case["H_kv"] * sum(k_len) * d * e
    full = case["B"] * H * case["N"]
    pairs = H * _reach(case)
    if case["op"] == "attend":
        return {"bytes": q + kv + full * (d * e + 4), "flops": 4 * pairs * d}
    # q, o, dO, k, v and the log-sum-exps in; dq, dk, dv out
    out = full * d * e + 2 * case["B"] * case["H_kv"] * case["N_k"] * d * e
    return {"bytes": 3 * q + kv + 4 * H * sum(q_len) + out, "flops": 10 * pairs * d}


def _heads(g, B, H, N, d, dtype, layout, std):
    """[B, H, N, d] standard normal times std, in the layout's memory order."""
    x = torch.randn((B, N, H, d) if layout == "bnhd" else (B, H, N, d), device="cuda", generator=g).mul_(std).to(dtype)
    return x.transpose(1, 2) if layout == "bnhd" else x


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _dtype(case["dtype"])
    if case["op"] in ("norm", "norm_backward"):
        n0, n1, n2, C = case["n0"], case["n1"], case["n2"], case["C"]

        def rows():
            # tokens of a residual stream: channels with their own mean and spread
            if case["layout"] == "bnhd":
                x = torch.randn((n0, n2, n1, C), device="cuda", generator=g)
            elif case["layout"] == "qkv":
                x = torch.randn((n0, n2, 3, n1, C), device="cuda", generator=g)
            else:
                x = torch.randn((n0, n1, n2, C), device="cuda", generator=g)
            x = (x * (0.5 + torch.rand(C, device="cuda", generator=g)) +
                 0.3 * torch.randn(C, device="cuda", generator=g)).to(dt)
            return x[:, :, 1].transpose(1, 2) if case["layout"] == "qkv" else \
                x.transpose(1, 2) if case["layout"] == "bnhd" else x

        wt = _dtype(case["wdtype"])
        s = dict(x=rows(), w=(1.0 + 0.2 * torch.randn(C, device="cuda", generator=g)).to(wt),
                 b=(0.1 * torch.randn(C, device="cuda", generator=g)).to(wt))
        if case["op"] == "norm_backward":
            s["dy"] = rows()
            x = s["x"].float()
            s["mean"] = x.mean(-1)
            s["rstd"] = torch.rsqrt((x - s["mean"][..., None]).square().mean(-1) + 1e-5)
        return s
    B, H, H_kv, N, N_k, d = (case[x] for x in ("B", "H", "H_kv", "N", "N_k", "d"))
    # scores with a standard deviation of 1.5 before the softmax
    if case["layout"] == "qkv":
        x = torch.randn((B, N, 3, H, d), device="cuda", generator=g)
        x[:, :, 0] *= 1.5
        q, k, v = (x.to(dt)[:, :, i].transpose(1, 2) for i in range(3))
    else:
        q = _heads(g, B, H, N, d, dt, case["layout"], 1.5)
        k, v = (_heads(g, B, H_kv, N_k, d, dt, case["layout"], 1.0) for _ in range(2))
    s = dict(q=q, k=k, v=v, q_len=None, k_len=None)
    if case["ragged"]:
        s["q_len"], s["k_len"] = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in _lengths(case))
    if case["op"] == "attend_backward":
        s["dO"] = _heads(g, B, H, N, d, dt, "bhnd" if case["layout"] == "bhnd" else "bnhd", 1.0)
        s["o"], s["lse"] = _attend(case, s)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        from paper_2602_01219_amd import mita
        if case["op"] in ("norm", "norm_backward"):
            s["cfg"] = mita.NormConfig(rows=(case["n0"], case["n1"], case["n2"]), C=case["C"], dtype=case["dtype"],
                                       wdtype=case["wdtype"])
            need = mita.norm_workspace_size(s["cfg"]) if case["op"] == "norm_backward" else 0
        else:
            s["cfg"] = mita.DenseConfig(B=case["B"], H=case["H"], H_kv=case["H_kv"], N=case["N"], N_k=case["N_k"],
                                        d=case["d"], dtype=case["dtype"], left=case["left"], right=case["right"])
            need = mita.dense_workspace_size(s["cfg"], mita.WS_FORWARD if case["op"] == "attend" else mita.WS_BACKWARD)
        s["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    return s


def _visible(case, n, m):
    """[N, N_k] truth values for a sequence of n queries and m keys."""
    i = torch.arange(case["N"], device="cuda")[:, None]
    j = torch.arange(case["N_k"], device="cuda")[None, :]
    p = i + (m - n)
    ok = (i < n) & (j < m)
    if case["left"] >= 0:
        ok = ok & (j >= p - case["left"])
    if case["right"] >= 0:
        ok = ok & (j <= p + case["right"])
    return ok


def _chunks(case, at_most=1 << 29):
    """Pieces of the batch and its query heads whose score matrices stay within memory: (b0, b1, h0, h1), whole
    groups of heads."""
    B, H, G = case["B"], case["H"], case["H"] // case["H_kv"]
    one = case["N"] * case["N_k"]
    alike = not case["ragged"]
    if alike and one * H <= at_most:
        nb = max(1, at_most // (one * H))
        return [(b, min(B, b + nb), 0, H) for b in range(0, B, nb)]
    nh = max(1, at_most // (one * G)) * G
    return [(b, b + 1, h, min(H, h + nh)) for b in range(B) for h in range(0, H, nh)]


def _scores(case, s, b0, b1, h0, h1):
    """(q, k, v) in 32 bits, k and v repeated for their query heads, and the masked scores."""
    G = case["H"] // case["H_kv"]
    q = s["q"][b0:b1, h0:h1].float()
    k, v = (s[x][b0:b1, h0 // G:h1 // G].float().repeat_interleave(G, 1) for x in ("k", "v"))
    z = torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(case["d"])
    mask = None
    if case["ragged"] or case["left"] >= 0 or case["right"] >= 0:
        q_len, k_len = _lengths(case)
        mask = _visible(case, q_len[b0], k_len[b0])
        z = z.masked_fill(~mask, -math.inf)
    return q, k, v, z


def _attend(case, s):
    B, H, N, d = case["B"], case["H"], case["N"], case["d"]
    o = torch.empty((B, H, N, d), dtype=s["q"].dtype, device="cuda")
    lse = torch.empty((B, H, N), device="cuda")
    for b0, b1, h0, h1 in _chunks(case):
        _, _, v, z = _scores(case, s, b0, b1, h0, h1)
        m = z.amax(-1, keepdim=True)
        m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
        e = torch.exp(z - m)
        total = e.sum(-1, keepdim=True)
        o[b0:b1, h0:h1] = torch.matmul(e, v) / torch.where(total > 0, total, torch.ones_like(total))
        lse[b0:b1, h0:h1] = (m + torch.log(total))[..., 0]
    return o, lse


def _attend_backward(case, s):
    B, H, H_kv, N, N_k, d = (case[x] for x in ("B", "H", "H_kv", "N", "N_k", "d"))
    G = H // H_kv
    dq = torch.empty((B, H, N, d), dtype=s["q"].dtype, device="cuda")
    dk, dv = (torch.empty((B, H_kv, N_k, d), dtype=s["q"].dtype, device="cuda") for _ in range(2))
    for b0, b1, h0, h1 in _chunks(case):
        q, k, v, z = _scores(case, s, b0, b1, h0, h1)
        lse, dO = s["lse"][b0:b1, h0:h1, :, None], s["dO"][b0:b1, h0:h1].float()
        p = torch.exp(z - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse))
        D = (dO * s["o"][b0:b1, h0:h1].float()).sum(-1, keepdim=True)
        ds = p * (torch.matmul(dO, v.transpose(-1, -2)) - D) / math.sqrt(d)
        dq[b0:b1, h0:h1] = torch.matmul(ds, k)
        gk, gv = torch.matmul(ds.transpose(-1, -2), q), torch.matmul(p.transpose(-1, -2), dO)
        dk[b0:b1, h0 // G:h1 // G] = gk.unflatten(1, (-1, G)).sum(2)
        dv[b0:b1, h0 // G:h1 // G] = gv.unflatten(1, (-1, G)).sum(2)
    return dq, dk, dv


def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        from paper_2602_01219_amd import mita
        cfg = state["cfg"]
        if op == "attend":
            return mita.dense_forward(cfg, state["q"], state["k"], state["v"], q_len=state["q_len"],
                                      k_len=state["k_len"], ws=state["ws"])
        if op == "attend_backward":
            return mita.dense_backward(cfg, state["q"], state["k"], state["v"], state["o"], state["lse"], state["dO"],
                                       q_len=state["q_len"], k_len=state["k_len"], ws=state["ws"])
        if op == "norm":
            return mita.norm_forward(cfg, state["x"], state["w"], state["b"])
        return mita.norm_backward(cfg, state["x"], state["mean"], state["rstd"], state["dy"], state["w"],
                                  ws=state["ws"])
    if op == "attend":
        return _attend(case, state)
    if op == "attend_backward":
        return _attend_backward(case, state)
    x, w = state["x"].float(), state["w"].float()
    if op == "norm":
        mean = x.mean(-1)
        c = x - mean[..., None]
        rstd = torch.rsqrt((c * c).mean(-1) + 1e-5)
        return (c * rstd[..., None] * w + state["b"].float()).to(state["x"].dtype), mean, rstd
    dy, mean, rstd = state["dy"].float(), state["mean"][..., None], state["rstd"][..., None]
    h = (x - mean) * rstd
    g = dy * w
    dx = rstd * (g - g.mean(-1, keepdim=True) - h * (g * h).mean(-1, keepdim=True))
    wt = state["w"].dtype
    return dx.to(state["x"].dtype), (dy * h).sum((0, 1, 2)).to(wt), dy.sum((0, 1, 2)).to(wt)


def exact(case, seed):
    """The definitions in 64 bits, one sequence and head at a time, only the keys and queries that exist."""
    s = _inputs(case, seed)
    f64 = torch.float64
    if case["op"] in ("norm", "norm_backward"):
        C = case["C"]
        x, w, b = (s[t].to(f64) for t in ("x", "w", "b"))
        if case["op"] == "norm":
            mean = x.sum(-1) / C
            var = ((x - mean.unsqueeze(-1)) ** 2).sum(-1) / C
            return w * (x - mean.unsqueeze(-1)) / (var + 1e-5).sqrt().unsqueeze(-1) + b, mean, 1 / (var + 1e-5).sqrt()
        dy, mean, rstd = s["dy"].to(f64), s["mean"].to(f64).unsqueeze(-1), s["rstd"].to(f64).unsqueeze(-1)
        h = (x - mean) * rstd
        gw = dy * w
        along = (gw * h).sum(-1, keepdim=True) / C
        dx = (gw - gw.sum(-1, keepdim=True) / C - along * h) * rstd
        return dx, (dy * h).reshape(-1, C).sum(0), dy.reshape(-1, C).sum(0)
    B, H, H_kv, N, N_k, d = (case[t] for t in ("B", "H", "H_kv", "N", "N_k", "d"))
    G, left, right = H // H_kv, case["left"], case["right"]
    back = case["op"] == "attend_backward"
    o = torch.zeros((B, H, N, d), dtype=f64, device="cuda")  # o, or dq
    lse = torch.full((B, H, N), -math.inf, dtype=f64, device="cuda")
    dk, dv = (torch.zeros((B, H_kv, N_k, d), dtype=f64, device="cuda") for _ in range(2)) if back else (None, None)
    for b, (n, m) in enumerate(zip(*_lengths(case))):
        if n == 0 or m == 0:
            continue
        ahead = torch.arange(m, device="cuda")[None] - (torch.arange(n, device="cuda")[:, None] + m - n)
        hidden = torch.zeros((n, m), dtype=torch.bool, device="cuda")
        if left >= 0:
            hidden |= ahead < -left
        if right >= 0:
            hidden |= ahead > right
        some = ~hidden.all(1)
        for h in range(H):
            q = s["q"][b, h, :n].to(f64)
            k, v = s["k"][b, h // G, :m].to(f64), s["v"][b, h // G, :m].to(f64)
            z = (q @ k.T) * d ** -0.5
            z[hidden] = -math.inf
            if not back:
                t = torch.logsumexp(z, 1)
                lse[b, h, :n] = t
                z = torch.exp(z - torch.where(some, t, torch.zeros_like(t))[:, None])
                o[b, h, :n] = z @ v
                continue
            t = s["lse"][b, h, :n].to(f64)
            z = torch.exp(z - torch.where(some, t, torch.zeros_like(t))[:, None])
            dO = s["dO"][b, h, :n].to(f64)
            dv[b, h // G, :m] += z.T @ dO
            r = dO @ v.T
            r -= (dO * s["o"][b, h, :n].to(f64)).sum(1)[:, None]
            r *= z
            r *= d ** -0.5
            o[b, h, :n] = r @ k
            dk[b, h // G, :m] += r.T @ q
    return (o, dk, dv) if back else (o, lse)

"""Performance cases of the operators that stand around attention in a decoder
layer: the root-mean-square norm that adds the residual (forward, also with an
output in 8 bits and its scales, and backward), rotary positions of queries and
keys (forward and backward), and attention of a batch whose sequences share a
prefix.

A case is one call that a program makes, on device tensors it already holds:

  op "rms"            y, its scales (8 bits), the sum h = x + res (with a residual), 1 / root mean square
  op "rms_backward"   the gradient of x (and of the residual) and the weight's
  op "rope"           the rotated queries and keys
  op "rope_backward"  the queries' and keys' gradients from the rotated ones'
  op "prefix"         o and the rows' log-sum-exps

An 8-bit output is returned as a tensor of 8-bit floating-point numbers, which
holds the values in units of the scales that are returned beside it.

Layouts: "bhnd" contiguous heads, "bnhd" the [B, N, H, d] that a projection
writes, seen as [B, H, N, d], "qkv" the slices of one fused projection
[B, N, 3, H, d]. With "ragged" every sequence (and prefix) has its own length
(the last sequence no keys of its own with "empty").

With own = False, run() uses elementary torch operations in 32 bits (angles of
positions in 64); exact() follows the definitions in 64 bits and shares nothing
with them but the inputs.
"""
import math

import torch

own = False


def _rms(name, op, rows, C, dtype, wdtype="f32", res=True, out="same", group=0):
    """group: elements that share a scale (0: the row)."""
    c = dict(op=op, rows=rows, C=C, dtype=dtype, wdtype=wdtype, res=res, out=out, group=group)
    if name:
        c["name"] = name
    return c


def _rope(name, op, B, H, H_kv, N, d, dtype, rot=0, layout="bnhd", interleaved=False, scaling="none", pos="count"):
    """pos: "count" from 0, "offset" the same first position for all, "own" each sequence's own positions."""
    c = dict(op=op, B=B, H=H, H_kv=H_kv, N=N, d=d, dtype=dtype, rot=rot or d, layout=layout, interleaved=interleaved,
             scaling=scaling, pos=pos)
    if name:
        c["name"] = name
    return c


def _prefix(name, Bp, S, H, H_kv, N, P, N_k, d, dtype, layout="bnhd", ragged=True, empty=False, left=-1, right=0):
    """Bp prefixes of up to P tokens, each shared by S sequences of up to N_k keys of their own."""
    c = dict(op="prefix", Bp=Bp, S=S, H=H, H_kv=H_kv, N=N, P=P, N_k=N_k, d=d, dtype=dtype, layout=layout,
             ragged=ragged, empty=empty, left=left, right=right)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # serving: the new tokens of 24 sequences before a layer, all latency
        _rms("token_rms_bf16", "rms", 24, 768, "bf16"),
        # a prompt's tokens before a projection whose product takes 8 bits, a scale for each 128 columns
        _rms("prompt_rms_e4m3", "rms", 16384, 4096, "bf16", out="e4m3", group=128),
        # a width that no vector divides, no residual, 8 bits with one scale per row
        _rms("odd_rms_e4m3", "rms", 4099, 1021, "bf16", wdtype="bf16", res=False, out="e4m3"),
        # training: the tokens of eight 64x64 images, with the gradient that comes along the residual
        _rms("block_rms_backward_bf16", "rms_backward", 32768, 768, "bf16"),
        # serving: the new token of 24 sequences, each at its own far position, four query heads to a key head
        _rope("token_rope_bf16", "rope", 24, 32, 8, 1, 128, "bf16", pos="own"),
        # a batch of images through a ViT-S layer, straight from its fused projection
        _rope("vit_rope_bf16", "rope", 64, 6, 6, 196, 64, "bf16", layout="qkv"),
        # a long prompt beyond the trained length, pairs side by side
        _rope("long_rope_bf16", "rope", 1, 32, 8, 32768, 128, "bf16", interleaved=True, scaling="parts"),
        # fp32 training, half of each head rotated, an odd length
        _rope("part_rope_backward_f32", "rope_backward", 3, 12, 4, 4099, 64, "f32", rot=32, layout="bhnd", pos="offset"),
        # one token of four samples that continue the 196 tokens of one image, fp32: the smallest call, all latency
        _prefix("pool_prefix_f32", 1, 4, 6, 6, 1, 196, 16, 64, "f32", "bhnd", ragged=False, right=-1),
        # serving: a token of each of 32 conversations that begin with the same 32768 tokens
        _prefix("decode_prefix_bf16", 1, 32, 32, 8, 1, 32768, 1024, 128, "bf16"),
        # twelve samples for each of four prompts, as many key heads as query heads
        _prefix("samples_prefix_bf16", 4, 12, 12, 12, 1, 5000, 300, 64, "bf16"),
        # eight padded questions about one document, three query heads to a key head, no tile divides a length
        _prefix("prompt_prefix_bf16", 1, 8, 12, 4, 515, 8003, 515, 128, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rms", "rms", "rms_backward", "rope", "rope", "rope_backward", "prefix", "prefix", "prefix", "prefix"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if op in ("rms", "rms_backward"):
        C = _log_int(rng, 33, 8192)
        if rng.random() < 0.7:
            C = (C + 7) // 8 * 8
        out, group = rng.choice([("same", 0), ("e4m3", 0), ("e4m3", 128)]) if op == "rms" else ("same", 0)
        wdtype = "bf16" if dtype == "bf16" and rng.random() < 0.3 else "f32"
        rows = max(1, min(_log_int(rng, 1, 65536), 25_000_000 // C))
        return _rms(None, op, rows, C, dtype, wdtype, rng.random() < 0.7, out, group)
    H_kv = rng.choice([1, 2, 3, 4, 6, 8, 12, 16])
    H = H_kv * rng.choice([1, 1, 1, 2, 3, 4, 8])
    if op in ("rope", "rope_backward"):
        d = rng.choice([64, 64, 80, 128, 128, 256])
        rot = rng.choice([d, d, d, d // 2, d // 4 // 2 * 2, 2 * rng.randint(1, d // 2)])
        layout = rng.choice(["bhnd", "bnhd", "bnhd"] + (["qkv"] if H == H_kv else []))
        N = rng.choice([1, _log_int(rng, 2, 32768), _log_int(rng, 2, 32768)])
        B = max(1, min(_log_int(rng, 1, 256 if N == 1 else 64), 60_000_000 // ((H + H_kv) * N * d)))
        N = max(1, min(N, 60_000_000 // ((H + H_kv) * d)))
        return _rope(None, op, B, H, H_kv, N, d, dtype, rot, layout, rng.random() < 0.5,
                     rng.choice(["none", "linear", "base", "parts"]), rng.choice(["count", "offset", "own"]))
    d = rng.choice([64, 128, 128])
    Bp, S = rng.choice([1, 1, 1, 2, 3, 5]), _log_int(rng, 1, 64)
    P = _log_int(rng, 100, 60000)
    if rng.random() < 0.65:  # a few new tokens
        N, N_k = rng.choice([1, 1, 1, 2, 5]), _log_int(rng, 5, 2000)
    else:  # a prompt behind the prefix
        N = _log_int(rng, 30, 1000)
        N_k = N if rng.random() < 0.8 else _log_int(rng, 30, 1000)
        P = min(P, 16000)
    most = 5.0e9 if dtype == "f32" else 3.5e10  # products, below the largest listed case
    P = max(100, min(P, int(5.0e7 / (Bp * H_kv * d)), int(most / (Bp * H * N * d))))
    S = max(1, min(S, int(most / (Bp * H * N * (P + N_k) * d)), int(2.0e8 / (Bp * H * N * (P + N_k))),
                   int(5.0e7 / (Bp * H_kv * N_k * d))))
    return _prefix(None, Bp, S, H, H_kv, N, P, N_k, d, dtype, rng.choice(["bhnd", "bnhd"]), rng.random() < 0.6,
                   rng.random() < 0.2, rng.choice([-1, -1, -1, _log_int(rng, 64, 8192)]), rng.choice([0, 0, -1]))


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _groups(case):
    return math.ceil(case["C"] / (case["group"] or case["C"]))


def _lengths(case):
    """(q_len and k_len of the sequences, p_len of the prefixes), as lists."""
    B, Bp, N, P, N_k = case["Bp"] * case["S"], case["Bp"], case["N"], case["P"], case["N_k"]
    k_len, p_len = [N_k] * B, [P] * Bp
    if case["ragged"]:
        k_len = [max(1, N_k - (b * 7 % B) * N_k * 5 // (8 * B)) for b in range(B)]
        p_len = [max(1, P - j * P * 3 // (8 * Bp)) for j in range(Bp)]
    if case["empty"]:
        k_len[-1] = 0
    q_len = [min(N, max(x, 1)) if N == N_k else N for x in k_len]
    return q_len, k_len, p_len


def _reach(case):
    """How many keys each query sees, added up."""
    q_len, k_len, p_len = _lengths(case)
    total = 0
    for b, (n, m) in enumerate(zip(q_len, k_len)):
        m += p_len[b // case["S"]]
        p = torch.arange(n, dtype=torch.int64) + (m - n)
        lo = torch.clamp(p - case["left"], min=0) if case["left"] >= 0 else torch.zeros_like(p)
        hi = torch.clamp(p + case["right"] + 1, min=0, max=m) if case["right"] >= 0 else torch.full_like(p, m)
        total += int(torch.clamp(hi - lo, min=0).sum())
    return total


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] in ("rms", "rms_backward"):
        rows, C, ew = case["rows"], case["C"], 4 if case["wdtype"] == "f32" else 2
        if case["op"] == "rms":  # x, residual, w in; y, scales, h, statistics out
            y = rows * C * e if case["out"] == "same" else rows * (C + 4 * _groups(case))
            return {"bytes": rows * C * e * (3 if case["res"] else 1) + y + C * ew + 4 * rows, "flops": 6 * rows * C}
        # h, dy, dh, w, statistics in; dx, dw out
        return {"bytes": rows * C * e * (4 if case["res"] else 3) + 2 * C * ew + 4 * rows, "flops": 9 * rows * C}
    if case["op"] in ("rope", "rope_backward"):
        tokens, H = case["B"] * case["N"], case["H"] + case["H_kv"]
        return {"bytes": 2 * tokens * H * case["d"] * e + (4 * tokens if case["pos"] == "own" else 0),
                "flops": 3 * tokens * H * case["rot"]}
    q_len, k_len, p_len = _lengths(case)
    H, d = case["H"], case["d"]
    kv = 2 * case["H_kv"] * (sum(k_len) + sum(p_len)) * d * e
    full = case["Bp"] * case["S"] * H * case["N"]
    return {"bytes": H * sum(q_len) * d * e + kv + full * (d * e + 4), "flops": 4 * H * _reach(case) * d}


def _heads(g, B, H, N, d, dtype, layout, std=1.0):
    """[B, H, N, d] standard normal times std, in the layout's memory order."""
    x = torch.randn((B, N, H, d) if layout == "bnhd" else (B, H, N, d), device="cuda", generator=g).mul_(std).to(dtype)
    return x.transpose(1, 2) if layout == "bnhd" else x


def _positions(case, g):
    """(positions [B, N] int32 or None, the first token's position): places in contexts of up to a million tokens."""
    B, N = case["B"], case["N"]
    if case["pos"] == "own":
        first = torch.randint(0, 1 << 20, (B, 1), device="cuda", generator=g, dtype=torch.int32)
        return first + torch.arange(N, device="cuda", dtype=torch.int32), 0
    return None, 0 if case["pos"] == "count" else 65521


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _dtype(case["dtype"])
    if case["op"] in ("rms", "rms_backward"):
        rows, C = case["rows"], case["C"]

        def tokens(std):
            # tokens of a residual stream: channels with their own spread, some of them large
            x = torch.randn((rows, C), device="cuda", generator=g)
            return (x * std * torch.exp(0.5 * torch.randn(C, device="cuda", generator=g))).to(dt)

        s = dict(w=(1.0 + 0.2 * torch.randn(C, device="cuda", generator=g)).to(_dtype(case["wdtype"])))
        if case["op"] == "rms":
            s["x"], s["res"] = tokens(0.5), tokens(1.5) if case["res"] else None
        else:
            s["h"], s["dy"], s["dh"] = tokens(1.5), tokens(1.0), tokens(1.0) if case["res"] else None
            s["rstd"] = torch.rsqrt(s["h"].float().square().mean(-1) + 1e-5)
        return s
    if case["op"] in ("rope", "rope_backward"):
        B, H, H_kv, N, d = (case[x] for x in ("B", "H", "H_kv", "N", "d"))
        if case["layout"] == "qkv":
            x = torch.randn((B, N, 3, H, d), device="cuda", generator=g).to(dt)
            q, k = (x[:, :, i].transpose(1, 2) for i in range(2))
        else:
            q, k = (_heads(g, B, h, N, d, dt, case["layout"]) for h in (H, H_kv))
        s = dict(q=q, k=k)
        s["pos"], s["first"] = _positions(case, g)
        return s
    Bp, H, H_kv, N, P, N_k, d = (case[x] for x in ("Bp", "H", "H_kv", "N", "P", "N_k", "d"))
    B = Bp * case["S"]
    # scores with a standard deviation of 1.5 before the softmax
    s = dict(q=_heads(g, B, H, N, d, dt, case["layout"], 1.5), q_len=None, k_len=None, p_len=None)
    s["kp"], s["vp"] = (_heads(g, Bp, H_kv, P, d, dt, case["layout"]) for _ in range(2))
    s["k"], s["v"] = (_heads(g, B, H_kv, N_k, d, dt, case["layout"]) for _ in range(2))
    if case["ragged"] or case["empty"]:
        s["q_len"], s["k_len"], s["p_len"] = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in _lengths(case))
    return s


# How positions beyond the trained ones are met: factor, positions of training, turns over these of pairs that are
# stretched whole (at most slow) and not at all (at least fast), and the size that rotated elements get
SCALED = dict(factor=8.0, trained=4096, slow=1.0, fast=32.0, scale=1.2)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        from paper_2602_01219_amd import mita
        if case["op"] in ("rms", "rms_backward"):
            s["cfg"] = mita.RmsConfig(rows=(case["rows"],), C=case["C"], dtype=case["dtype"], wdtype=case["wdtype"],
                                      out=case["out"], group=case["group"])
            need = mita.rms_workspace_size(s["cfg"]) if case["op"] == "rms_backward" else 0
        elif case["op"] in ("rope", "rope_backward"):
            more = {} if case["scaling"] == "none" else dict(factor=SCALED["factor"])
            if case["scaling"] == "parts":
                more = SCALED
            s["cfg"] = mita.RopeConfig(B=case["B"], H=case["H"], H_kv=case["H_kv"], N=case["N"], d=case["d"],
                                       rot=case["rot"], dtype=case["dtype"], interleaved=case["interleaved"],
                                       scaling=case["scaling"], first=s["first"], **more)
            need = 0
        else:
            s["cfg"] = mita.PrefixConfig(B=case["Bp"] * case["S"], H=case["H"], H_kv=case["H_kv"], N=case["N"],
                                         Bp=case["Bp"], P=case["P"], N_k=case["N_k"], d=case["d"],
                                         dtype=case["dtype"], left=case["left"], right=case["right"])
            need = mita.prefix_workspace_size(s["cfg"])
        s["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    return s


def run(state):
    op = state["case"]["op"]
    if own:
        from paper_2602_01219_amd import mita
        cfg = state["cfg"]
        if op == "rms":
            return mita.rms_forward(cfg, state["x"], w=state["w"], res=state["res"])
        if op == "rms_backward":
            return mita.rms_backward(cfg, state["h"], state["rstd"], state["dy"], w=state["w"], dh=state["dh"],
                                     ws=state["ws"])
        if op == "rope":
            return mita.rope_forward(cfg, state["q"], state["k"], pos=state["pos"])
        if op == "rope_backward":
            return mita.rope_backward(cfg, state["q"], state["k"], pos=state["pos"])
        return mita.prefix_forward(cfg, state["q"], state["kp"], state["vp"], state["k"], state["v"],
                                   q_len=state["q_len"], p_len=state["p_len"], k_len=state["k_len"], ws=state["ws"])
    if op == "rms":
        return _rms_forward(state["case"], state)
    if op == "rms_backward":
        return _rms_backward(state)
    if op == "prefix":
        return _attend(state["case"], state)
    return _rotate(state["case"], state)


def _rms_forward(case, s):
    x = s["x"].float()
    h = x + s["res"].float() if case["res"] else x
    rstd = torch.rsqrt((h * h).mean(-1) + 1e-5)
    y = h * rstd[:, None] * s["w"].float()
    scales = None
    if case["out"] == "e4m3":
        n, g = _groups(case), case["group"] or case["C"]
        full = torch.zeros((case["rows"], n * g), device="cuda")
        full[:, :case["C"]] = y
        full = full.view(case["rows"], n, g)
        scales = torch.clamp(full.abs().amax(-1), min=2.0 ** -117) / 448.0
        y = (full / scales[..., None]).view(case["rows"], n * g)[:, :case["C"]].to(torch.float8_e4m3fn)
    else:
        y = y.to(s["x"].dtype)
    return y, scales, h.to(s["x"].dtype) if case["res"] else None, rstd


def _rms_backward(s):
    w, dy, rstd = s["w"].float(), s["dy"].float(), s["rstd"][:, None]
    u = s["h"].float() * rstd
    g = dy * w
    dx = rstd * (g - u * (g * u).mean(-1, keepdim=True))
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return dx.to(s["h"].dtype), (dy * u).sum(0).to(s["w"].dtype)


def _frequencies(case):
    """(radians per position of each pair, in 64 bits, and what the rotated elements are multiplied by)."""
    rot, factor, base = case["rot"], SCALED["factor"], 10000.0
    if case["scaling"] == "base" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    f = base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "parts":
        turns = SCALED["trained"] * f / (2 * math.pi)
        keep = torch.clamp((turns - SCALED["slow"]) / (SCALED["fast"] - SCALED["slow"]), 0, 1)
        f = keep * f + (1 - keep) * f / factor
    return f, SCALED["scale"] if case["scaling"] == "parts" else 1.0


def _rotate(case, s):
    rot = case["rot"]
    f, size = _frequencies(case)
    pos = s["pos"]
    if pos is None:
        pos = (s["first"] + torch.arange(case["N"], device="cuda"))[None]
    angle = (pos.double()[..., None] * f)[:, None]  # [B or 1, 1, N, rot / 2]
    cos, sin = (size * torch.cos(angle)).float(), (size * torch.sin(angle)).float()
    if case["op"] == "rope_backward":
        sin = -sin

    def one(x):
        y = x.float()
        if case["interleaved"]:
            a, b = y[..., :rot:2], y[..., 1:rot:2]
            turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
        else:
            a, b = y[..., :rot // 2], y[..., rot // 2:rot]
            turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
        return torch.cat((turned, y[..., rot:]), -1).to(x.dtype)

    return one(s["q"]), one(s["k"])


def _attend(case, s):
    Bp, S, H, H_kv, N, P, N_k, d = (case[x] for x in ("Bp", "S", "H", "H_kv", "N", "P", "N_k", "d"))
    G = H // H_kv
    q_len, k_len, p_len = (torch.tensor(x, device="cuda") for x in _lengths(case))
    i = torch.arange(N, device="cuda")
    ends = p_len.repeat_interleave(S)  # of the prefix, for each sequence
    place = (ends + k_len - q_len)[:, None] + i  # [B, N]
    there = i < q_len[:, None]

    def hidden(j, exists):
        """Truth values [B, 1, N, keys]: keys at places j [B or 1, keys] that a query does not see."""
        ok = there[..., None] & exists[:, None]
        if case["left"] >= 0:
            ok = ok & (j[:, None] >= (place - case["left"])[..., None])
        if case["right"] >= 0:
            ok = ok & (j[:, None] <= (place + case["right"])[..., None])
        return ~ok[:, None]

    q = s["q"].float() / math.sqrt(d)
    rows = q.view(Bp, S, H_kv, G, N, d).transpose(1, 2).reshape(Bp, H_kv, S * G * N, d)  # those of one prefix

    def spread(x):
        return x.view(Bp, H_kv, S, G, N, -1).transpose(1, 2).reshape(Bp * S, H, N, -1)

    j = torch.arange(P, device="cuda")[None]
    zp = spread(torch.matmul(rows, s["kp"].float().transpose(-1, -2)))
    zp = zp.masked_fill(hidden(j, j < ends[:, None]), -math.inf)
    j = torch.arange(N_k, device="cuda")[None]
    z = torch.matmul(q.reshape(Bp * S, H_kv, G * N, d), s["k"].float().transpose(-1, -2)).view(Bp * S, H, N, N_k)
    z = z.masked_fill(hidden(ends[:, None] + j, j < k_len[:, None]), -math.inf)
    m = torch.maximum(zp.amax(-1, keepdim=True), z.amax(-1, keepdim=True))
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    ep, e = torch.exp(zp - m), torch.exp(z - m)
    total = ep.sum(-1, keepdim=True) + e.sum(-1, keepdim=True)
    lse = (m + torch.log(total))[..., 0]
    total = torch.where(total > 0, total, torch.ones_like(total))
    ep = ep.view(Bp, S, H_kv, G, N, P).transpose(1, 2).reshape(Bp, H_kv, S * G * N, P)
    o = spread(torch.matmul(ep, s["vp"].float()))
    o = o + torch.matmul(e.view(Bp * S, H_kv, G * N, N_k), s["v"].float()).view(Bp * S, H, N, d)
    return (o / total).to(s["q"].dtype), lse


def exact(case, seed):
    """The definitions in 64 bits: rows whole, pairs as complex numbers, each sequence's keys in one piece."""
    s = _inputs(case, seed)
    f64 = torch.float64
    if case["op"] == "rms":
        h = s["x"].to(f64)
        if case["res"]:
            h = h + s["res"].to(f64)
        root = (h.pow(2).sum(1) / case["C"] + 1e-5).sqrt()
        y, scales = (h / root.unsqueeze(1)) * s["w"].to(f64), None
        if case["out"] == "e4m3":
            parts = y.split(case["group"] or case["C"], dim=1)
            units = [p.abs().max(dim=1).values.clamp(min=2.0 ** -117) / 448 for p in parts]
            y, scales = torch.cat([p / u.unsqueeze(1) for p, u in zip(parts, units)], 1), torch.stack(units, 1)
        return y, scales, h if case["res"] else None, 1 / root
    if case["op"] == "rms_backward":
        u, dy = s["h"].to(f64) * s["rstd"].to(f64).unsqueeze(1), s["dy"].to(f64)
        gw = dy * s["w"].to(f64)
        along = (gw * u).sum(1, keepdim=True) / case["C"]
        dx = (gw - along * u) * s["rstd"].to(f64).unsqueeze(1)
        return dx + s["dh"].to(f64) if case["res"] else dx, (dy * u).sum(0)
    if case["op"] in ("rope", "rope_backward"):
        rot, names = case["rot"], dict(none=1.0, linear=1.0, base=1.0, parts=SCALED["scale"])
        base = 10000.0
        if case["scaling"] == "base" and rot > 2:
            base *= SCALED["factor"] ** (rot / (rot - 2.0))
        rates = []
        for i in range(rot // 2):
            r = math.exp(-2.0 * i / rot * math.log(base))
            if case["scaling"] == "linear":
                r /= SCALED["factor"]
            if case["scaling"] == "parts":
                t = (SCALED["trained"] * r / math.tau - SCALED["slow"]) / (SCALED["fast"] - SCALED["slow"])
                t = min(1.0, max(0.0, t))
                r *= t + (1.0 - t) / SCALED["factor"]
            rates.append(r)
        p = torch.arange(case["N"], device="cuda", dtype=f64) + s["first"] if s["pos"] is None else s["pos"].to(f64)
        angle = p.unsqueeze(-1) * torch.tensor(rates, dtype=f64, device="cuda")
        unit = torch.polar(torch.full_like(angle, names[case["scaling"]]), angle)
        if case["op"] == "rope_backward":
            unit = unit.conj()
        if unit.dim() == 3:
            unit = unit.unsqueeze(1)
        both = []
        for x in (s["q"].to(f64), s["k"].to(f64)):
            if case["interleaved"]:
                z = torch.complex(x[..., 0:rot:2], x[..., 1:rot:2]) * unit
                x[..., 0:rot:2], x[..., 1:rot:2] = z.real, z.imag
            else:
                z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * unit
                x[..., :rot // 2], x[..., rot // 2:rot] = z.real, z.imag
            both.append(x)
        return tuple(both)
    S, H, H_kv, N, d, left, right = (case[t] for t in ("S", "H", "H_kv", "N", "d", "left", "right"))
    G, B = H // H_kv, case["Bp"] * S
    o = torch.zeros((B, H, N, d), dtype=f64, device="cuda")
    lse = torch.full((B, H, N), -math.inf, dtype=f64, device="cuda")
    q_len, k_len, p_len = _lengths(case)
    for b in range(B):
        n, pl, m = q_len[b], p_len[b // S], k_len[b] + p_len[b // S]
        ahead = torch.arange(m, device="cuda")[None] - (torch.arange(n, device="cuda")[:, None] + m - n)
        blind = torch.zeros((n, m), dtype=torch.bool, device="cuda")
        if left >= 0:
            blind |= ahead < -left
        if right >= 0:
            blind |= ahead > right
        some = ~blind.all(1)
        for h in range(H_kv):
            k, v = (torch.cat((s[x][b // S, h, :pl], s[y][b, h, :m - pl])).to(f64) for x, y in (("kp", "k"), ("vp", "v")))
            z = (s["q"][b, h * G:(h + 1) * G, :n].to(f64) @ k.T) * d ** -0.5
            z[:, blind] = -math.inf
            t = torch.logsumexp(z, 2)
            lse[b, h * G:(h + 1) * G, :n] = t
            z = torch.exp(z - torch.where(some, t, torch.zeros_like(t)).unsqueeze(2))
            o[b, h * G:(h + 1) * G, :n] = z @ v
    return o, lse

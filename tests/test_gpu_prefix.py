"""Attention over shared prefixes on the GPU against the float64 reference of the dense
attention (tests/dense_reference.py) over each sequence's prefix and own keys in one
tensor, with its bounds: the parts' join adds a weight's rounding and a product per
part, which its sum over n keys' n u covers."""
from __future__ import annotations

import pytest
import torch

from paper_2602_01219_amd import mita
from tests.dense_reference import reference, worst
from tests.gpu_helpers import log
from tests.prefix_cases import CASES
from tests.test_gpu_dense import gen, heads, lens, poison, workspace

pytestmark = pytest.mark.gpu


def whole_keys(cfg, p, x, p_len, k_len):
    """[B, H_kv, P + N_k, d]: each sequence's prefix and own keys one behind the other, NaN behind."""
    B, Hk, _, d = cfg.k_shape
    out = torch.full((B, Hk, cfg.P + cfg.N_k, d), float("nan"), dtype=cfg.torch_dtype, device="cuda")
    for b in range(B):
        n, m = p_len[b // (B // cfg.Bp)], k_len[b]
        out[b, :, :n] = p[b // (B // cfg.Bp), :, :n]
        if m:
            out[b, :, n:n + m] = x[b, :, :m]
    return out


def lengths(cfg, p_len, k_len):
    return p_len or [cfg.P] * cfg.Bp, k_len or [cfg.N_k] * cfg.B


def make(cfg, layout, seed, std=1.5):
    g = gen(seed)
    B, H, N, d = cfg.q_shape
    Hk, dt = cfg.p_shape[1], cfg.torch_dtype
    q = heads(g, B, H, N, d, dt, layout, std)
    kp, vp = (heads(g, cfg.Bp, Hk, cfg.P, d, dt, layout) for _ in range(2))
    k, v = (heads(g, B, Hk, cfg.N_k, d, dt, layout) if cfg.N_k else None for _ in range(2))
    return q, kp, vp, k, v


def expected(cfg, t, q_len, p_len, k_len):
    q, kp, vp, k, v = t
    pl, kl = lengths(cfg, p_len, k_len)
    S = cfg.B // cfg.Bp
    dense = mita.DenseConfig(cfg.B, cfg.H, cfg.N, cfg.d, H_kv=cfg.H_kv, N_k=cfg.P + cfg.N_k, dtype=cfg.dtype,
                             left=cfg.left, right=cfg.right, scale=cfg.scale)
    return reference(dense, q, whole_keys(cfg, kp, k, pl, kl), whole_keys(cfg, vp, v, pl, kl), q_len,
                     [pl[b // S] + kl[b] for b in range(cfg.B)])


def run_case(cfg, layout="bhnd", q_len=None, p_len=None, k_len=None, std=1.5, seed=1):
    t = make(cfg, layout, seed, std)
    q, kp, vp, k, v = t
    poison(q, q_len), poison(kp, p_len), poison(vp, p_len)
    if cfg.N_k:
        poison(k, k_len), poison(v, k_len)
    o, lse = mita.prefix_forward(cfg, *t, q_len=lens(q_len), p_len=lens(p_len), k_len=lens(k_len),
                                 o=torch.full_like(q, float("nan")), ws=workspace(mita.prefix_workspace_size(cfg)))
    R = expected(cfg, t, q_len, p_len, k_len)
    e = dict(o=worst(o, R.o, R.eo), lse=worst(lse, R.lse, R.elz))
    log(f"[prefix] {cfg} {layout} {q_len} {p_len} {k_len}: " + " ".join(f"{n} {x:.3f}" for n, x in e.items()))
    assert max(e.values()) <= 1.0, e
    return o, lse


def config(case, d, dtype):
    B, Bp, H, Hk, N, P, Nk, _, left, right = case[:10]
    return mita.PrefixConfig(B, H, N, P, d, Bp=Bp, H_kv=Hk, N_k=Nk, dtype=dtype, left=left, right=right)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", CASES, ids=lambda s: "-".join(str(x) for x in s[:10]))
def test_against_float64(case, d, dtype):
    run_case(config(case, d, dtype), case[7], *case[10:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_scores_move_the_reference(dtype):
    # scores of standard deviation 25: the parts' maxima lie far apart, most weights vanish
    run_case(mita.PrefixConfig(12, 4, 1, 1900, 64, H_kv=2, N_k=300, dtype=dtype, right=0), std=25.0)
    run_case(mita.PrefixConfig(12, 4, 1, 900, 64, H_kv=2, N_k=300, dtype=dtype, right=0), std=25.0)
    run_case(mita.PrefixConfig(2, 4, 150, 300, 64, H_kv=2, N_k=150, dtype=dtype, right=0, scale=0.9), std=6.0)


@pytest.mark.parametrize("case", CASES[3:10:2] + CASES[14:17], ids=lambda s: "-".join(str(x) for x in s[:10]))
def test_as_dense_attention_of_the_whole_keys(case):
    cfg = config(case, 64, "bf16")
    q, kp, vp, k, v = make(cfg, case[7], 2)
    pl, kl = lengths(cfg, *case[11:])
    o, lse = mita.prefix_forward(cfg, q, kp, vp, k, v, q_len=lens(case[10]), p_len=lens(pl), k_len=lens(kl))
    dense = mita.DenseConfig(cfg.B, cfg.H, cfg.N, 64, H_kv=cfg.H_kv, N_k=cfg.P + cfg.N_k, left=cfg.left, right=cfg.right)
    kc, vc = (whole_keys(cfg, a, b, pl, kl) for a, b in ((kp, k), (vp, v)))
    S = cfg.B // cfg.Bp
    o2, lse2 = mita.dense_forward(dense, q, kc, vc, q_len=lens(case[10]),
                                  k_len=lens([pl[b // S] + kl[b] for b in range(cfg.B)]))
    R = expected(cfg, (q, kp, vp, k, v), *case[10:])
    assert float(((o - o2).double().abs() / (2 * R.eo + 1e-30)).max()) <= 1.0
    same = torch.isinf(lse) & (lse == lse2)
    assert float(torch.where(same, 0.0, (lse - lse2).double().abs() / (2 * R.elz + 1e-30)).max()) <= 1.0


def test_lengths_past_the_sizes_are_clamped():
    cfg = mita.PrefixConfig(4, 2, 3, 50, 64, Bp=2, N_k=60, right=0)
    t = make(cfg, "bhnd", 3)
    a = mita.prefix_forward(cfg, *t, q_len=lens([3, 0, 3, 3]), p_len=lens([50, 0]), k_len=lens([60, 0, 60, 5]))
    b = mita.prefix_forward(cfg, *t, q_len=lens([9, -5, 2 ** 31 - 1, 3]), p_len=lens([51, -2 ** 31]),
                            k_len=lens([2 ** 31 - 1, -1, 61, 5]))
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("N,P", [(1, 300), (1, 1300), (140, 300)])
def test_values_out_of_range(N, P):
    # a NaN or a score past the range makes its row NaN, and that alone
    cfg = mita.PrefixConfig(6, 2, N, P, 64, N_k=200, dtype="f32", right=0)
    q, kp, vp, k, v = make(cfg, "bhnd", 4)
    ok = mita.prefix_forward(cfg, q, kp, vp, k, v)
    q[1, 1, 0, 5] = float("nan")
    q[4, 0, N - 1] *= 1e9
    o, lse = mita.prefix_forward(cfg, q, kp, vp, k, v)
    assert torch.isnan(o[1, 1, 0]).all() and torch.isnan(lse[1, 1, 0])
    assert torch.isnan(o[4, 0, N - 1]).all() and torch.isnan(lse[4, 0, N - 1])
    keep = torch.ones((6, 2, N), dtype=torch.bool, device="cuda")
    keep[1, 1, 0] = keep[4, 0, N - 1] = False
    assert torch.equal(o[keep], ok[0][keep]) and torch.equal(lse[keep], ok[1][keep])


@pytest.mark.parametrize("N,P", [(1, 600), (1, 1600), (140, 600)])
def test_parts_without_weight(N, P):
    # scores so low in the prefix that they weigh nothing beside the own keys', and the other way round
    cfg = mita.PrefixConfig(6, 2, N, P, 64, N_k=200, dtype="f32")
    for low in ("prefix", "own"):
        q, kp, vp, k, v = make(cfg, "bhnd", 5)
        q[..., 0] = 1.0
        (kp if low == "prefix" else k)[..., 0] = -1e4
        o, lse = mita.prefix_forward(cfg, q, kp, vp, k, v)
        R = expected(cfg, (q, kp, vp, k, v), None, None, None)
        assert max(worst(o, R.o, R.eo), worst(lse, R.lse, R.elz)) <= 1.0


def test_offsets_past_32_bits():
    # 70000 prefix tokens of 256 heads in token order: the last head's last token lies 4.6 GB in
    P, H = 70000, 256
    cfg = mita.PrefixConfig(3, 1, 1, P, 128, N_k=20, right=0)
    q, kp, vp, k, v = make(cfg, "bhnd", 6)
    far = [torch.empty((1, P, H, 128), dtype=torch.bfloat16, device="cuda").transpose(1, 2)[:, H - 1:].copy_(x)
           for x in (kp, vp)]
    a = mita.prefix_forward(cfg, q, kp, vp, k, v)
    b = mita.prefix_forward(cfg, q, *far, k, v)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    R = expected(cfg, (q, kp, vp, k, v), None, None, None)
    assert max(worst(a[0], R.o, R.eo), worst(a[1], R.lse, R.elz)) <= 1.0


def test_repeated_heads_and_strided_caches():
    # one key head shown as two, own keys in a larger cache whose rows behind them stay as they are
    cfg = mita.PrefixConfig(4, 2, 2, 90, 64, N_k=40, right=0)
    g = gen(7)
    q = heads(g, 4, 2, 2, 64, torch.bfloat16, "bnhd")
    kp, vp = (heads(g, 1, 1, 90, 64, torch.bfloat16, "bhnd").expand(1, 2, 90, 64) for _ in range(2))
    cache = [torch.full((4, 2, 100, 64), float("nan"), device="cuda").bfloat16() for _ in range(2)]
    for c in cache:
        c[:, :, 30:70] = heads(g, 4, 2, 40, 64, torch.bfloat16, "bhnd")
    k, v = (c[:, :, 30:70] for c in cache)
    before = [c.clone() for c in cache]
    a = mita.prefix_forward(cfg, q, kp, vp, k, v)
    b = mita.prefix_forward(cfg, q, kp.contiguous(), vp.contiguous(), k.contiguous(), v.contiguous())
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(cache, before))


@pytest.mark.parametrize("N", [1, 150])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_same_bits_every_time_on_any_stream_and_in_a_graph(dtype, N):
    cfg = mita.PrefixConfig(8, 4, N, 1400, 64, Bp=2, H_kv=2, N_k=600, dtype=dtype, right=0)
    t = make(cfg, "bnhd", 8)
    kl = lens([600 - 70 * b for b in range(8)])
    ws = workspace(mita.prefix_workspace_size(cfg))
    call = lambda **kw: mita.prefix_forward(cfg, *t, k_len=kl, **kw)
    first = call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [call(stream=side) for _ in range(5)]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for o in got for x, y in zip(first, o))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(ws=ws)
    for seed in (9, 10, 11):  # the next step: other values, longer sequences, eager calls on the same workspace
        g = gen(seed)
        for x in t:
            x.copy_(torch.randn(x.shape, device="cuda", generator=g))
        kl += 3
        eager = call(ws=ws)
        for x in out:
            x.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(eager, out))


def test_two_calls_at_once_on_workspaces_of_their_own():
    cfg = mita.PrefixConfig(16, 4, 1, 3000, 64, H_kv=2, N_k=100, right=0)
    one, two = make(cfg, "bhnd", 12), make(cfg, "bhnd", 13)
    want = [mita.prefix_forward(cfg, *t) for t in (one, two)]
    sides = [torch.cuda.Stream() for _ in range(2)]
    for s in sides:
        s.wait_stream(torch.cuda.current_stream())
    got = [[mita.prefix_forward(cfg, *t, stream=s) for t, s in zip((one, two), sides)] for _ in range(10)]
    for s in sides:
        torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(x, y) for pair in got for a, b in zip(pair, want) for x, y in zip(a, b))


def test_more_rows_than_one_grid_dimension():
    """2^24 + 48 rows of two parts, sixteen to a workgroup of the join: 2^20 workgroups and three more."""
    B, H, Hk, P = 2 ** 20 + 3, 16, 2, 1600
    config = lambda n: mita.PrefixConfig(n, H, 1, P, 64, H_kv=Hk, N_k=1)
    g = gen(16)
    new = lambda *shape: torch.randn((*shape, 64), device="cuda", generator=g, dtype=torch.bfloat16)
    q, kp, vp, k, v = new(B, H, 1), new(1, Hk, P), new(1, Hk, P), new(B, Hk, 1), new(B, Hk, 1)
    o, lse = mita.prefix_forward(config(B), q, kp, vp, k, v, o=torch.full_like(q, float("nan")))
    assert bool(torch.isfinite(o).all()) and bool(torch.isfinite(lse).all())
    for at in (0, 2 ** 19, B - 16, B - 8):
        i = slice(at, at + 8)
        R = expected(config(8), (q[i], kp, vp, k[i], v[i]), None, None, None)
        assert max(worst(o[i], R.o, R.eo), worst(lse[i], R.lse, R.elz)) <= 1.0


def test_without_log_sum_exps():
    cfg = mita.PrefixConfig(3, 2, 1, 900, 64, N_k=10)
    t = make(cfg, "bhnd", 14)
    o, lse = mita.prefix_forward(cfg, *t, want_lse=False)
    assert lse is None and torch.equal(o, mita.prefix_forward(cfg, *t)[0])


def test_refusals():
    cfg = mita.PrefixConfig(4, 2, 1, 16, 64, Bp=2, N_k=8)
    q, kp, vp, k, v = make(cfg, "bhnd", 15)
    bad = lambda *a, **kw: pytest.raises(ValueError, mita.prefix_forward, cfg, *a, **kw)
    bad(q.cpu(), kp, vp, k, v)
    bad(q, kp.float(), vp, k, v)
    bad(q, kp[:1], vp, k, v)
    bad(q, kp, vp)
    bad(q, kp, vp, k, v[:, :, :4])
    bad(q, kp, vp, k, v, p_len=lens([1, 2, 3, 4]))
    bad(q, kp, vp, k, v, k_len=lens([1, 2, 3, 4]).long())
    bad(q, kp, vp, k, v, lse=torch.empty((4, 2, 2), device="cuda")[..., ::2])
    with pytest.raises(ValueError):
        mita.prefix_forward(mita.PrefixConfig(4, 2, 1, 16, 64, Bp=2), q, kp, vp, k, v)
    for kw in (dict(o=q), dict(o=kp.view(4, 2, 8, 64)[:, :, :1])):
        with pytest.raises(mita.MitaError) as e:
            mita.prefix_forward(cfg, q, kp, vp, k, v, **kw)
        assert e.value.status == mita.MITA_ERR_INVALID_ARG
    cfg = mita.PrefixConfig(4, 2, 1, 2000, 64, Bp=2, N_k=8)
    q, kp, vp, k, v = make(cfg, "bhnd", 15)
    assert mita.prefix_workspace_size(cfg) > 0
    with pytest.raises(mita.MitaError) as e:
        mita.prefix_forward(cfg, q, kp, vp, k, v, ws=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.status == mita.MITA_ERR_WORKSPACE

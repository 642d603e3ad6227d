"""Dense attention forward and backward on the GPU against float64 references
(tests/dense_reference.py, whose bounds the errors are measured in)."""
from __future__ import annotations

import copy
import pickle

import pytest
import torch

from paper_2602_01219_amd import mita
from tests.dense_reference import reference, worst
from tests.gpu_helpers import log

pytestmark = pytest.mark.gpu


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def heads(g, B, H, N, d, dtype, layout, std=1.0):
    if layout == "bnhd":
        return (torch.randn((B, N, H, d), device="cuda", generator=g) * std).to(dtype).transpose(1, 2)
    return (torch.randn((B, H, N, d), device="cuda", generator=g) * std).to(dtype)


def lens(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


def poison(t, x_len):
    """NaN behind every sequence's end."""
    if x_len is not None:
        for b, n in enumerate(x_len):
            t[b, :, n:] = float("nan")
    return t


def workspace(n):
    return torch.full((max(n, 1),), 0xFF, dtype=torch.uint8, device="cuda")


def run_case(cfg, layout="bhnd", q_len=None, k_len=None, std=1.5, seed=1, backward=True):
    g = gen(seed)
    B, H, N, d = cfg.q_shape
    Hk, Nk = cfg.k_shape[1:3]
    dt = cfg.torch_dtype
    if layout == "qkv":
        x = torch.randn((B, N, 3, H, d), device="cuda", generator=g).to(dt)
        q, k, v = (x[:, :, i].transpose(1, 2) for i in range(3))
    else:
        q = heads(g, B, H, N, d, dt, layout, std)
        k, v = (heads(g, B, Hk, Nk, d, dt, layout) for _ in range(2))
    poison(q, q_len), poison(k, k_len), poison(v, k_len)
    ql, kl = lens(q_len), lens(k_len)
    o = torch.full_like(q, float("nan"))
    ws = workspace(mita.dense_workspace_size(cfg))
    o, lse = mita.dense_forward(cfg, q, k, v, q_len=ql, k_len=kl, o=o if layout != "qkv" else None, ws=ws)
    R = reference(cfg, q, k, v, q_len, k_len)
    e = dict(o=worst(o, R.o, R.eo), lse=worst(lse, R.lse, R.elz))
    if backward:
        dO = poison(heads(g, B, H, N, d, dt, "bnhd" if layout == "bnhd" else "bhnd"), q_len)
        oin, lin = poison(o.clone(), q_len), lse.clone()
        if layout == "qkv":  # gradients into the slices of the projection's gradient
            dx = torch.full((B, N, 3, H, d), float("nan"), device="cuda").to(dt)
            dq, dk, dv = (dx[:, :, i].transpose(1, 2) for i in range(3))
        else:
            dq, dk, dv = (torch.full_like(t, float("nan")) for t in (q, k, v))
        ws = workspace(mita.dense_workspace_size(cfg, mita.WS_BACKWARD))
        mita.dense_backward(cfg, q, k, v, oin, lin, dO, q_len=ql, k_len=kl, dq=dq, dk=dk, dv=dv, ws=ws)
        R = reference(cfg, q, k, v, q_len, k_len, dO=dO, o=o, lse=lse)
        e.update(dq=worst(dq, R.dq, R.edq), dk=worst(dk, R.dk, R.edk), dv=worst(dv, R.dv, R.edv))
    log(f"[dense] {cfg} {layout} {q_len} {k_len}: " + " ".join(f"{n} {x:.3f}" for n, x in e.items()))
    assert max(e.values()) <= 1.0, e


SHAPES = [
    # B, H, Hk, N, Nk, layout, left, right, q_len, k_len
    (1, 1, 1, 1, 1, "bhnd", -1, -1, None, None),
    (2, 3, 3, 33, 33, "bhnd", -1, -1, None, None),
    (1, 2, 2, 196, 196, "qkv", -1, -1, None, None),
    (2, 2, 1, 129, 129, "bnhd", -1, 0, None, None),
    (1, 2, 2, 64, 257, "bhnd", -1, 0, None, None),            # new queries behind a prefix
    (1, 6, 2, 150, 70, "bnhd", -1, 0, None, None),            # the first queries see nothing
    (1, 2, 2, 300, 300, "bhnd", 0, 0, None, None),            # each sees itself
    (1, 4, 1, 277, 277, "bhnd", 37, 5, None, None),
    (1, 2, 1, 400, 391, "bnhd", 64, 0, None, None),
    (1, 1, 1, 200, 200, "bhnd", 3, -1, None, None),
    (4, 4, 2, 131, 131, "bnhd", -1, -1, [131, 1, 0, 64], [131, 1, 0, 64]),
    (4, 3, 1, 131, 131, "bhnd", -1, 0, [131, 77, 0, 1], [131, 77, 0, 1]),
    (4, 2, 2, 40, 170, "bhnd", -1, 0, [40, 0, 7, 40], [170, 33, 0, 5]),
    (3, 2, 2, 1, 700, "bnhd", -1, 0, None, [700, 1, 0]),
    (2, 8, 1, 1, 1500, "bnhd", 200, 0, None, [1500, 801]),
    (1, 16, 2, 3, 2100, "bhnd", -1, 0, None, None),           # a few tokens, keys split
    (1, 1, 1, 2050, 2050, "bhnd", -1, -1, None, None),        # one head: both sides split
    (1, 2, 1, 1100, 1030, "bhnd", 500, 0, [1000], [999]),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(x) for x in s[:8]))
def test_forward_and_backward(shape, d, dtype):
    B, H, Hk, N, Nk, layout, left, right, q_len, k_len = shape
    cfg = mita.DenseConfig(B, H, N, d, H_kv=Hk, N_k=Nk, dtype=dtype, left=left, right=right)
    run_case(cfg, layout, q_len, k_len)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_scores_move_the_reference(dtype):
    # scores of standard deviation 25: the running maximum moves often, most weights vanish
    run_case(mita.DenseConfig(1, 2, 190, 64, N_k=700, dtype=dtype), std=25.0)
    run_case(mita.DenseConfig(1, 2, 190, 64, N_k=190, dtype=dtype, scale=0.9, right=0), std=6.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tiles_filled_by_waves_without_rows(dtype):
    # one token of many sequences: the waves without rows copy tiles for the one that has them, many tiles long
    B = 32
    k_len = [8192 - 250 * b for b in range(B)]
    run_case(mita.DenseConfig(B, 16, 1, 128, H_kv=8, N_k=8192, dtype=dtype, right=0), "bnhd", None, k_len,
             backward=False)
    run_case(mita.DenseConfig(2, 2, 2, 64, H_kv=2, N_k=5000, dtype=dtype, right=0), "bnhd", None, [5000, 4001])


def test_many_query_heads_and_long_windows():
    run_case(mita.DenseConfig(1, 71, 9, 64, H_kv=1, N_k=40))
    run_case(mita.DenseConfig(1, 2, 100, 64, N_k=100, left=2 ** 31 - 1, right=2 ** 31 - 1))


def test_lengths_past_the_sizes_are_clamped():
    cfg = mita.DenseConfig(2, 2, 50, 64, N_k=60)
    g = gen(3)
    q, k, v = heads(g, 2, 2, 50, 64, torch.bfloat16, "bhnd"), *(heads(g, 2, 2, 60, 64, torch.bfloat16, "bhnd")
                                                                  for _ in range(2))
    a = mita.dense_forward(cfg, q, k, v, q_len=lens([50, 0]), k_len=lens([60, 0]))
    b = mita.dense_forward(cfg, q, k, v, q_len=lens([1000, -5]), k_len=lens([2 ** 31 - 1, -2 ** 31]))
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_repeated_heads_and_batches():
    # one key head shown as three (stride 0), and one batch element as two
    cfg = mita.DenseConfig(2, 3, 90, 64)
    g = gen(4)
    q = heads(g, 2, 3, 90, 64, torch.bfloat16, "bhnd")
    k1, v1 = heads(g, 2, 1, 90, 64, torch.bfloat16, "bhnd"), heads(g, 1, 3, 90, 64, torch.bfloat16, "bhnd")
    k, v = k1.expand(2, 3, 90, 64), v1.expand(2, 3, 90, 64)
    o, lse = mita.dense_forward(cfg, q, k, v)
    o2, lse2 = mita.dense_forward(cfg, q, k.contiguous(), v.contiguous())
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    dO = heads(g, 2, 3, 90, 64, torch.bfloat16, "bhnd")
    one = mita.dense_backward(cfg, q, k, v, o, lse, dO)
    two = mita.dense_backward(cfg, q, k.contiguous(), v.contiguous(), o, lse, dO)
    assert all(torch.equal(x, y) for x, y in zip(one, two))


def test_offsets_past_32_bits():
    # 70000 tokens of 256 heads in token order: the last head's last token lies 4.6 GB in
    N_k, H = 70000, 256
    cfg = mita.DenseConfig(1, 1, 2, 128, N_k=N_k, right=0)
    g = gen(5)
    q = heads(g, 1, 1, 2, 128, torch.bfloat16, "bhnd")
    bufs = [torch.empty((1, N_k, H, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    k, v = (x.transpose(1, 2)[:, H - 1:] for x in bufs)
    k.copy_(heads(g, 1, 1, N_k, 128, torch.bfloat16, "bhnd"))
    v.copy_(heads(g, 1, 1, N_k, 128, torch.bfloat16, "bhnd"))
    o, lse = mita.dense_forward(cfg, q, k, v)
    o2, lse2 = mita.dense_forward(cfg, q, k.contiguous(), v.contiguous())
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    dO = heads(g, 1, 1, 2, 128, torch.bfloat16, "bhnd")
    dk, dv = (torch.empty((1, N_k, H, 128), dtype=torch.bfloat16, device="cuda").transpose(1, 2)[:, H - 1:]
              for _ in range(2))
    mita.dense_backward(cfg, q, k, v, o, lse, dO, dk=dk, dv=dv)
    _, dk2, dv2 = mita.dense_backward(cfg, q, k.contiguous(), v.contiguous(), o, lse, dO)
    assert torch.equal(dk, dk2) and torch.equal(dv, dv2)
    R = reference(cfg, q, k, v, dO=dO, o=o, lse=lse)
    assert max(worst(o, R.o, R.eo), worst(dk, R.dk, R.edk), worst(dv, R.dv, R.edv)) <= 1.0


def test_grouped_heads_4_gib_apart():
    # two query heads of one key head, their rows 2^31 elements apart
    N = 70
    cfg = mita.DenseConfig(1, 2, N, 64, H_kv=1, right=0)
    g = gen(15)
    buf = torch.empty(2 ** 31 + N * 64, dtype=torch.bfloat16, device="cuda")
    q = buf.as_strided((1, 2, N, 64), (2 ** 32, 2 ** 31, 64, 1))
    q.copy_(heads(g, 1, 2, N, 64, torch.bfloat16, "bhnd"))
    k, v = (heads(g, 1, 1, N, 64, torch.bfloat16, "bhnd") for _ in range(2))
    dO = heads(g, 1, 2, N, 64, torch.bfloat16, "bhnd")
    o, lse = mita.dense_forward(cfg, q, k, v)
    near = q.contiguous()
    o2, lse2 = mita.dense_forward(cfg, near, k, v)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    far = mita.dense_backward(cfg, q, k, v, o, lse, dO, dq=torch.empty_like(near))
    assert all(torch.equal(x, y) for x, y in zip(far, mita.dense_backward(cfg, near, k, v, o, lse, dO)))


def test_configurations_copy_and_pickle_after_use():
    cfg = mita.DenseConfig(1, 1, 3, 64)
    g = gen(16)
    x = heads(g, 1, 1, 3, 64, torch.bfloat16, "bhnd")
    mita.dense_forward(cfg, x, x.clone(), x.clone())
    for other in (copy.deepcopy(cfg), pickle.loads(pickle.dumps(cfg))):
        assert other == cfg and "_plans" not in other.__dict__


def test_a_stream_of_its_own_without_given_outputs():
    # the call's allocations belong to the stream it runs on
    cfg = mita.DenseConfig(2, 2, 64, 64, N_k=2048)
    g = gen(17)
    q = heads(g, 2, 2, 64, 64, torch.bfloat16, "bhnd")
    k, v = (heads(g, 2, 2, 2048, 64, torch.bfloat16, "bhnd") for _ in range(2))
    ref = mita.dense_forward(cfg, q, k, v)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [mita.dense_forward(cfg, q, k, v, stream=side) for _ in range(20)]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for o in got for a, b in zip(o, ref))


def test_gradient_against_differences():
    # directional derivatives of sum(o * dO) in float64 (step 1e-4: truncation about 1e-8 of the third
    # derivative, far below the kernel's fp32 error, bounded by the element bounds along the direction)
    cfg = mita.DenseConfig(1, 4, 21, 64, H_kv=2, N_k=34, dtype="f32", left=9, right=2)
    g = gen(6)
    x = [heads(g, 1, 4, 21, 64, torch.float32, "bhnd")] + [heads(g, 1, 2, 34, 64, torch.float32, "bhnd") for _ in range(2)]
    dO = heads(g, 1, 4, 21, 64, torch.float32, "bhnd")
    o, lse = mita.dense_forward(cfg, *x)
    grads = mita.dense_backward(cfg, *x, o, lse, dO)
    R = reference(cfg, *x, dO=dO, o=o, lse=lse)
    f = lambda y: float((reference(cfg, *y).o * dO.double()).sum())
    for i, (grad, bound) in enumerate(zip(grads, (R.edq, R.edk, R.edv))):
        way = torch.randn(grad.shape, device="cuda", generator=g, dtype=torch.float64)
        hi, lo = ([t.double() + (s * 1e-4 * way if j == i else 0) for j, t in enumerate(x)] for s in (1, -1))
        diff = (f(hi) - f(lo)) / 2e-4
        got = float((grad.double() * way).sum())
        # the given o and lse are rounded to fp32: D and P carry their errors, below the element bounds
        assert abs(got - diff) <= float((bound * way.abs()).sum()) + 1e-6 * abs(diff) + 1e-6, (i, got, diff)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_same_bits_every_time_on_any_stream_and_in_a_graph(dtype):
    cfg = mita.DenseConfig(2, 4, 150, 64, H_kv=2, N_k=1400, dtype=dtype, right=0)
    g = gen(7)
    dt = cfg.torch_dtype
    q, dO = (heads(g, 2, 4, 150, 64, dt, "bhnd") for _ in range(2))
    k, v = (heads(g, 2, 2, 1400, 64, dt, "bnhd") for _ in range(2))

    def both(ws=(None, None), out=None, stream=None):
        out = out or [torch.empty_like(q), torch.empty((2, 4, 150), device="cuda"), torch.empty_like(q),
                      torch.empty_like(k), torch.empty_like(v)]
        o, lse, dq, dk, dv = out
        mita.dense_forward(cfg, q, k, v, o=o, lse=lse, ws=ws[0], stream=stream)
        mita.dense_backward(cfg, q, k, v, o, lse, dO, dq=dq, dk=dk, dv=dv, ws=ws[1], stream=stream)
        return out

    first = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = both()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for x, y in zip(first, other))
    # the stream as an argument
    out = [torch.empty_like(x) for x in first]
    ws = [torch.empty(max(1, mita.dense_workspace_size(cfg, w)), dtype=torch.uint8, device="cuda")
          for w in (mita.WS_FORWARD, mita.WS_BACKWARD)]
    side.wait_stream(torch.cuda.current_stream())
    both(ws, out, side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for x, y in zip(first, out))
    # captured and replayed with new inputs, eager calls on the same workspaces in between
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(ws, out)
    for seed in (8, 9, 10):
        g = gen(seed)
        for t in (q, k, v, dO):
            t.copy_(torch.randn(t.shape, device="cuda", generator=g))
        eager = both(ws)
        for t in out:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(eager, out))


def test_rows_do_not_depend_on_the_rest_of_the_batch():
    # a sequence alone and as an element of a padded batch: the same gradients and outputs bit for bit,
    # where the batch does not change how the keys are split
    g = gen(11)
    q, k, v, dO = (heads(g, 3, 2, 200, 64, torch.bfloat16, "bhnd") for _ in range(4))
    cfg = mita.DenseConfig(3, 2, 200, 64, right=0)
    n = lens([200, 90, 0])
    o, lse = mita.dense_forward(cfg, q, k, v, q_len=n, k_len=n)
    grads = mita.dense_backward(cfg, q, k, v, o, lse, dO, q_len=n, k_len=n)
    one = mita.DenseConfig(1, 2, 90, 64, right=0)
    cut = [t[1:2, :, :90] for t in (q, k, v, dO)]
    o1, lse1 = mita.dense_forward(one, *cut[:3])
    assert torch.equal(o[1:2, :, :90], o1) and torch.equal(lse[1:2, :, :90], lse1)
    g1 = mita.dense_backward(one, *cut[:3], o1, lse1, cut[3])
    assert all(torch.equal(x[1:2, :, :90], y) for x, y in zip(grads, g1))
    assert all((x[1, :, 90:] == 0).all() and (x[2] == 0).all() for x in (o, *grads))
    assert torch.isneginf(lse[2]).all()


def test_without_log_sum_exps():
    cfg = mita.DenseConfig(1, 2, 5, 64, N_k=900)
    g = gen(12)
    q = heads(g, 1, 2, 5, 64, torch.bfloat16, "bhnd")
    k, v = (heads(g, 1, 2, 900, 64, torch.bfloat16, "bhnd") for _ in range(2))
    o, lse = mita.dense_forward(cfg, q, k, v, want_lse=False)
    assert lse is None and torch.equal(o, mita.dense_forward(cfg, q, k, v)[0])


def test_mita_route_only_is_dense_attention():
    """MiTA with one landmark whose expert holds every key, without the shared
    expert, is dense attention."""
    g = gen(13)
    q, k, v, dO = (heads(g, 1, 2, 256, 64, torch.float32, "bhnd") for _ in range(4))
    m = mita.Config(B=1, H=2, N=256, d=64, grid_h=16, grid_w=16, M=1, lm_h=1, lm_w=1, k=256, dtype="f32", use_shared=0)
    o = mita.forward(m, q, k, v)
    gm = mita.backward(m, q, k, v, o, dO)
    cfg = mita.DenseConfig(1, 2, 256, 64, dtype="f32")
    o2, lse = mita.dense_forward(cfg, q, k, v)
    gd = mita.dense_backward(cfg, q, k, v, o2, lse, dO)
    R = reference(cfg, q, k, v, dO=dO, o=o2, lse=lse)
    for x, y, e in zip((o, *gm), (o2, *gd), (R.eo, R.edq, R.edk, R.edv)):
        assert float(((x - y).double().abs() / (2 * e + 1e-30)).max()) <= 1.0


def test_refusals():
    g = gen(14)
    q, k, v = (heads(g, 1, 2, 16, 64, torch.bfloat16, "bhnd") for _ in range(3))
    cfg = mita.DenseConfig(1, 2, 16, 64)
    bad = lambda *a, **kw: pytest.raises(ValueError, mita.dense_forward, cfg, *a, **kw)
    bad(q.cpu(), k, v)
    bad(q, k.cpu(), v)
    bad(q.float(), k, v)
    bad(q[:, :1], k, v)
    bad(q, k.transpose(2, 3).contiguous().transpose(2, 3), v)
    bad(q, k[:, :, :1].expand(1, 2, 16, 64), v)
    bad(q, k, v, q_len=torch.zeros(1, dtype=torch.int64, device="cuda"))
    bad(q, k, v, k_len=torch.zeros(2, dtype=torch.int32, device="cuda"))
    bad(q, k, v, lse=torch.empty((1, 2, 32), device="cuda")[..., ::2])
    for kw in (dict(o=q), dict(o=k)):
        with pytest.raises(mita.MitaError) as e:
            mita.dense_forward(cfg, q, k, v, **kw)
        assert e.value.status == mita.MITA_ERR_INVALID_ARG
    o, lse = mita.dense_forward(cfg, q, k, v)
    for kw in (dict(dq=q), dict(dk=v), dict(dq=o)):
        with pytest.raises(mita.MitaError) as e:
            mita.dense_backward(cfg, q, k, v, o, lse, o.clone(), **kw)
        assert e.value.status == mita.MITA_ERR_INVALID_ARG
    same = torch.empty_like(k)
    with pytest.raises(mita.MitaError):
        mita.dense_backward(cfg, q, k, v, o, lse, o.clone(), dk=same, dv=same)
    long = mita.DenseConfig(1, 2, 1, 64, N_k=4096)
    k4, v4 = (heads(g, 1, 2, 4096, 64, torch.bfloat16, "bhnd") for _ in range(2))
    assert mita.dense_workspace_size(long) > 0
    with pytest.raises(mita.MitaError) as e:
        mita.dense_forward(long, q[:, :, :1].contiguous(), k4, v4, ws=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.status == mita.MITA_ERR_WORKSPACE

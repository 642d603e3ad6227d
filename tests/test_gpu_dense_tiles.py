"""The 128-row kernel of the dense attention's forward (and the backward of the
same calls) against float64 references, in the bounds of tests/dense_reference.py."""
from __future__ import annotations

import pytest
import torch

from paper_2602_01219_amd import mita
from tests.dense_tile_cases import TILE_CASES
from tests.test_gpu_dense import gen, heads, run_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", TILE_CASES, ids=lambda s: "-".join(str(x) for x in s[:8]))
def test_forward_and_backward(case, d, dtype):
    B, H, Hk, N, Nk, layout, left, right, q_len, k_len = case
    cfg = mita.DenseConfig(B, H, N, d, H_kv=Hk, N_k=Nk, dtype=dtype, left=left, right=right)
    run_case(cfg, layout, q_len, k_len)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_large_scores_move_the_reference(d, dtype):
    run_case(mita.DenseConfig(8, 16, 140, d, N_k=700, dtype=dtype), std=25.0, backward=False)
    run_case(mita.DenseConfig(8, 16, 140, d, N_k=1100, dtype=dtype, right=0), std=25.0, backward=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_same_bits_in_a_graph(dtype):
    # whole (200 keys) and split (1100 keys), replayed with new inputs beside eager calls
    for Nk in (200, 1100):
        cfg = mita.DenseConfig(8, 16, 140, 64, N_k=Nk, dtype=dtype, right=0)
        g = gen(1)
        q = heads(g, 8, 16, 140, 64, cfg.torch_dtype, "bnhd")
        k, v = (heads(g, 8, 16, Nk, 64, cfg.torch_dtype, "bhnd") for _ in range(2))
        mita.dense_forward(cfg, q, k, v)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = mita.dense_forward(cfg, q, k, v)
        for seed in (2, 3, 4):
            g = gen(seed)
            for t in (q, k, v):
                t.copy_(torch.randn(t.shape, device="cuda", generator=g))
            eager = mita.dense_forward(cfg, q, k, v)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(eager, out))

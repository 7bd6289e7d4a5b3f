"""Differential attention of single tokens: its whole error is its output's rounding.

Limit of the relative 2-norm of the error.  A bf16 output alone: an even error of up to half a
step, 2^-8 of the element's power of two, so 2^-8 / sqrt(3) = 2.26e-3 of that and, with significands
between 1 and 2 (mean square about 2.2 where their logarithms are even), 1.5e-3 of the elements; up
to 1.7e-3 where more significands are small.  Weights of two bf16 (2^-17) or of fp16 (2^-11 / sqrt(3)
at most = 2.8e-4, times about 2 where the maps cancel) add in squares: below 1.8e-3.  One bf16 weight
(eight times fp16's) gives 2.2e-3 and more.  LIMIT lies between; test_diff_rounding.py shows both sides
in 64 bits."""
import numpy as np
import pytest
import torch

import cw_workloads as cw
import oracle
import paper_2606_16824_amd as cwlib
from conftest import paged_inputs
from gpu_util import to_gpu

pytestmark = pytest.mark.gpu
LIMIT = 1.9e-3
CASES = [
    # lp, pairs, g, d, page
    ([900, 1500, 333, 2100, 640], 2, 4, 128, 16),
    ([900, 1500, 333, 2100, 640], 2, 4, 64, 64),
    ([40, 77, 129, 64, 31, 100], 4, 2, 128, 64),
]


@pytest.mark.parametrize("dt", ["bf16", "fp8"])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_single_tokens(i, dt):
    lp, pairs, g, d, page = CASES[i]
    print(f"\n[case] diff precision {CASES[i]} {dt}", flush=True)
    w = cw.materialize(cw.custom_spec(lp, [1] * len(lp), num_kv_heads=2 * pairs, gqa_group=g, head_dim=d, page_size=page,
                                      kv_dtype=dt, seed=8))
    lam = np.random.default_rng(8).uniform(0.2, 0.8, size=pairs * g).astype(np.float32)
    dw, s = to_gpu(w), w.spec
    out = cwlib.diff_attention(dw.q, dw.k_new, dw.v_new, dw.k_pool, dw.v_pool, dw.block_table, s.prefix_lens, s.suffix_lens, g,
                               s.softmax_scale, torch.from_numpy(lam).cuda(), k_scale=dw.k_scale, v_scale=dw.v_scale)
    torch.cuda.synchronize()
    ref, _ = oracle.diff_attention(paged_inputs(w), lam)
    relative = np.linalg.norm(out.cpu().double().numpy() - ref) / np.linalg.norm(ref)
    print(f"[precision] relative {relative:.3e}", flush=True)
    assert relative <= LIMIT

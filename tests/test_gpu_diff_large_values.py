"""Differential attention over bf16 pools with values of the largest size that the header allows
(2^80): fp32 sums of weights, each up to 2^16, times values."""
import numpy as np
import pytest
import torch

import cw_workloads as cw
import oracle
import paper_2606_16824_amd as cwlib
from conftest import paged_inputs
from gpu_util import to_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
def test_values_of_2_80(d):
    print(f"\n[case] diff values of 2^80 d={d}", flush=True)
    lp, ls = [1300, 0, 70, 900, 2000], [90, 130, 33, 1, 1]
    w = cw.materialize(cw.custom_spec(lp, ls, num_kv_heads=4, gqa_group=3, head_dim=d, page_size=16, seed=61))
    w.v_pool.copy_((w.v_pool.float().clamp(-4, 4) * 2.0 ** 78).to(torch.bfloat16))  # (slots behind a prefix stay NaN)
    w.v_new.copy_((w.v_new.float().clamp(-4, 4) * 2.0 ** 78).to(torch.bfloat16))
    w.k_pool *= 3  # (scores of up to 15: far above the running max's 2^-8 of a block)
    dw, s = to_gpu(w), w.spec
    lam = np.random.default_rng(4).uniform(0.2, 0.8, size=6).astype(np.float32)
    out = cwlib.diff_attention(dw.q, dw.k_new, dw.v_new, dw.k_pool, dw.v_pool, dw.block_table, s.prefix_lens, s.suffix_lens, 3,
                               s.softmax_scale, torch.from_numpy(lam).cuda())
    torch.cuda.synchronize()
    ref, terms = oracle.diff_attention(paged_inputs(w), lam)
    # bf16 weights of chunks in numerator and sum, 2^-10 for the fp32 parts, the scores' sums
    r = 2 * 2.0 ** -8 + 2.0 ** -10 + 2.0 ** -15 * terms["scores"]
    got = out.cpu().double().numpy()
    assert np.isfinite(got).all() and np.abs(got).max() > 2.0 ** 77
    over = np.abs(got - ref) / (r * terms["mass"] + 2.0 ** -8 * np.abs(ref))
    print(f"[large values] worst {over.max():.3f} of the tolerance", flush=True)
    assert over.max() <= 1.0

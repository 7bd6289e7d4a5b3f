"""Chunks of differential attention over fp8 pools whose values are so small that fp16, which the kernel holds
them in, has only some of its bits left: page scales that are no powers of two.

All values of a pool are one code, so that no errors cancel.  Tolerance, per element, as in
test_gpu_diff_fp8_scores.py, r mass, and 2^-25 of each value (half a step of fp16 below 2^-14) with the maps' weights,
which sum to 1 and |lam|; stored: + 2^-8 |x|."""
import numpy as np
import pytest
import torch

import cw_workloads as cw
import oracle
import paper_2606_16824_amd as cwlib
from conftest import paged_inputs
from gpu_util import to_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale,code", [(1.9375 * 2.0 ** -29, 0x77), (1.0625 * 2.0 ** -27, 0x6B), (1.37 * 2.0 ** -22, 0x55),
                                        (1.99 * 2.0 ** -15, 0x09), (1.7 * 2.0 ** -33, 0x7E), (1.3, 0x6D)])
@pytest.mark.parametrize("d,page", [(128, 16), (64, 64)])
def test_values_of_any_size(d, page, scale, code):
    print(f"\n[case] diff small values d={d} page={page} {scale} code {code}", flush=True)
    w = cw.materialize(cw.custom_spec([300, 64], [40, 70], num_kv_heads=4, gqa_group=3, head_dim=d, page_size=page,
                                      kv_dtype="fp8", seed=7))
    w.v_scale.fill_(scale)
    w.v_pool.fill_(code)
    value = torch.tensor([code], dtype=torch.uint8).view(torch.float8_e4m3fn).float() * scale
    w.v_new.copy_(value.to(torch.bfloat16).expand(w.v_new.shape))
    lam = np.array([-1.0, 0.5, -0.25, 1.0, -1.0, 0.0], dtype=np.float32)
    dw, s = to_gpu(w), w.spec
    out = cwlib.diff_attention(dw.q, dw.k_new, dw.v_new, dw.k_pool, dw.v_pool, dw.block_table, s.prefix_lens, s.suffix_lens, 3,
                               s.softmax_scale, torch.from_numpy(lam).cuda(), k_scale=dw.k_scale, v_scale=dw.v_scale)
    torch.cuda.synchronize()
    ref, terms = oracle.diff_attention(paged_inputs(w), lam)
    r = 2 * 2.0 ** -11 + 2.0 ** -10 + 2.0 ** -10 + 2.0 ** -15 * terms["scores"]
    tol = r * terms["mass"] + 2.0 ** -25 * (1 + np.abs(lam.astype(np.float64)))[None, :, None] + 2.0 ** -8 * np.abs(ref)
    over = np.abs(out.cpu().double().numpy() - ref) / tol
    print(f"[diff small values] worst {over.max():.3f} of the tolerance", flush=True)
    assert over.max() <= 1.0

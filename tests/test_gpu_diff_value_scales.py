"""Single new tokens over fp8 pages: V scales of any size, also on pages that carry no weight.

Tolerance, per element, as in test_gpu_diff_fp8_scores.py: r mass with the fp16 weights' 2^-11
in numerator and sum, 2^-10 for the fp32 parts and 2^-15 of the scores; stored: + 2^-8 |x|."""
import numpy as np
import pytest
import torch

import cw_workloads as cw
import oracle
import paper_2606_16824_amd as cwlib
from conftest import paged_inputs
from gpu_util import to_gpu
from test_gpu_diff_fp8_scores import _peaked

pytestmark = pytest.mark.gpu


def _check(w, lam, what, after=1.0):
    dw, s = to_gpu(w), w.spec
    out = cwlib.diff_attention(dw.q, dw.k_new, dw.v_new, dw.k_pool, dw.v_pool, dw.block_table, s.prefix_lens, s.suffix_lens,
                               s.gqa_group, s.softmax_scale, torch.from_numpy(lam).cuda(), k_scale=dw.k_scale,
                               v_scale=dw.v_scale, out_scale=after)
    torch.cuda.synchronize()
    ref, terms = oracle.diff_attention(paged_inputs(w), lam, out_scale=after)
    got = out.cpu().double().numpy()
    assert np.isfinite(got).all(), what
    r = 2 * 2.0 ** -11 + 2.0 ** -10 + 2.0 ** -15 * terms["scores"]
    over = np.abs(got - ref) / (after * r * terms["mass"] + 2.0 ** -8 * np.abs(ref))
    print(f"[{what}] worst {over.max():.3f} of the tolerance", flush=True)
    assert over.max() <= 1.0, what


@pytest.mark.parametrize("where", ["first", "middle", "last"])
@pytest.mark.parametrize("d,page", [(128, 16), (64, 64)])
def test_a_page_without_weight_may_have_any_value_scale(d, page, where):
    """One page's keys point away from every query (its weights are below 2^-150) and its values are
    2^27 times larger than the others."""
    print(f"\n[case] diff value scale of a page without weight, {where} d={d} page={page}", flush=True)
    lp = [700, 333, 1500]
    w, lam = _peaked(lp, [1, 1, 1], 2, 3, d, page, seed=17 + d, size=60.0)
    for b in range(3):
        n = -(-lp[b] // page)
        pg = int(w.block_table[b, {"first": 0, "middle": n // 2, "last": n - 1}[where]])
        w.k_pool[pg] ^= 0x80  # the codes' sign (0xFF stays a NaN behind the prefix)
        w.v_scale[pg] *= 2.0 ** 27
    _check(w, lam, f"no weight {where} {d} {page}")


@pytest.mark.parametrize("exponent", [-130, -100, 60])
@pytest.mark.parametrize("d,page", [(128, 16), (64, 16), (128, 64)])
def test_all_value_scales_tiny_or_huge(d, page, exponent):
    """Also where the last tile of 32 keys ends in its first 16, behind which there is no page."""
    print(f"\n[case] diff value scales about 2^{exponent} d={d} page={page}", flush=True)
    lp = [37, 5, 1000, 16]
    w = cw.materialize(cw.custom_spec(lp, [1] * 4, num_kv_heads=4, gqa_group=3, head_dim=d, page_size=page, kv_dtype="fp8",
                                      seed=5 + d))
    w.v_scale.copy_((w.v_scale.double() * 16 * 2.0 ** exponent).float())
    w.v_new.zero_()
    rng = np.random.default_rng(3)
    lam = rng.uniform(0.2, 0.8, size=6).astype(np.float32)
    _check(w, lam, f"scales 2^{exponent} {d} {page}", after=2.0 ** (-exponent if exponent > -128 else 120))

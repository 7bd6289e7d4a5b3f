"""Differential attention over fp8 pools where attention is peaked: scores of 40 to 80, whose errors
the softmax turns into errors of the weights.

Tolerance, per element, before the norm (the maps' difference): r mass, mass = sum (p1 + |lam| p2)
|v|.  The scores are exact products (fp8 codes and bf16 values in the operand type) summed in
fp32, at most D = 128 roundings of 2^-24 of sum |q k| = `scores`, then times c and the page's
scale and less the running max, three more; a weight moves by as much relatively, in numerator and
sum: 2 (128 + 3) 2^-24 scores < 2^-15 scores.  No other part grows with the scores.  Weights:
2^-11 in fp16, numerator and sum; chunks: 2^-10 for a value (code x scale in fp16, the scale
rounded too); 2^-10 for the other fp32 parts.  Stored: + 2^-8 |x|."""
import numpy as np
import pytest
import torch

import cw_workloads as cw
import oracle
import paper_2606_16824_amd as cwlib
from conftest import paged_inputs
from gpu_util import to_gpu

pytestmark = pytest.mark.gpu


def _peaked(lp, ls, pairs, g, d, page, seed, size):
    """Keys along their map's sign pattern and queries along it too, so a score is nearly the sum of
    its terms' sizes; page scales of any significand."""
    w = cw.materialize(cw.custom_spec(lp, ls, num_kv_heads=2 * pairs, gqa_group=g, head_dim=d, page_size=page, kv_dtype="fp8",
                                      seed=seed))
    rng = np.random.default_rng(seed)
    sign = torch.from_numpy(rng.choice([-1.0, 1.0], size=(2 * pairs, d)).astype(np.float32))
    mag = lambda *s: torch.from_numpy(rng.uniform(0.5, 1.5, size=s).astype(np.float32))
    t = w.q.shape[0]
    unit = size / d ** 0.5  # d terms of about this, times softmax_scale = 1 / sqrt(d): `size`
    q = mag(t, pairs, g, 2, d) * sign.view(1, pairs, 1, 2, d)
    w.q.copy_(q.reshape(t, 2 * pairs * g, d).to(torch.bfloat16))
    w.k_new.copy_((mag(t, 2 * pairs, d) * sign * unit).to(torch.bfloat16))
    n = w.k_pool.shape[0]
    w.k_scale.copy_(torch.from_numpy(rng.uniform(0.01, 0.1, size=(n, 2 * pairs)).astype(np.float32)))
    k = mag(n, 2 * pairs, page, d) * sign[None, :, None, :] * unit
    codes = (k / w.k_scale[:, :, None, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    for b in range(len(lp)):
        for j in range(-(-lp[b] // page)):
            pg, rows = int(w.block_table[b, j]), min(page, lp[b] - j * page)
            w.k_pool[pg, :, :rows] = codes[pg, :, :rows]
    lam = rng.uniform(0.2, 0.8, size=pairs * g).astype(np.float32)
    return w, lam


@pytest.mark.parametrize("d,page,lp,ls", [
    (128, 16, [700, 37, 0, 333], [90, 130, 70, 2]),
    (128, 64, [701, 64, 5, 500], [40, 33, 90, 150]),
    (64, 64, [700, 37, 0, 333], [90, 130, 70, 2]),
    (64, 16, [1023, 95, 31, 1], [17, 66, 130, 300]),
    (128, 16, [700, 37, 333], [1, 1, 1]),
    (64, 64, [700, 37, 333], [1, 1, 1]),
])
def test_peaked_scores(d, page, lp, ls):
    print(f"\n[case] diff peaked scores d={d} page={page} {lp} {ls}", flush=True)
    w, lam = _peaked(lp, ls, 2, 3, d, page, seed=41 + d + page + len(lp), size=60.0)
    dw, s = to_gpu(w), w.spec
    out = cwlib.diff_attention(dw.q, dw.k_new, dw.v_new, dw.k_pool, dw.v_pool, dw.block_table, s.prefix_lens, s.suffix_lens,
                               3, s.softmax_scale, torch.from_numpy(lam).cuda(), k_scale=dw.k_scale, v_scale=dw.v_scale)
    torch.cuda.synchronize()
    ref, terms = oracle.diff_attention(paged_inputs(w), lam)
    chunk = np.repeat(s.suffix_lens > 1, s.suffix_lens)[:, None, None]
    r = 2 * 2.0 ** -11 + 2.0 ** -10 + np.where(chunk, 2.0 ** -10, 0.0) + 2.0 ** -15 * terms["scores"]
    over = np.abs(out.cpu().double().numpy() - ref) / (r * terms["mass"] + 2.0 ** -8 * np.abs(ref))
    print(f"[peaked] scores up to {terms['scores'].max():.0f}, worst {over.max():.3f} of the tolerance", flush=True)
    assert 40 < terms["scores"].max() < 150 and over.max() <= 1.0

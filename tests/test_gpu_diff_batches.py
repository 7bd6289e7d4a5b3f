"""Differential attention of batches as a server has them: from 8 to some hundred single tokens on
ragged prefixes (above 8 an item's sequence is searched by the whole wave), alone and beside chunks,
with the plan in the kernel arguments and too large for them.  Tolerance, per element, as in
test_gpu_diff_fp8_scores.py; over bf16 pools a chunk's weights are bf16 (2^-8 in numerator and sum)
and a single token's two bf16 (2^-16)."""
import numpy as np
import pytest
import torch

import cw_workloads as cw
import oracle
import paper_2606_16824_amd as cwlib
from conftest import paged_inputs
from gpu_util import to_gpu

pytestmark = pytest.mark.gpu


def _lens(rng, singles, chunks):
    lp = rng.integers(0, 400, size=singles + chunks)
    lp[rng.random(len(lp)) < 0.1] = 0
    lp[rng.random(len(lp)) < 0.1] = 32
    ls = np.concatenate([np.ones(singles, dtype=np.int64), rng.integers(2, 90, size=chunks)])
    ls[rng.random(len(ls)) < 0.03] = 0
    order = rng.permutation(len(lp))
    return lp[order], ls[order]


@pytest.mark.parametrize("dt", ["bf16", "fp8"])
@pytest.mark.parametrize("singles,chunks,d,page,pairs,g,in_args", [
    (9, 0, 128, 16, 2, 3, True),  # eight are left: the most that are searched by scalar loads
    (10, 0, 128, 16, 2, 3, True),
    (48, 0, 64, 64, 1, 4, True),
    (64, 0, 128, 64, 1, 2, True),
    (250, 0, 64, 16, 1, 1, True),
    (900, 0, 128, 16, 1, 1, False),
    (12, 3, 128, 16, 2, 2, None),
    (60, 5, 64, 16, 1, 3, None),
    (40, 40, 128, 64, 2, 1, None),
    (500, 20, 64, 64, 1, 2, False),
])
def test_batch(singles, chunks, d, page, pairs, g, in_args, dt):
    print(f"\n[case] diff batch of {singles} singles, {chunks} chunks d={d} page={page} {dt}", flush=True)
    rng = np.random.default_rng(singles + chunks + d)
    lp, ls = _lens(rng, singles, chunks)
    w = cw.materialize(cw.custom_spec(lp.tolist(), ls.tolist(), num_kv_heads=2 * pairs, gqa_group=g, head_dim=d, page_size=page,
                                      kv_dtype=dt, seed=singles + d))
    dw, s = to_gpu(w), w.spec
    lam = rng.uniform(-0.3, 0.9, size=pairs * g).astype(np.float32)
    out = torch.full((dw.q.shape[0], pairs * g, 2 * d), float("nan"), dtype=torch.bfloat16, device="cuda")
    before = cwlib.arg_plan_calls()
    cwlib.diff_attention(dw.q, dw.k_new, dw.v_new, dw.k_pool, dw.v_pool, dw.block_table, s.prefix_lens, s.suffix_lens, g,
                         s.softmax_scale, torch.from_numpy(lam).cuda(), k_scale=dw.k_scale, v_scale=dw.v_scale, out=out)
    torch.cuda.synchronize()
    if in_args is not None:
        assert cwlib.arg_plan_calls() - before == (1 if in_args else 0)
    ref, terms = oracle.diff_attention(paged_inputs(w), lam)
    chunk = np.repeat(s.suffix_lens > 1, s.suffix_lens)[:, None, None]
    fp8 = dt == "fp8"
    r = np.where(chunk, 2 * 2.0 ** (-11 if fp8 else -8) + (2.0 ** -10 if fp8 else 0.0), 2 * 2.0 ** (-11 if fp8 else -16))
    r = r + 2.0 ** -10 + 2.0 ** -15 * terms["scores"]
    got = out.cpu().double().numpy()
    over = np.abs(got - ref) / (r * terms["mass"] + 2.0 ** -8 * np.abs(ref))
    print(f"[batch] worst {over.max():.3f} of the tolerance over {len(ref)} rows", flush=True)
    assert np.isfinite(got).all() and over.max() <= 1.0


@pytest.mark.parametrize("dt", ["bf16", "fp8"])
def test_a_captured_batch_whose_plan_does_not_fit_the_arguments(dt):
    """Replayed between eager calls of another batch on the same workspace."""
    print(f"\n[case] captured diff batch {dt}", flush=True)
    cwlib.init()
    rng = np.random.default_rng(77)
    lp, ls = _lens(rng, 400, 12)
    calls = []
    for a, b in ((lp, ls), (lp[:60], ls[:60])):
        w = cw.materialize(cw.custom_spec(a.tolist(), b.tolist(), num_kv_heads=2, gqa_group=2, head_dim=64, page_size=16,
                                          kv_dtype=dt, seed=len(a)))
        dw = to_gpu(w)
        calls.append((dw, torch.empty(dw.q.shape[0], 2, 128, dtype=torch.bfloat16, device="cuda")))
    lam = torch.rand(2, generator=torch.Generator().manual_seed(1)).cuda()
    ws = torch.empty(max(cwlib.diff_workspace_bytes(c.spec.prefix_lens, c.spec.suffix_lens, 1, 2, 64, 16, dt) for c, _ in calls),
                     dtype=torch.uint8, device="cuda")

    def run(i):
        dw, out = calls[i]
        s = dw.spec
        return cwlib.diff_attention(dw.q, dw.k_new, dw.v_new, dw.k_pool, dw.v_pool, dw.block_table, s.prefix_lens,
                                    s.suffix_lens, 2, s.softmax_scale, lam, k_scale=dw.k_scale, v_scale=dw.v_scale, out=out,
                                    workspace=ws)

    before = cwlib.arg_plan_calls()
    want = run(0).clone()
    assert cwlib.arg_plan_calls() == before
    other = run(1).clone()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run(0)
    for rep in range(4):
        calls[0][1].fill_(float("nan"))
        again = run(1)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(again, other) and torch.equal(calls[0][1], want), rep

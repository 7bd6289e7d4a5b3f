"""Helpers of the tests of attention with shaped scores: inputs, calls, and the error bound.

Bound, per element, from the kernels' arithmetic.  Exponents (natural units), S = the row's largest
scale sum |q k|, B its largest |bias|, cap the cap:
  dx = 2^-16 S (dot products of up to 128 exact products in fp32: below 128 * 2^-24 of their sum of
       magnitudes, and the scale's and page scale's products) + 2^-20 cap (the header's figure) + 2^-21 (S + B
       + cap) (bias less running max, and the exponent: two or three fp32 roundings of numbers up to 2 log2e (S + B + cap))
Outputs: |d out| <= (2 u + 2 dx + e) mass + 2^-8 |out|, mass = sum w |v| / sum w, u the rounding of the
weights, in the numerator and in the sum: 2^-8 (chunks over bf16 pools), 2^-11 (fp16: over fp8 pools), 2^-11 for single
tokens (two bf16 or fp16); e = 2^-12 for exp2, sums of some thousand terms and merges, for chunks over fp8 pools
2^-10 more for the cached values (code x scale in fp16, scale rounded too).  Chunks over fp8 pools hold every
value in fp16, whose steps below 2^-14 are 2^-24: + 2^-25, half of one, however small the value (the weights sum
to 1; a window of one token returns a value of 2^-20 with just that error).
lse: u + dx + 2^-18 + 2^-22 |lse|."""
import numpy as np
import torch

import cw_workloads as cw
import oracle
import paper_2606_16824_amd as cwlib
from conftest import paged_inputs
from gpu_util import to_gpu


def inputs(lp, ls, hkv, g, d, page, dt, seed=3, sharp=3.0):
    """Queries larger by `sharp`, so that scores reach the caps."""
    w = cw.materialize(cw.custom_spec(lp, ls, num_kv_heads=hkv, gqa_group=g, head_dim=d, page_size=page, kv_dtype=dt, seed=seed))
    w.q.copy_((w.q.float() * sharp).to(torch.bfloat16))
    return w


def shape_of(w, cap=0.0, slopes=False, window=0, docs=0, full=None, seed=1, empty=False):
    """Options of a call. `docs`: documents per sequence; `empty`: some rows' documents begin behind them (and
    some begin before the sequence)."""
    s = w.spec
    rng = np.random.default_rng(seed)
    hq = s.num_kv_heads * s.gqa_group
    kw = dict(score_cap=cap, window=window)
    kw["slopes"] = np.exp2(rng.uniform(-6, 0, size=hq)).astype(np.float32) if slopes else None
    begins = []
    for lp, ls in zip(s.prefix_lens.tolist(), s.suffix_lens.tolist()):
        pos = lp + np.arange(ls)
        cuts = np.unique(np.concatenate([[0], rng.integers(0, lp + ls, size=max(0, docs - 1))])) if ls else np.zeros(1, dtype=int)
        begin = cuts[np.searchsorted(cuts, pos, side="right") - 1]
        if empty:
            kind = rng.integers(0, 5, size=ls)
            begin = np.where(kind == 0, pos + 1 + rng.integers(0, 200, size=ls), np.where(kind == 1, -7, begin))
        begins.append(begin)
    kw["key_begins"] = np.concatenate(begins).astype(np.int32) if docs or empty else None
    kw["full_lens"] = None if full is None else np.array([int(x) for x in full], dtype=np.int32)
    return kw


def call(dw, kw, **more):
    s = dw.spec
    dev = {k: torch.from_numpy(kw[k]).cuda() if kw[k] is not None else None for k in ("slopes", "key_begins")}
    return cwlib.shaped_attention(dw.q, dw.k_new, dw.v_new, dw.k_pool, dw.v_pool, dw.block_table, s.prefix_lens, s.suffix_lens,
                                  s.gqa_group, s.softmax_scale, k_scale=dw.k_scale, v_scale=dw.v_scale, **{**kw, **dev}, **more)


def reference(w, kw):
    return oracle.shaped_attention(paged_inputs(w), kw["score_cap"], kw["slopes"], kw["window"], kw["key_begins"], kw["full_lens"])


def bounds(w, kw, ref, lse, terms):
    single = np.repeat(w.spec.suffix_lens == 1, w.spec.suffix_lens)[:, None, None]
    fp8 = w.spec.kv_dtype == "fp8"
    cap, s, b = kw["score_cap"], terms["scores"], terms["bias"]
    dx = 2.0 ** -16 * s + 2.0 ** -20 * cap + 2.0 ** -21 * (s + b + cap)
    u = np.where(single, 2.0 ** -11, 2.0 ** -11 if fp8 else 2.0 ** -8)
    r = 2 * u + 2 * dx + 2.0 ** -12 + np.where(single, 0.0, 2.0 ** -10 if fp8 else 0.0)
    with np.errstate(invalid="ignore"):
        half = np.where(single, 0.0, 2.0 ** -25 if fp8 else 0.0)
        return r * terms["mass"] + half + 2.0 ** -8 * np.abs(ref) + 1e-38, (u + dx)[..., 0] + 2.0 ** -18 + 2.0 ** -22 * np.abs(lse)


def check(w, kw, what, dw=None, **more):
    dw = to_gpu(w) if dw is None else dw
    out = torch.full(dw.q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full(dw.q.shape[:2], float("nan"), device="cuda")
    assert call(dw, kw, out=out, lse=lse, **more) is out
    torch.cuda.synchronize()
    ref, ref_lse, terms = reference(w, kw)
    tol, tol_lse = bounds(w, kw, ref, ref_lse, terms)
    got, got_lse = out.cpu().double().numpy(), lse.cpu().double().numpy()
    assert np.isfinite(got).all(), what
    blind = np.isneginf(ref_lse)
    assert np.array_equal(np.isneginf(got_lse), blind), what
    assert not got[blind].any(), what
    over = np.abs(got - ref) / tol
    over_lse = np.where(blind, 0.0, np.abs(np.where(blind, 0.0, got_lse) - np.where(blind, 0.0, ref_lse)) / np.where(blind, 1.0, tol_lse))
    print(f"[{what}] worst {over.max():.3f}, lse {over_lse.max():.3f} of the tolerance, relative "
          f"{np.linalg.norm(got - ref) / max(np.linalg.norm(ref), 1e-30):.2e}, {int(blind.sum())} blind rows", flush=True)
    assert over.max() <= 1.0 and over_lse.max() <= 1.0, what
    return out, lse

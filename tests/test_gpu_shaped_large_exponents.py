"""shaped_attention with biases up to the documented 2^64 and with scores as far from 0: a running max cannot
then be held to one of its log2 units, and the weights must stay finite and not all vanish.

Exponents are held to dx = 2^-16 S + 2^-20 cap + 2^-21 (S + B + cap) (S the row's largest scale sum |q k|, B its largest
|bias|).  Where the largest exponent lies more than 2 dx + 40 above the next one, the weights of all other keys are below
e^-40 of its own, and the row returns that key's value:
  |d out| <= 2^-8 |v| (stored in bf16) + 2^-10 |v| (chunks over fp8 pools: code x scale in fp16, the scale rounded too;
             single tokens: weight and its product with the page's scale in fp16) + 2^-12 |v| (exp2 and sums)
             + 2^-25 (a value in fp16) + 2^-40 (the others: at most 1500 of magnitude below 2^5 at e^-40 = 2^-57)
  |d lse| <= u + dx + 2^-18 + 2^-22 |lse|, u the rounding of the weights, whose sum is taken after it: one weight that is
             off by a factor 1 + u moves the logarithm of their sum by ln(1 + u) <= u, 2^-8 (chunks over bf16 pools) or 2^-11
Other rows are some mean of their values: at most the largest of their sequence, up to its roundings."""
import numpy as np
import pytest
import torch

import paper_2606_16824_amd as cwlib
from conftest import paged_inputs
from gpu_util import to_gpu
from oracle.paged_attention import bf16_bits_to_f64, gather_sequence_kv
from shaped_util import call, inputs, shape_of

pytestmark = pytest.mark.gpu

LP, LS = [300, 0, 77, 500, 64, 1500], [1, 70, 1, 129, 64, 1]
DTS = [(64, "bf16"), (128, "bf16"), (64, "fp8"), (128, "fp8")]


def _reference(w, kw):
    """Per (new token, query head): lse, its bound, the largest visible |value|, whether one key rules, its value."""
    inp, s = paged_inputs(w), w.spec
    q = bf16_bits_to_f64(inp.q)
    total, hq, d = q.shape
    lse, bound, most, rules = (np.zeros((total, hq)) for _ in range(4))
    value = np.zeros((total, hq, d))
    u = np.where(np.repeat(s.suffix_lens == 1, s.suffix_lens) | (s.kv_dtype == "fp8"), 2.0 ** -11, 2.0 ** -8)
    cap, row = kw["score_cap"], 0
    for b, (lp, ls) in enumerate(zip(s.prefix_lens.tolist(), s.suffix_lens.tolist())):
        k, v = gather_sequence_kv(inp, b)
        key = np.arange(lp + ls)
        for p in range(lp, lp + ls):
            seen = key <= p
            if kw["full_lens"] is not None:
                seen |= key < kw["full_lens"][b]
            if kw["window"]:
                seen &= key > p - kw["window"]
            j = key[seen]
            for h in range(hq):
                kj, vj = k[j, h // s.gqa_group], v[j, h // s.gqa_group]
                x = s.softmax_scale * (kj @ q[row, h])
                size = s.softmax_scale * (np.abs(kj) @ np.abs(q[row, h])).max()
                x = cap * np.tanh(x / cap) if cap else x
                bias = np.zeros(len(j)) if kw["slopes"] is None else float(kw["slopes"][h]) * np.abs(p - j)
                x = x - bias
                dx = 2.0 ** -16 * size + 2.0 ** -20 * cap + 2.0 ** -21 * (size + np.abs(bias).max() + cap)
                top = int(np.argmax(x))
                second = np.delete(x, top).max() if len(j) > 1 else -np.inf
                lse[row, h] = x[top] + np.log(np.exp(x - x[top]).sum())
                bound[row, h] = u[row] + dx + 2.0 ** -18 + 2.0 ** -22 * abs(lse[row, h])
                most[row, h] = np.abs(vj).max()
                rules[row, h] = x[top] - second > 2 * dx + 40
                value[row, h] = vj[top]
            row += 1
    return lse, bound, most, rules > 0, value


def _check(w, kw, what, least):
    """`least`: the share of rows that one key must rule, so that the comparison is not empty."""
    lse, bound, most, rules, value = _reference(w, kw)
    assert rules.mean() >= least, what
    dw = to_gpu(w)
    for tiles in (0, 1, 3):  # whole key ranges, or pieces of so many tiles
        out = torch.full(dw.q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
        got_lse = torch.full(dw.q.shape[:2], float("nan"), device="cuda")
        cwlib.set_tuning(0, tiles)
        try:
            call(dw, kw, out=out, lse=got_lse)
        finally:
            cwlib.set_tuning(0, 0)
        torch.cuda.synchronize()
        got, got_lse = out.cpu().double().numpy(), got_lse.cpu().double().numpy()
        assert np.isfinite(got).all() and np.isfinite(got_lse).all(), (what, tiles)
        off = np.abs(got_lse - lse) / bound
        tol = (2.0 ** -8 + 2.0 ** -10 + 2.0 ** -12) * np.abs(value) + 2.0 ** -25 + 2.0 ** -40
        over = np.where(rules[..., None], np.abs(got - value) / tol, 0.0)
        print(f"[{what} tiles {tiles}] {rules.mean():.3f} ruled by a key: worst {over.max():.3f} of the tolerance, lse {off.max():.3f}", flush=True)
        assert over.max() <= 1.0 and off.max() <= 1.0, (what, tiles)
        assert (np.abs(got).max(-1) <= most * (1 + 2.0 ** -7) + 2.0 ** -24).all(), (what, tiles)


@pytest.mark.parametrize("power", [14, 20, 27, 40, 53])
@pytest.mark.parametrize("d,dt", DTS)
def test_biases_up_to_their_limit(d, dt, power):
    """Slopes of either sign, biases up to 1.9 * 2^power * 1500."""
    print(f"\n[case] shaped biases 2^{power} {d} {dt}", flush=True)
    w = inputs(LP, LS, 2, 4, d, 16, dt, seed=20)
    slopes = np.array([1.0, -1.0, 1.37, -1.61, 1.4, -1.03, 0.5, -0.71], dtype=np.float32) * np.float32(2.0 ** power)
    # (the last: keys on both sides, two of them equally far)
    for kw, least in ((shape_of(w), 0.99), (shape_of(w, window=200, cap=30.0), 0.99), (shape_of(w, full=[0, 51, 0, 600, 128, 0]), 0.9)):
        kw["slopes"] = slopes
        _check(w, kw, f"shaped biases 2^{power} {d} {dt} window {kw['window']}", least)


@pytest.mark.parametrize("power", [10, 24, 30, 44])
@pytest.mark.parametrize("d,dt", DTS)
def test_scores_far_from_zero(d, dt, power):
    """Scores of some 2^power: q and k (over fp8 pools the K scales) that much larger."""
    print(f"\n[case] shaped scores 2^{power} {d} {dt}", flush=True)
    w = inputs(LP, LS, 2, 4, d, 64, dt, seed=21)
    if dt == "fp8":  # (queries and new keys, which chunks hold in fp16, stay as they are)
        w.k_scale.mul_(2.0 ** power)
    else:
        for x in (w.k_pool, w.k_new):
            x.copy_((x.float() * 2.0 ** (power // 2)).to(torch.bfloat16))
        w.q.copy_((w.q.float() * 2.0 ** (power - power // 2)).to(torch.bfloat16))
    kw = shape_of(w, window=200)
    kw["slopes"] = np.array([1.0, -1.0] * 4, dtype=np.float32)
    for kw in (shape_of(w), kw):
        _check(w, kw, f"shaped scores 2^{power} {d} {dt} window {kw['window']}", 0.4)

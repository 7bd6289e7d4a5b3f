"""shaped_attention where the automatic plan cuts query tiles into unequal key ranges, under windows,
prefix masks, documents, caps and slopes: rows from all over the sequences against the oracle (the
bound: shaped_util)."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_16824_amd as cwlib
from conftest import paged_inputs
from gpu_util import to_gpu
from oracle.paged_attention import bf16_bits_to_f64, gather_sequence_kv
from shaped_util import bounds, call, check, inputs, shape_of

gpu = pytest.mark.gpu

LP, LS, HKV, G = [5000, 300, 70], [1290, 40, 1], 4, 16
TOTAL = sum(LS)


def _bytes(d, page, dt, kw):
    return cwlib.shaped_workspace_bytes(LP, LS, HKV, G, d, page, dt, window=kw["window"], full_lens=kw["full_lens"])


def _rows(w, kw, tokens):
    """oracle.shaped_attention's results of the new tokens `tokens` (ascending), a kv head's rows at a time."""
    inp, s = paged_inputs(w), w.spec
    q, g = bf16_bits_to_f64(inp.q), s.gqa_group
    out = np.zeros((len(tokens), q.shape[1], q.shape[2]))
    lse, terms = np.full(out.shape[:2], -np.inf), {"mass": np.zeros_like(out)}
    terms["scores"], terms["bias"] = np.zeros(out.shape[:2] + (1,)), np.zeros(out.shape[:2] + (1,))
    slopes = np.zeros(q.shape[1]) if kw["slopes"] is None else kw["slopes"].astype(np.float64)
    first = 0
    for b, (lp, ls) in enumerate(zip(s.prefix_lens.tolist(), s.suffix_lens.tolist())):
        at = np.flatnonzero((tokens >= first) & (tokens < first + ls))
        k, v = gather_sequence_kv(inp, b)
        p, j = (lp + tokens[at] - first)[:, None], np.arange(lp + ls)[None, :]
        seen = j <= p
        if kw["full_lens"] is not None:
            seen |= j < int(kw["full_lens"][b])
        if kw["window"]:
            seen &= j > p - kw["window"]
        if kw["key_begins"] is not None:
            seen &= j >= kw["key_begins"][tokens[at]].astype(np.int64)[:, None]
        for h in range(q.shape[1]):
            kh, vh, qh = k[:, h // g], v[:, h // g], q[tokens[at], h]
            x = s.softmax_scale * (qh @ kh.T)
            if kw["score_cap"]:
                x = kw["score_cap"] * np.tanh(x / kw["score_cap"])
            bias = slopes[h] * np.abs(p - j)
            x = np.where(seen, x - bias, -np.inf)
            top = x.max(1, keepdims=True)
            some = np.isfinite(top[:, 0])
            e = np.exp(x[some] - top[some])
            l = e.sum(1, keepdims=True)
            i = at[some]
            lse[i, h] = (top[some] + np.log(l))[:, 0]
            out[i, h], terms["mass"][i, h] = (e / l) @ vh, (e / l) @ np.abs(vh)
            terms["scores"][at, h, 0] = np.where(seen, s.softmax_scale * (np.abs(qh) @ np.abs(kh).T), 0.0).max(1)
            terms["bias"][at, h, 0] = np.where(seen, np.abs(bias), 0.0).max(1)
        first += ls
    return out, lse, terms


def _check(w, kw, got, got_lse, tokens, what):
    ref, ref_lse, terms = _rows(w, kw, tokens)
    # (of all rows, with the sampled ones' terms where they are)
    full = lambda x, fill: _spread(x, tokens, int(w.spec.suffix_lens.sum()), fill)
    blind = np.isneginf(ref_lse)
    tol, tol_lse = bounds(w, kw, full(ref, 0.0), full(np.where(blind, 0.0, ref_lse), 0.0), {n: full(x, 0.0) for n, x in terms.items()})
    tol, tol_lse, got, got_lse = tol[tokens], tol_lse[tokens], got.cpu().double().numpy()[tokens], got_lse.cpu().double().numpy()[tokens]
    assert np.array_equal(np.isneginf(got_lse), blind) and not got[blind].any(), what
    over = (np.abs(got - ref) / tol).max()
    over_lse = (np.abs(np.where(blind, 0.0, got_lse) - np.where(blind, 0.0, ref_lse)) / tol_lse).max()
    print(f"[{what}] worst {over:.3f}, lse {over_lse:.3f} of the tolerance, {len(tokens)} tokens, {int(blind.sum())} blind rows", flush=True)
    assert over <= 1.0 and over_lse <= 1.0, what


def _spread(x, tokens, total, fill):
    y = np.full((total,) + x.shape[1:], fill)
    y[tokens] = x
    return y


def test_rows_agree_with_the_oracle():
    """The row reference of this file on a small batch (no call is made)."""
    w = inputs([70, 5, 33], [20, 9, 1], 2, 3, 64, 16, "bf16", seed=3)
    for shape in (dict(), dict(cap=20.0, window=13), dict(docs=3, slopes=True, empty=True), dict(full=[80, 0, 20], slopes=True, window=40)):
        kw = shape_of(w, **shape)
        want = oracle.shaped_attention(paged_inputs(w), kw["score_cap"], kw["slopes"], kw["window"], kw["key_begins"], kw["full_lens"])
        tokens = np.array([0, 3, 19, 20, 28, 29])
        got = _rows(w, kw, tokens)
        for x, y in zip((got[0], got[1], got[2]["mass"], got[2]["scores"], got[2]["bias"]),
                        (want[0], want[1], want[2]["mass"], want[2]["scores"], want[2]["bias"])):
            assert np.allclose(x, y[tokens], rtol=1e-12, atol=1e-12)


@gpu
@pytest.mark.parametrize("d,page,dt,shape", [
    (64, 16, "bf16", dict(cap=20.0)),
    (128, 64, "fp8", dict(window=4000, slopes=True)),
    (128, 16, "bf16", dict(window=4500, slopes=True, full=[6000, 0, 60])),
    (64, 64, "fp8", dict(docs=3, cap=30.0)),
    (128, 64, "fp8", dict(full=[5600, 300, 0])),
    (128, 16, "bf16", dict(docs=4, empty=True)),
    (64, 16, "fp8", dict(window=4000, cap=20.0, slopes=True, full=[5200, 0, 0], docs=2)),
])
def test_cut_plan(d, page, dt, shape):
    print(f"\n[case] shaped cut plan {d} {page} {dt} {shape}", flush=True)
    w = inputs(LP, LS, HKV, G, d, page, dt, seed=31)
    kw = shape_of(w, seed=4, **shape)
    cwlib.init()
    # with a given number of workgroups the chunks' tiles are not levelled; then only the single token's keys
    # are cut, into 70 rows of partials at most per head
    automatic = _bytes(d, page, dt, kw)
    cwlib.set_tuning(1, 256)
    try:
        whole = _bytes(d, page, dt, kw)
    finally:
        cwlib.set_tuning(1, 0)
    assert whole < 1 << 20 and automatic >= whole + 256 * d * 4 * 32, "the chunks' plan was not cut"
    dw = to_gpu(w)
    out = torch.full(dw.q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full(dw.q.shape[:2], float("nan"), device="cuda")
    call(dw, kw, out=out, lse=lse)
    torch.cuda.synchronize()
    assert torch.isfinite(out.float()).all()
    # every fourth token (a tile has 16), and the ends of every eighth tile
    at = np.arange(TOTAL)
    tokens = np.flatnonzero((at % 4 == 1) | (at % 128 == 0) | (at % 128 == 15) | (at >= TOTAL - 2))
    _check(w, kw, out, lse, tokens, f"shaped cut plan {d} {dt} {shape}")


@gpu
@pytest.mark.parametrize("dt", ["bf16", "fp8"])
def test_a_cap_that_nothing_reaches(dt):
    print(f"\n[case] shaped cap out of reach {dt}", flush=True)
    w = inputs([500, 0, 40], [90, 130, 1], 2, 4, 128, 16, dt, seed=7, sharp=1.0)
    check(w, shape_of(w, cap=4096.0), f"shaped cap out of reach {dt}")

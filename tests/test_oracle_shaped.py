"""The oracle of shaped scores, position axes and the residual norms against torch and hand-worked cases."""
import numpy as np
import pytest
import torch

import cw_workloads as cw
import oracle
from conftest import paged_inputs


def _case(dt="bf16", lp=(37, 0, 20), ls=(9, 5, 1), hkv=2, g=3, seed=5):
    return paged_inputs(cw.materialize(cw.custom_spec(lp, ls, num_kv_heads=hkv, gqa_group=g, head_dim=64, page_size=16,
                                                      kv_dtype=dt, seed=seed)))


@pytest.mark.parametrize("dt", ["bf16", "fp8"])
@pytest.mark.parametrize("cap,sloped,window,docs,full", [
    (0.0, False, 0, False, False), (3.0, False, 0, False, False), (0.0, True, 0, False, False), (0.0, False, 6, False, False),
    (0.0, False, 0, True, False), (0.0, False, 0, False, True), (2.0, True, 9, True, True)])
def test_against_torch(dt, cap, sloped, window, docs, full):
    inp = _case(dt)
    cu, q = inp.cu(), torch.from_numpy(oracle.bf16_bits_to_f64(inp.q))
    total, hq = q.shape[:2]
    slopes = np.array([0.5, 0.25, 0.125, 0.0, 1.0, 0.03]) if sloped else None
    begins = np.array([0, 3, 38, 38, 40, 41, -5, 44, 45, 0, 1, 1, 9, 2, 20]) if docs else None  # (row 12 sees nothing)
    fulls = np.array([42, 99, 7]) if full else None
    out, lse, _ = oracle.shaped_attention(inp, cap, slopes, window, begins, fulls)
    for b in range(3):
        k, v = (torch.from_numpy(x) for x in oracle.gather_sequence_kv(inp, b))
        lp, ls = int(inp.prefix_lens[b]), int(inp.suffix_lens[b])
        p, j = torch.arange(lp, lp + ls)[:, None], torch.arange(lp + ls)[None, :]
        seen = torch.ones(ls, lp + ls).tril(lp).bool()
        if full:
            seen |= j < fulls[b]
        if window:
            seen &= p - j < window
        if docs:
            seen &= j >= torch.from_numpy(begins[cu[b]:cu[b] + ls])[:, None]
        for h in range(hq):
            s = q[cu[b]:cu[b] + ls, h] @ k[:, h // 3].T * inp.softmax_scale
            s = torch.tanh(s / cap) * cap if cap else s
            s = s - float(slopes[h]) * (p - j).abs().double() if sloped else s
            s = s.masked_fill(~seen, -torch.inf)
            want = torch.nan_to_num(torch.softmax(s, 1) @ v[:, h // 3])
            assert np.allclose(out[cu[b]:cu[b] + ls, h], want.numpy(), atol=1e-12)
            assert np.allclose(lse[cu[b]:cu[b] + ls, h], torch.logsumexp(s, 1).numpy(), atol=1e-12)


def test_plain_call_is_the_step_attention():
    inp = _case()
    out, lse, _ = oracle.shaped_attention(inp)
    want, want_lse = oracle.extend_attention_rowwise(inp)
    assert np.allclose(out, want, atol=1e-12) and np.allclose(lse, want_lse, atol=1e-12)


def test_a_window_of_one_returns_the_own_value():
    inp = _case()
    out, _, _ = oracle.shaped_attention(inp, window=1, cap=7.0)
    v = oracle.bf16_bits_to_f64(inp.v_new)
    assert np.allclose(out, np.repeat(v, 3, axis=1), atol=1e-13)


def test_a_large_cap_is_none_and_a_small_one_levels():
    inp = _case()
    plain = oracle.shaped_attention(inp)[0]
    assert np.allclose(oracle.shaped_attention(inp, cap=1e5)[0], plain, atol=1e-8)
    flat, _, _ = oracle.shaped_attention(inp, cap=1e-9)  # all scores nearly 0: the mean of the visible values
    k, v = oracle.gather_sequence_kv(inp, 1)
    assert np.allclose(flat[inp.cu()[1] + 4, 0], v[:5, 0].mean(axis=0), atol=1e-7)


def test_axes_by_hand():
    table = np.concatenate([np.cos(np.outer(np.arange(9), [1.0, 0.5])), np.sin(np.outer(np.arange(9), [1.0, 0.5]))], 1)
    cos, sin = oracle.axis_angles(table, np.array([[3, 0], [8, 2]]), [1, 0])
    assert np.allclose(cos, [[np.cos(8.0), np.cos(1.5)], [np.cos(2.0), 1.0]])
    assert np.allclose(sin, [[np.sin(8.0), np.sin(1.5)], [np.sin(2.0), 0.0]])


def test_residual_norm_matches_torch():
    rng = np.random.default_rng(2)
    x, r, g = rng.normal(size=(4, 40)), rng.normal(size=(4, 40)), rng.normal(size=40)
    a, b = rng.uniform(0.5, 1.5, size=40), rng.uniform(0.5, 1.5, size=40)
    res, y = oracle.residual_norm(x, r, a, g, 0.7, b, 1e-5)
    t = torch.nn.functional.rms_norm
    want = 0.7 * torch.from_numpy(r) + torch.from_numpy(g) * t(torch.from_numpy(x), (40,), torch.from_numpy(a), 1e-5)
    assert np.allclose(res, want.numpy(), atol=1e-13)
    assert np.allclose(y, t(want, (40,), torch.from_numpy(b), 1e-5).numpy(), atol=1e-13)
    res, y = oracle.residual_norm(x, r)
    assert np.allclose(res, x + r) and y is None

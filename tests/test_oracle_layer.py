"""The oracle of the layer operators against hand-worked cases and torch's own routines."""
import numpy as np
import pytest
import torch

import cw_workloads as cw
import oracle
from conftest import paged_inputs


def test_step_tables_by_hand():
    table = np.array([[7, 9, 99, 99], [99, 99, 99, 99], [3, 99, 99, 99]])
    # 20 cached + 15 new: pages 2 and 3 held, one new; nothing cached + 16 new: one; 5 + 0: none
    got = oracle.step_tables([20, 0, 5], [15, 16, 0], [40, 41, 42], table, 16, 33)
    assert got[0].tolist() == [[7, 9, 40, 99], [41, 99, 99, 99], [3, 99, 99, 99]]
    assert got[1].tolist() == [0, 15, 31, 31]
    assert got[2].tolist() == [0] * 15 + [1] * 16 + [-1, -1]
    assert got[3].tolist() == list(range(20, 35)) + list(range(16)) + [-1, -1]
    assert got[4][:15].tolist() == [9 * 16 + i for i in range(4, 16)] + [40 * 16 + i for i in range(3)]
    assert got[4][15:].tolist() == [41 * 16 + i for i in range(16)] + [-1, -1]
    assert got[5].tolist() == [2, 31, 0]


def test_step_tables_short_list_and_short_row():
    got = oracle.step_tables([0, 0], [16, 40], [5, 6], np.full((2, 2), 99), 16, 56)
    assert got[0].tolist() == [[5, 99], [6, -1]] and got[5].tolist() == [3, 56, 1]
    assert got[4][16:].tolist() == [6 * 16 + i for i in range(16)] + [-1] * 24


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_complex_product(interleaved):
    rng = np.random.default_rng(1)
    x, a = rng.normal(size=(5, 3, 64)), rng.uniform(0, 6, size=(5, 16))
    y = oracle.norm_rotate(x, None, 0.0, np.cos(a), np.sin(a), interleaved)
    z = x[..., 0:32:2] + 1j * x[..., 1:32:2] if interleaved else x[..., :16] + 1j * x[..., 16:32]
    w = y[..., 0:32:2] + 1j * y[..., 1:32:2] if interleaved else y[..., :16] + 1j * y[..., 16:32]
    assert np.allclose(w, z * np.exp(1j * a)[:, None, :], atol=1e-13)
    assert np.array_equal(y[..., 32:], x[..., 32:])


def test_norm_matches_torch():
    rng = np.random.default_rng(2)
    x, w = rng.normal(size=(4, 2, 64)), rng.uniform(0.5, 1.5, size=64)
    got = oracle.norm_rotate(x, w, 1e-5, np.ones((4, 8)), np.zeros((4, 8)), False)
    want = torch.nn.functional.rms_norm(torch.from_numpy(x), (64,), torch.from_numpy(w), 1e-5)
    assert np.allclose(got, want.numpy(), atol=1e-13)


@pytest.mark.parametrize("dt", ["bf16", "fp8"])
def test_diff_attention_matches_torch_sdpa(dt):
    spec = cw.custom_spec([37, 0, 20], [9, 5, 1], num_kv_heads=4, gqa_group=3, head_dim=64, page_size=16, kv_dtype=dt,
                          seed=5)
    inp = paged_inputs(cw.materialize(spec))
    lam = np.random.default_rng(3).uniform(-0.5, 0.9, size=6)
    out, terms = oracle.diff_attention(inp, lam)
    q = torch.from_numpy(oracle.bf16_bits_to_f64(inp.q))
    cu = inp.cu()
    for b in range(3):
        k, v = (torch.from_numpy(x) for x in oracle.gather_sequence_kv(inp, b))
        lp, ls = int(inp.prefix_lens[b]), int(inp.suffix_lens[b])
        see = torch.arange(lp + ls)[None, :] <= lp + torch.arange(ls)[:, None]
        for h in range(6):
            j = h // 3
            val = torch.cat([v[:, 2 * j], v[:, 2 * j + 1]], 1)
            o = [torch.nn.functional.scaled_dot_product_attention(q[cu[b]:cu[b] + ls, 2 * h + m][None], k[None, :, 2 * j + m],
                                                                  val[None], attn_mask=see, scale=inp.softmax_scale)[0]
                 for m in (0, 1)]
            assert np.allclose(out[cu[b]:cu[b] + ls, h], (o[0] - lam[h] * o[1]).numpy(), atol=1e-12)
    assert np.all(np.abs(terms["x"]) <= terms["mass"] + 1e-12)

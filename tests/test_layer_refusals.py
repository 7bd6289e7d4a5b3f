"""The layer operators' checks: the C entry points reject bad arguments before any GPU work
(addresses here are never dereferenced), the binding checks every tensor.  Runs without a GPU."""
import numpy as np
import pytest
import torch

import paper_2606_16824_amd as cwlib
from paper_2606_16824_amd import _lib as L

FAKE = 0x100000
BIG = 1 << 40


def lib():
    return cwlib.library()


def _spread(names, step=1 << 32):
    """A distinct, aligned, far-apart address for every name."""
    return {n: FAKE + step * i for i, n in enumerate(names)}


# ------------------------------------------------------------------ step tables


def _tables(**over):
    a = _spread(["lp", "ls", "free", "table", "cu", "seq", "pos", "slots", "info", "ws"])
    a.update(n=3, num_free=10, page=16, stride=4, tokens=20, wsb=0)
    a.update(over)
    return lib().cw_build_step_tables(a["lp"], a["ls"], a["n"], a["free"], a["num_free"], a["page"], a["table"], a["stride"],
                                      a["tokens"], a["cu"], a["seq"], a["pos"], a["slots"], a["info"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("over,status", [
    (dict(page=32), L.CW_ERR_UNSUPPORTED),
    (dict(page=0), L.CW_ERR_UNSUPPORTED),
    (dict(n=-1), L.CW_ERR_BAD_LENS),
    (dict(num_free=-1), L.CW_ERR_BAD_LENS),
    (dict(tokens=-1), L.CW_ERR_BAD_LENS),
    (dict(stride=0), L.CW_ERR_BAD_LENS),
    (dict(lp=None), L.CW_ERR_NULL),
    (dict(ls=None), L.CW_ERR_NULL),
    (dict(table=None), L.CW_ERR_NULL),
    (dict(free=None), L.CW_ERR_NULL),
    (dict(lp=FAKE + 2), L.CW_ERR_ALIGN),
    (dict(slots=FAKE + 4), L.CW_ERR_ALIGN),
    (dict(info=FAKE + 4), L.CW_ERR_ALIGN),
    (dict(n=5000), L.CW_ERR_WORKSPACE),
    (dict(n=5000, ws=None, wsb=1 << 20), L.CW_ERR_WORKSPACE),
    (dict(n=5000, ws=FAKE + 4, wsb=1 << 20), L.CW_ERR_ALIGN),
    (dict(seq=FAKE), L.CW_ERR_ALIAS),  # on prefix_lens
    (dict(pos=FAKE + (1 << 32) * 5 + 76), L.CW_ERR_ALIAS),  # the last entry of seq_ids
    (dict(table=FAKE + (1 << 32) * 2), L.CW_ERR_ALIAS),  # on the free list
])
def test_step_tables_rejects(over, status):
    assert _tables(**over) == status
    assert lib().cw_last_error_message().decode()


def test_step_tables_workspace():
    assert [cwlib.step_tables_workspace_bytes(n) for n in (-1, 0, 1, 4096)] == [0, 0, 0, 0]
    assert cwlib.step_tables_workspace_bytes(4097) >= 2 * 4098 * 4


# ------------------------------------------------------------------ norm and rotation


def _rope(**over):
    a = _spread(["q", "k", "v", "wq", "wk", "cs", "pos", "qo", "ko", "vo", "kp", "vp", "ks", "vs", "slots"])
    a.update(qs=1536, kst=1536, vst=1536, t=4, hq=8, hkv=2, d=128, eps=1e-6, np=100, rot=128, inter=0, pages=10, page=16, dt=0)
    a.update(over)
    return lib().cw_qk_norm_rope(a["q"], a["qs"], a["k"], a["kst"], a["v"], a["vst"], a["t"], a["hq"], a["hkv"], a["d"], a["wq"],
                                 a["wk"], a["eps"], a["cs"], a["np"], a["rot"], a["inter"], a["pos"], a["qo"], a["ko"], a["vo"],
                                 a["kp"], a["vp"], a["ks"], a["vs"], a["slots"], a["pages"], a["page"], a["dt"], None)


@pytest.mark.parametrize("over,status", [
    (dict(d=96), L.CW_ERR_UNSUPPORTED),
    (dict(page=32), L.CW_ERR_UNSUPPORTED),
    (dict(hkv=0), L.CW_ERR_UNSUPPORTED),
    (dict(hq=0), L.CW_ERR_UNSUPPORTED),
    (dict(rot=8), L.CW_ERR_UNSUPPORTED),
    (dict(rot=24), L.CW_ERR_UNSUPPORTED),
    (dict(rot=144), L.CW_ERR_UNSUPPORTED),
    (dict(rot=0), L.CW_ERR_UNSUPPORTED),
    (dict(eps=-1.0), L.CW_ERR_UNSUPPORTED),
    (dict(eps=float("nan")), L.CW_ERR_UNSUPPORTED),
    (dict(dt=5), L.CW_ERR_UNSUPPORTED),
    (dict(dt=1, ks=None), L.CW_ERR_NULL),
    (dict(t=-1), L.CW_ERR_BAD_LENS),
    (dict(np=-1), L.CW_ERR_BAD_LENS),
    (dict(pages=-1), L.CW_ERR_BAD_LENS),
    (dict(q=None), L.CW_ERR_NULL),
    (dict(k=None), L.CW_ERR_NULL),
    (dict(cs=None), L.CW_ERR_NULL),
    (dict(pos=None), L.CW_ERR_NULL),
    (dict(qo=None), L.CW_ERR_NULL),
    (dict(ko=None), L.CW_ERR_NULL),
    (dict(vp=None), L.CW_ERR_NULL),
    (dict(kp=None), L.CW_ERR_NULL),
    (dict(slots=None), L.CW_ERR_NULL),
    (dict(v=None), L.CW_ERR_NULL),
    (dict(v=None, kp=None, vp=None), L.CW_ERR_NULL),  # v_out without v
    (dict(qs=1532), L.CW_ERR_ALIGN),
    (dict(qs=1016), L.CW_ERR_ALIGN),  # less than a token's heads
    (dict(kst=-1536), L.CW_ERR_ALIGN),
    (dict(q=FAKE + 8), L.CW_ERR_ALIGN),
    (dict(cs=FAKE + 8 + (5 << 32)), L.CW_ERR_ALIGN),
    (dict(pos=FAKE + 2 + (6 << 32)), L.CW_ERR_ALIGN),
    (dict(slots=FAKE + 4 + (14 << 32)), L.CW_ERR_ALIGN),
    (dict(qo=FAKE), L.CW_ERR_ALIAS),  # q of another stride
    (dict(qo=FAKE + 16, qs=1024), L.CW_ERR_ALIAS),
    (dict(ko=FAKE + (7 << 32)), L.CW_ERR_ALIAS),  # on q_out
    (dict(vo=FAKE + (1 << 32), kst=256, vst=256), L.CW_ERR_ALIAS),  # v_out is k
    (dict(vp=FAKE + (10 << 32)), L.CW_ERR_ALIAS),  # both pools the same
    (dict(kp=FAKE + (6 << 32)), L.CW_ERR_ALIAS),  # on positions
])
def test_norm_rope_rejects(over, status):
    assert _rope(**over) == status
    assert lib().cw_last_error_message().decode()


def test_norm_rope_without_tokens_is_a_no_op():
    assert _rope(t=0, q=None, qo=None) == L.CW_OK


# ------------------------------------------------------------------ differential attention


def _diff(**over):
    lp = np.array(over.pop("lp", [10, 20]), dtype=np.int32)
    ls = np.array(over.pop("ls", [5, 1]), dtype=np.int32)
    a = _spread(["q", "kn", "vn", "kp", "vp", "ks", "vs", "bt", "lam", "w", "out", "ws"])
    a.update(stride=4, pages=100, pairs=2, g=4, d=128, page=16, scale=0.1, dt=0, eps=1e-5, after=0.5, wsb=BIG)
    a.update(over)
    return lib().cw_diff_attention(a["q"], a["kn"], a["vn"], a["kp"], a["vp"], a["ks"], a["vs"], a["bt"], a["stride"], a["pages"],
                                   lp.ctypes.data, ls.ctypes.data, len(lp), a["pairs"], a["g"], a["d"], a["page"], a["scale"],
                                   a["dt"], a["lam"], a["w"], a["eps"], a["after"], a["out"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("over,status", [
    (dict(pairs=0), L.CW_ERR_UNSUPPORTED),
    (dict(pairs=513), L.CW_ERR_UNSUPPORTED),
    (dict(g=0), L.CW_ERR_UNSUPPORTED),
    (dict(g=17), L.CW_ERR_UNSUPPORTED),
    (dict(d=32), L.CW_ERR_UNSUPPORTED),
    (dict(page=8), L.CW_ERR_UNSUPPORTED),
    (dict(dt=9), L.CW_ERR_UNSUPPORTED),
    (dict(scale=0.0), L.CW_ERR_UNSUPPORTED),
    (dict(scale=float("inf")), L.CW_ERR_UNSUPPORTED),
    (dict(after=float("nan")), L.CW_ERR_UNSUPPORTED),
    (dict(eps=-1.0), L.CW_ERR_UNSUPPORTED),
    (dict(dt=1, vs=None), L.CW_ERR_NULL),
    (dict(q=None), L.CW_ERR_NULL),
    (dict(lam=None), L.CW_ERR_NULL),
    (dict(out=None), L.CW_ERR_NULL),
    (dict(bt=None), L.CW_ERR_NULL),
    (dict(kp=None), L.CW_ERR_NULL),
    (dict(lp=[-1, 0]), L.CW_ERR_BAD_LENS),
    (dict(ls=[1, -1]), L.CW_ERR_BAD_LENS),
    (dict(lp=[64, 0]), L.CW_ERR_BAD_LENS),
    (dict(pages=-1), L.CW_ERR_BAD_LENS),
    (dict(q=FAKE + 8), L.CW_ERR_ALIGN),
    (dict(w=FAKE + 4), L.CW_ERR_ALIGN),
    (dict(lam=FAKE + 2), L.CW_ERR_ALIGN),
    (dict(wsb=16), L.CW_ERR_WORKSPACE),
    (dict(ws=None), L.CW_ERR_WORKSPACE),
    (dict(out=FAKE), L.CW_ERR_ALIAS),
    (dict(out=FAKE + (8 << 32)), L.CW_ERR_ALIAS),
    (dict(out=FAKE + (9 << 32)), L.CW_ERR_ALIAS),
    (dict(out=FAKE + (11 << 32)), L.CW_ERR_ALIAS),
])
def test_diff_rejects(over, status):
    assert _diff(**over) == status
    assert lib().cw_last_error_message().decode()


def test_diff_without_rows_is_a_no_op_and_needs_no_pools_without_a_prefix():
    assert _diff(ls=[0, 0], q=None, out=None) == L.CW_OK
    assert _diff(lp=[0, 0], kp=None, vp=None, wsb=1) == L.CW_ERR_WORKSPACE
    assert _diff(lp=[0, 9], ls=[3, 0], kp=None, vp=None, wsb=1) == L.CW_ERR_WORKSPACE  # no row reads the prefix


def test_diff_workspace_query():
    lens = ([5, 300], [1, 40])
    assert cwlib.diff_workspace_bytes(*lens, 2, 4, 128, 16) > 0
    assert cwlib.diff_workspace_bytes(*lens, 2, 4, 96, 16) == 0
    assert cwlib.diff_workspace_bytes(*lens, 2, 17, 128, 16) == 0
    assert cwlib.diff_workspace_bytes(*lens, 2, 4, 128, 24) == 0
    assert cwlib.diff_workspace_bytes([5, -1], [1, 1], 2, 4, 128, 16) == 0
    assert cwlib.diff_workspace_bytes([], [], 2, 4, 128, 16) > 0


# ------------------------------------------------------------------ the binding (CPU tensors: the last check is the device's)

BF, I32, I64, F32 = torch.bfloat16, torch.int32, torch.int64, torch.float32


def _tables_args():
    return dict(prefix_lens=torch.zeros(3, dtype=I32), suffix_lens=torch.zeros(3, dtype=I32), free_pages=torch.zeros(9, dtype=I32),
                block_table=torch.zeros(4, 8, dtype=I32), page_size=16, max_tokens=7, cu_rows=torch.zeros(4, dtype=I32),
                seq_ids=torch.zeros(7, dtype=I32), positions=torch.zeros(7, dtype=I32), slots=torch.zeros(7, dtype=I64),
                info=torch.zeros(3, dtype=I64))


@pytest.mark.parametrize("name,bad,msg", [
    (None, None, "on the GPU"),
    ("prefix_lens", torch.zeros(3, dtype=I64), "prefix_lens has dtype"),
    ("suffix_lens", torch.zeros(2, dtype=I32), "suffix_lens has shape"),
    ("free_pages", torch.zeros(9, 1, dtype=I32), "free_pages must be"),
    ("block_table", torch.zeros(2, 8, dtype=I32), "rows for 3 sequences"),
    ("block_table", torch.zeros(4, 8), "block_table must be"),
    ("max_tokens", -1, "negative"),
    ("cu_rows", torch.zeros(3, dtype=I32), "cu_rows has shape"),
    ("seq_ids", torch.zeros(6, dtype=I32), "seq_ids has shape"),
    ("positions", torch.zeros(7, dtype=I64), "positions has dtype"),
    ("slots", torch.zeros(7, dtype=I32), "slots has dtype"),
    ("info", torch.zeros(2, dtype=I64), "info has shape"),
    ("prefix_lens", [1, 2, 3], "prefix_lens must be"),
])
def test_tables_binding(name, bad, msg, monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    a = _tables_args()
    if name:
        a[name] = bad
    with pytest.raises(ValueError, match=msg):
        cwlib.build_step_tables(**a)


def _rope_args(pool=BF):
    t, hq, hkv, d = 5, 4, 2, 64
    a = dict(q=torch.zeros(t, hq, d, dtype=BF), k=torch.zeros(t, hkv, d, dtype=BF), cos_sin=torch.zeros(10, 64),
             positions=torch.zeros(t, dtype=I32), q_weight=torch.zeros(d), k_weight=torch.zeros(d), v=torch.zeros(t, hkv, d, dtype=BF),
             k_pool=torch.zeros(3, hkv, 16, d, dtype=pool), v_pool=torch.zeros(3, hkv, 16, d, dtype=pool),
             slots=torch.zeros(t, dtype=I64), q_out=torch.zeros(t, hq, d, dtype=BF), k_out=torch.zeros(t, hkv, d, dtype=BF),
             v_out=torch.zeros(t, hkv, d, dtype=BF))
    if pool is not BF:
        a.update(k_scale=torch.ones(3, hkv), v_scale=torch.ones(3, hkv))
    return a


@pytest.mark.parametrize("name,bad,msg", [
    (None, None, "on the GPU"),
    ("q", torch.zeros(5, 4, 64), "q has dtype"),
    ("q", torch.zeros(5, 256, dtype=BF), "3-D"),
    ("k", torch.zeros(4, 2, 64, dtype=BF), "k has shape"),
    ("v", torch.zeros(5, 2, 64), "v has dtype"),
    ("v", None, "needs k_pool, v_pool, slots and v"),
    ("cos_sin", torch.zeros(10), "cos_sin must be"),
    ("positions", torch.zeros(4, dtype=I32), "positions has shape"),
    ("q_weight", torch.zeros(32), "q_weight has shape"),
    ("k_weight", torch.zeros(64, dtype=BF), "k_weight has dtype"),
    ("v_pool", None, "needs k_pool"),
    ("slots", None, "needs k_pool"),
    ("slots", torch.zeros(5, dtype=I32), "slots has dtype"),
    ("k_pool", torch.zeros(3, 1, 16, 64, dtype=BF), "v_pool has shape"),
    ("k_scale", torch.ones(3, 2), "fp8 pools only"),
    ("q_out", torch.zeros(5, 2, 64, dtype=BF), "q_out has shape"),
    ("v_out", torch.zeros(5, 2, 64), "v_out has dtype"),
])
def test_rope_binding(name, bad, msg, monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    a = _rope_args()
    # tensors on the CPU pass every check of shape and type, and stop at the device's
    monkeypatch.setattr(cwlib, "_head_rows", lambda t, n, total, heads, d: cwlib._want(t, n, (BF,), (total, heads, d)))
    if name:
        a[name] = bad
    with pytest.raises(ValueError, match=msg):
        cwlib.qk_norm_rope(**a)


def test_rope_binding_fp8_and_leftovers(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(cwlib, "_head_rows", lambda t, n, total, heads, d: cwlib._want(t, n, (BF,), (total, heads, d)))
    a = _rope_args(torch.uint8)
    a["k_scale"] = None
    with pytest.raises(ValueError, match="needs k_scale"):
        cwlib.qk_norm_rope(**a)
    a = _rope_args()
    a["k_pool"] = a["v_pool"] = None
    with pytest.raises(ValueError, match="for a page write"):
        cwlib.qk_norm_rope(**a)
    a = _rope_args()
    a.update(v=None, k_pool=None, v_pool=None, slots=None)
    with pytest.raises(ValueError, match="v_out without v"):
        cwlib.qk_norm_rope(**a)


def _diff_args():
    t, pairs, g, d = 6, 2, 3, 64
    return dict(q=torch.zeros(t, 2 * pairs * g, d, dtype=BF), k_new=torch.zeros(t, 2 * pairs, d, dtype=BF),
                v_new=torch.zeros(t, 2 * pairs, d, dtype=BF), k_pool=torch.zeros(8, 2 * pairs, 16, d, dtype=BF),
                v_pool=torch.zeros(8, 2 * pairs, 16, d, dtype=BF), block_table=torch.zeros(2, 4, dtype=I32), prefix_lens=[20, 0],
                suffix_lens=[5, 1], gqa_group=g, softmax_scale=0.1, lam=torch.zeros(pairs * g), norm_weight=torch.zeros(2 * d),
                out=torch.zeros(t, pairs * g, 2 * d, dtype=BF))


@pytest.mark.parametrize("name,bad,msg", [
    (None, None, "on the GPU"),
    ("q", torch.zeros(6, 6, 64, dtype=BF), "q has shape"),
    ("k_new", torch.zeros(6, 2, 64, dtype=BF), "k_new has shape"),
    ("v_pool", torch.zeros(8, 4, 16, 64), "v_pool has dtype"),
    ("lam", torch.zeros(12), "lam has shape"),
    ("lam", torch.zeros(6, dtype=BF), "lam has dtype"),
    ("norm_weight", torch.zeros(64), "norm_weight has shape"),
    ("out", torch.zeros(6, 6, 64, dtype=BF), "out has shape"),
    ("suffix_lens", [5], "1-D of one length"),
])
def test_diff_binding(name, bad, msg, monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    a = _diff_args()
    if name:
        a[name] = bad
    with pytest.raises(ValueError, match=msg):
        cwlib.diff_attention(**a)


def test_diff_binding_wants_pairs_of_heads(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    a = _diff_args()
    for n in ("k_new", "v_new"):
        a[n] = a[n][:, :3].contiguous()
    for n in ("k_pool", "v_pool"):
        a[n] = a[n][:, :3].contiguous()
    a["q"] = torch.zeros(6, 9, 64, dtype=BF)
    with pytest.raises(ValueError, match="pairs of them"):
        cwlib.diff_attention(**a)

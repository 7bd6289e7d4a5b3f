"""What shaped_attention, qk_norm_rope_axes and residual_norm refuse, before any GPU work (addresses here are never
dereferenced), and the checks of their binding.  Runs without a GPU."""
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2606_16824_amd as cwlib
from conftest import ROOT
from paper_2606_16824_amd import _lib as L

FAKE = 0x100000
BIG = 1 << 40
BF, I32, I64 = torch.bfloat16, torch.int32, torch.int64


def lib():
    return cwlib.library()


def _spread(names, step=1 << 32):
    return {n: FAKE + step * i for i, n in enumerate(names)}


# ------------------------------------------------------------------ attention


def _shaped(**over):
    lp = np.array(over.pop("lp", [10, 20]), dtype=np.int32)
    ls = np.array(over.pop("ls", [5, 1]), dtype=np.int32)
    full = over.pop("full", [3, 0])
    full = None if full is None else np.array(full, dtype=np.int32)
    a = _spread(["q", "kn", "vn", "kp", "vp", "ks", "vs", "bt", "slopes", "begins", "out", "lse", "ws"])
    a.update(stride=4, pages=100, hkv=2, g=4, d=128, page=16, scale=0.1, dt=0, cap=50.0, window=9, wsb=BIG)
    a.update(over)
    return lib().cw_shaped_attention(a["q"], a["kn"], a["vn"], a["kp"], a["vp"], a["ks"], a["vs"], a["bt"], a["stride"], a["pages"],
                                     lp.ctypes.data, ls.ctypes.data, len(lp), a["hkv"], a["g"], a["d"], a["page"], a["scale"],
                                     a["dt"], a["cap"], a["slopes"], a["window"], a["begins"],
                                     None if full is None else full.ctypes.data, a["out"], a["lse"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("over,status", [
    (dict(hkv=0), L.CW_ERR_UNSUPPORTED),
    (dict(hkv=1025), L.CW_ERR_UNSUPPORTED),
    (dict(g=0), L.CW_ERR_UNSUPPORTED),
    (dict(g=17), L.CW_ERR_UNSUPPORTED),
    (dict(d=32), L.CW_ERR_UNSUPPORTED),
    (dict(page=8), L.CW_ERR_UNSUPPORTED),
    (dict(dt=9), L.CW_ERR_UNSUPPORTED),
    (dict(scale=0.0), L.CW_ERR_UNSUPPORTED),
    (dict(scale=float("inf")), L.CW_ERR_UNSUPPORTED),
    (dict(scale=3e38, cap=2.0 ** -10), L.CW_ERR_UNSUPPORTED),  # their quotient is no fp32 number
    (dict(cap=-1.0), L.CW_ERR_UNSUPPORTED),
    (dict(cap=2.0 ** -11), L.CW_ERR_UNSUPPORTED),
    (dict(cap=5000.0), L.CW_ERR_UNSUPPORTED),
    (dict(cap=float("nan")), L.CW_ERR_UNSUPPORTED),
    (dict(cap=float("inf")), L.CW_ERR_UNSUPPORTED),
    (dict(window=-1), L.CW_ERR_BAD_LENS),
    (dict(full=[0, -1]), L.CW_ERR_BAD_LENS),
    (dict(dt=1, vs=None), L.CW_ERR_NULL),
    (dict(q=None), L.CW_ERR_NULL),
    (dict(kn=None), L.CW_ERR_NULL),
    (dict(vn=None), L.CW_ERR_NULL),
    (dict(out=None), L.CW_ERR_NULL),
    (dict(bt=None), L.CW_ERR_NULL),
    (dict(kp=None), L.CW_ERR_NULL),
    (dict(lp=[-1, 0]), L.CW_ERR_BAD_LENS),
    (dict(ls=[1, -1]), L.CW_ERR_BAD_LENS),
    (dict(lp=[64, 0]), L.CW_ERR_BAD_LENS),
    (dict(pages=-1), L.CW_ERR_BAD_LENS),
    (dict(q=FAKE + 8), L.CW_ERR_ALIGN),
    (dict(ws=FAKE + 8 + (12 << 32)), L.CW_ERR_ALIGN),
    (dict(slopes=FAKE + 2 + (8 << 32)), L.CW_ERR_ALIGN),
    (dict(begins=FAKE + 2 + (9 << 32)), L.CW_ERR_ALIGN),
    (dict(lse=FAKE + 2 + (11 << 32)), L.CW_ERR_ALIGN),
    (dict(wsb=16), L.CW_ERR_WORKSPACE),
    (dict(ws=None), L.CW_ERR_WORKSPACE),
    (dict(out=FAKE), L.CW_ERR_ALIAS),
    (dict(out=FAKE + (8 << 32)), L.CW_ERR_ALIAS),
    (dict(lse=FAKE + (9 << 32)), L.CW_ERR_ALIAS),
    (dict(lse=FAKE + (10 << 32)), L.CW_ERR_ALIAS),
    (dict(ws=FAKE + (9 << 32)), L.CW_ERR_ALIAS),  # the plan would be written over key_begins
])
def test_shaped_rejects(over, status):
    assert _shaped(**over) == status
    assert lib().cw_last_error_message().decode()


def test_shaped_without_rows_is_a_no_op_and_options_may_be_left_out():
    assert _shaped(ls=[0, 0], q=None, out=None) == L.CW_OK
    assert _shaped(slopes=None, begins=None, lse=None, full=None, cap=0.0, window=0, wsb=1) == L.CW_ERR_WORKSPACE  # all else passed
    assert _shaped(window=(1 << 31) - 1, full=[(1 << 31) - 1, 0], cap=4096.0, wsb=1) == L.CW_ERR_WORKSPACE
    assert _shaped(lp=[0, 9], ls=[3, 0], kp=None, vp=None, wsb=1) == L.CW_ERR_WORKSPACE  # no row reads the prefix


def test_shaped_workspace_query():
    q = cwlib.shaped_workspace_bytes
    assert q([5, 300], [1, 40], 2, 4, 128, 16) > 0
    for bad in ((2, 4, 96, 16), (2, 17, 128, 16), (2, 4, 128, 24)):
        assert q([5, 300], [1, 40], *bad) == 0
    assert q([5, -1], [1, 1], 2, 4, 128, 16) == 0
    assert q([5, 1], [1, 1], 2, 4, 128, 16, full_lens=[0, -4]) == 0
    assert q([], [], 2, 4, 128, 16) > 0
    # a window leaves fewer keys, so fewer partials
    assert q([60000] * 4, [1] * 4, 8, 4, 128, 16, window=1000) < q([60000] * 4, [1] * 4, 8, 4, 128, 16)
    for window in (-1, 1 << 31):
        with pytest.raises(ValueError, match="window"):
            q([5], [1], 2, 4, 128, 16, window=window)
    with pytest.raises(ValueError, match="full_lens has shape"):
        q([5], [1], 2, 4, 128, 16, full_lens=[1, 2])


# ------------------------------------------------------------------ norm and rotation by axes


def _rope(**over):
    axis_of = over.pop("axis_of", [0] * 24 + [1] * 20 + [2] * 20)
    axis_of = None if axis_of is None else np.array(axis_of, dtype=np.int32)
    a = _spread(["q", "k", "v", "wq", "wk", "cs", "pos", "qo", "ko", "vo", "kp", "vp", "ks", "vs", "slots"])
    a.update(qs=1536, kst=1536, vst=1536, t=4, hq=8, hkv=2, d=128, eps=1e-6, np=100, rot=128, inter=0, axes=3, pages=10, page=16, dt=0)
    a.update(over)
    return lib().cw_qk_norm_rope_axes(a["q"], a["qs"], a["k"], a["kst"], a["v"], a["vst"], a["t"], a["hq"], a["hkv"], a["d"],
                                      a["wq"], a["wk"], a["eps"], a["cs"], a["np"], a["rot"], a["inter"], a["pos"], a["axes"],
                                      None if axis_of is None else axis_of.ctypes.data, a["qo"], a["ko"], a["vo"], a["kp"],
                                      a["vp"], a["ks"], a["vs"], a["slots"], a["pages"], a["page"], a["dt"], None)


@pytest.mark.parametrize("over,status", [
    (dict(axes=0), L.CW_ERR_UNSUPPORTED),
    (dict(axes=-3), L.CW_ERR_UNSUPPORTED),
    (dict(axes=5), L.CW_ERR_UNSUPPORTED),
    (dict(axes=2), L.CW_ERR_UNSUPPORTED),  # pairs follow a third
    (dict(axis_of=[0] * 63 + [-1]), L.CW_ERR_UNSUPPORTED),
    (dict(axis_of=None), L.CW_ERR_NULL),
    (dict(d=96), L.CW_ERR_UNSUPPORTED),
    (dict(rot=24), L.CW_ERR_UNSUPPORTED),
    (dict(eps=-1.0), L.CW_ERR_UNSUPPORTED),
    (dict(t=-1), L.CW_ERR_BAD_LENS),
    (dict(q=None), L.CW_ERR_NULL),
    (dict(pos=None), L.CW_ERR_NULL),
    (dict(v=None), L.CW_ERR_NULL),
    (dict(qs=1004), L.CW_ERR_ALIGN),
    (dict(pos=FAKE + 2 + (6 << 32)), L.CW_ERR_ALIGN),
    (dict(qo=FAKE), L.CW_ERR_ALIAS),
    (dict(ko=FAKE + (6 << 32) + 32), L.CW_ERR_ALIAS),  # on the positions of the third axis
])
def test_axes_rejects(over, status):
    assert _rope(**over) == status
    assert lib().cw_last_error_message().decode()


def test_axes_without_tokens_is_a_no_op():
    assert _rope(t=0, q=None, pos=None) == L.CW_OK


# ------------------------------------------------------------------ residual


def _resid(**over):
    a = _spread(["x", "r", "post", "gate", "pre", "ro", "y"])
    a.update(xs=128, wide=0, t=4, n=128, gs=128, s=1.0, eps=1e-6)
    a.update(over)
    return lib().cw_residual_norm(a["x"], a["xs"], a["r"], a["wide"], a["t"], a["n"], a["post"], a["gate"], a["gs"], a["s"],
                                  a["pre"], a["eps"], a["ro"], a["y"], None)


@pytest.mark.parametrize("over,status", [
    (dict(n=0), L.CW_ERR_UNSUPPORTED),
    (dict(n=132), L.CW_ERR_UNSUPPORTED),
    (dict(n=16392, xs=16392, gs=16392), L.CW_ERR_UNSUPPORTED),
    (dict(eps=-1.0), L.CW_ERR_UNSUPPORTED),
    (dict(eps=float("nan")), L.CW_ERR_UNSUPPORTED),
    (dict(s=float("inf")), L.CW_ERR_UNSUPPORTED),
    (dict(t=-1), L.CW_ERR_BAD_LENS),
    (dict(t=1 << 30), L.CW_ERR_BAD_LENS),
    (dict(x=None), L.CW_ERR_NULL),
    (dict(r=None), L.CW_ERR_NULL),
    (dict(ro=None), L.CW_ERR_NULL),
    (dict(y=None), L.CW_ERR_NULL),
    (dict(pre=None), L.CW_ERR_NULL),
    (dict(xs=120), L.CW_ERR_ALIGN),
    (dict(xs=132), L.CW_ERR_ALIGN),
    (dict(xs=-128), L.CW_ERR_ALIGN),
    (dict(gs=64), L.CW_ERR_ALIGN),
    (dict(gate=FAKE + 8 + (3 << 32)), L.CW_ERR_ALIGN),
    (dict(post=FAKE + 4 + (2 << 32)), L.CW_ERR_ALIGN),
    (dict(ro=FAKE + (1 << 32) + 16), L.CW_ERR_ALIAS),  # shifted against the residual
    (dict(ro=FAKE), L.CW_ERR_ALIAS),
    (dict(y=FAKE), L.CW_ERR_ALIAS),
    (dict(y=FAKE + (1 << 32) + 512), L.CW_ERR_ALIAS),  # on the residual
    (dict(y=FAKE + (1 << 32), ro=FAKE + (1 << 32)), L.CW_ERR_ALIAS),
    (dict(y=FAKE + (3 << 32) + 1008), L.CW_ERR_ALIAS),  # the last token's gate
    (dict(ro=FAKE + (1 << 32) + 1024, wide=1), L.CW_ERR_ALIAS),
])
def test_residual_rejects(over, status):
    assert _resid(**over) == status
    assert lib().cw_last_error_message().decode()


def test_residual_without_tokens_is_a_no_op():
    assert _resid(t=0, x=None, r=None, ro=None, y=None) == L.CW_OK


# ------------------------------------------------------------------ the binding (CPU tensors: the last check is the device's)


def _shaped_args(pool=BF):
    t, hkv, g, d = 9, 2, 4, 64
    z = lambda *s: torch.zeros(*s, dtype=BF)
    a = dict(q=z(t, hkv * g, d), k_new=z(t, hkv, d), v_new=z(t, hkv, d), k_pool=torch.zeros(16, hkv, 16, d, dtype=pool),
             v_pool=torch.zeros(16, hkv, 16, d, dtype=pool), block_table=torch.zeros(3, 8, dtype=I32), prefix_lens=[40, 0, 17],
             suffix_lens=[5, 3, 1], gqa_group=g, softmax_scale=0.1, slopes=torch.zeros(hkv * g), key_begins=torch.zeros(t, dtype=I32),
             full_lens=[1, 2, 3], out=z(t, hkv * g, d), lse=torch.zeros(t, hkv * g), workspace=torch.zeros(1 << 20, dtype=torch.uint8))
    if pool is not BF:
        a.update(k_scale=torch.ones(16, hkv), v_scale=torch.ones(16, hkv))
    return a


@pytest.mark.parametrize("name,bad,msg", [
    (None, None, "on the GPU"),
    ("q", torch.zeros(9, 8, 64), "q has dtype"),
    ("out", torch.zeros(9, 4, 64, dtype=BF), "out has shape"),
    ("lse", torch.zeros(9, 8, dtype=torch.float64), "lse has dtype"),
    ("k_pool", torch.zeros(16, 2, 16, 64), "unsupported pool dtype"),
    ("block_table", torch.zeros(2, 8, dtype=I32), "rows for 3"),
    ("slopes", torch.zeros(4), "slopes has shape"),
    ("slopes", torch.zeros(8, dtype=BF), "slopes has dtype"),
    ("slopes", [1.0] * 8, "must be a torch.Tensor"),
    ("key_begins", torch.zeros(9, dtype=I64), "key_begins has dtype"),
    ("key_begins", torch.zeros(8, dtype=I32), "key_begins has shape"),
    ("full_lens", [1, 2], "full_lens has shape"),
    ("window", -3, "on the GPU|window"),
])
def test_shaped_binding(name, bad, msg, monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    a = _shaped_args()
    if name is not None:
        a[name] = bad
    with pytest.raises(ValueError, match=msg):
        cwlib.shaped_attention(**a)


@pytest.mark.parametrize("name,bad,msg", [
    (None, None, "on the GPU"),
    ("positions", torch.zeros(5, dtype=I32), "2-D int32"),
    ("positions", torch.zeros(3, 4, dtype=I32), "positions has shape"),
    ("positions", torch.zeros(3, 5, dtype=I64), "positions has dtype"),
    ("q", torch.zeros(5, 4, 64), "q has dtype"),
])
def test_axes_binding(name, bad, msg, monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    z = lambda *s: torch.zeros(*s, dtype=BF)
    # tensors on the CPU pass every check of shape and type, and stop at the device's
    monkeypatch.setattr(cwlib, "_head_rows", lambda t, n, total, heads, d: cwlib._want(t, n, (BF,), (total, heads, d)))
    a = dict(q=z(5, 4, 64), k=z(5, 2, 64), cos_sin=torch.zeros(10, 64), positions=torch.zeros(3, 5, dtype=I32), axis_of=[0] * 32)
    if name is not None:
        a[name] = bad
    with pytest.raises(ValueError, match=msg):
        cwlib.qk_norm_rope_axes(**a)


@pytest.mark.parametrize("name,bad,msg", [
    (None, None, "on the GPU"),
    ("x", torch.zeros(128, dtype=BF), "x must be a 2-D"),
    ("x", torch.zeros(5, 128), "x has dtype"),
    ("residual", torch.zeros(5, 64, dtype=BF), "residual has shape"),
    ("residual", torch.zeros(5, 128, dtype=torch.float16), "residual has dtype"),
    ("residual_out", torch.zeros(5, 128), "residual_out has dtype"),
    ("y_out", torch.zeros(5, 128, dtype=BF), "without pre_weight"),
    ("post_weight", torch.zeros(64), "post_weight has shape"),
    ("pre_weight", torch.zeros(128, dtype=BF), "pre_weight has dtype"),
    ("gate", torch.zeros(128), "gate has dtype"),
    ("gate", torch.zeros(4, 128, dtype=BF), "gate has shape"),
])
def test_residual_binding(name, bad, msg, monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    rows = lambda t, n, total, width: (cwlib._want(t, n, (BF,), (total, width)), width)
    monkeypatch.setattr(cwlib, "_rows", rows)
    monkeypatch.setattr(cwlib, "_dptr", lambda t: None)
    a = dict(x=torch.zeros(5, 128, dtype=BF), residual=torch.zeros(5, 128, dtype=BF))
    if name is not None:
        a[name] = bad
    with pytest.raises(ValueError, match=msg):
        cwlib.residual_norm(**a)


@pytest.mark.parametrize("lang", ["c11", "c++17"])
def test_the_layer_header_compiles_alone(lang, tmp_path):
    cc = shutil.which("gcc" if lang == "c11" else "g++")
    src = tmp_path / ("t.c" if lang == "c11" else "t.cpp")
    src.write_text('#include "cw_layer.h"\nint main(void) { return cw_residual_norm == 0 || cw_shaped_attention == 0; }\n')
    r = subprocess.run([cc, f"-std={lang}", "-Wall", "-Wno-address", "-Werror", "-D__HIP_PLATFORM_AMD__", "-I", f"{ROOT}/include", "-I",
                        "/opt/rocm/include", "-fsyntax-only", str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

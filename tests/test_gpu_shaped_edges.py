"""shaped_attention at the ends of what it takes: first positions far outside a sequence, slopes of either sign,
page scales far apart or zero, a kept plan under other limits, a captured plan in memory."""
import numpy as np
import pytest
import torch

import paper_2606_16824_amd as cwlib
from gpu_util import to_gpu
from shaped_util import call, check, inputs, shape_of

pytestmark = pytest.mark.gpu

LP, LS = [300, 0, 77, 500, 64], [1, 70, 1, 129, 64]
DTS = [(64, "bf16"), (128, "bf16"), (64, "fp8"), (128, "fp8")]


@pytest.mark.parametrize("d,dt", DTS)
def test_first_positions_far_outside(d, dt):
    print(f"\n[case] shaped far begins {d} {dt}", flush=True)
    w = inputs(LP, LS, 2, 4, d, 16, dt, seed=9)
    pos = np.concatenate([lp + np.arange(ls) for lp, ls in zip(LP, LS)])
    rng = np.random.default_rng(2)
    for only_last in (False, True):
        kw = shape_of(w, cap=20.0)
        ends = np.stack([np.full_like(pos, -2 ** 31), np.full_like(pos, 2 ** 31 - 1), pos, pos + 1])
        kind = rng.integers(0, 4, size=len(pos))
        kw["key_begins"] = (np.full_like(pos, 2 ** 31 - 1) if only_last else ends[kind, np.arange(len(pos))]).astype(np.int32)
        check(w, kw, f"shaped far begins {d} {dt} {only_last}")


@pytest.mark.parametrize("d,dt", DTS)
@pytest.mark.parametrize("cap", [0.0, 30.0])
def test_slopes_of_either_sign(d, dt, cap):
    """Flat, steep, and growing with the distance (every block then raises the running max)."""
    print(f"\n[case] shaped slopes {d} {dt} {cap}", flush=True)
    w = inputs(LP, LS, 2, 4, d, 64, dt, seed=10)
    kw = shape_of(w, cap=cap, window=200)
    kw["slopes"] = np.array([0.0, 30.0, -0.05, -1.0, 1e-6, 2.0, -30.0, 0.5], dtype=np.float32)
    check(w, kw, f"shaped slopes {d} {dt} {cap}")
    kw["full_lens"] = np.array([200, 50, 0, 600, 128], dtype=np.int32)
    check(w, kw, f"shaped slopes full {d} {dt} {cap}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("spread", [[1.0, 2.0 ** -7], [2.0 ** 6, 2.0 ** -6, 1.0, 0.0], [0.0], [0.0, 1.0], [2.0 ** -60, 2.0 ** -50]])
def test_page_scales(d, page, spread):
    """Single tokens hold weights times V scales in fp16 or, where the scales lie further apart, as two bf16."""
    print(f"\n[case] shaped scales {d} {page} {spread}", flush=True)
    w = inputs([900, 200, 33, 64], [1, 70, 1, 1], 2, 4, d, page, "fp8", seed=11)
    rng = np.random.default_rng(5)
    for s in (w.k_scale, w.v_scale):
        s.copy_(torch.from_numpy(rng.choice(spread, size=tuple(s.shape)).astype(np.float32)) * (1.0 if s is w.v_scale else 0.25))
    check(w, shape_of(w, cap=20.0), f"shaped scales {d} {page} {spread}")


@pytest.mark.parametrize("dt", ["bf16", "fp8"])
def test_kept_plan_and_other_limits(dt):
    """Equal lengths, other windows and prefix masks, in turn: each call's first bits again."""
    print(f"\n[case] shaped kept {dt}", flush=True)
    w = inputs(LP, LS, 2, 4, 128, 16, dt, seed=12)
    dw = to_gpu(w)
    kws = [shape_of(w), shape_of(w, window=100), shape_of(w, window=101), shape_of(w, full=[0] * 5), shape_of(w, full=[200, 50, 0, 629, 128]),
           shape_of(w, full=[200, 50, 0, 300, 128]), shape_of(w, full=[200, 50, 0, 300, 128], window=100)]
    first = [check(w, kw, f"shaped kept {dt} {i}", dw=dw)[0] for i, kw in enumerate(kws)]
    for order in ([6, 0, 4, 5, 3, 1, 2], [2, 1, 2, 5, 4, 6, 0, 3]):
        for i in order:
            assert torch.equal(call(dw, kws[i]), first[i]), i


def test_captured_plan_in_memory():
    """A batch whose plan does not fit the kernel arguments, replayed after eager calls of others on the workspace."""
    print("\n[case] shaped captured large plan", flush=True)
    cwlib.init()
    rng = np.random.default_rng(6)
    ls = np.where(np.arange(400) % 4 == 0, rng.integers(2, 40, size=400), 1)
    w = inputs(rng.integers(0, 400, size=400), ls, 2, 2, 64, 16, "bf16", seed=13)
    kw = shape_of(w, cap=20.0, window=150, docs=2)
    dw = to_gpu(w)
    other = inputs(LP, LS, 2, 2, 64, 16, "bf16", seed=14)
    dother, kw_other = to_gpu(other), shape_of(other, window=10)
    ws = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    want = call(dw, kw, workspace=ws).clone()
    want_other = call(dother, kw_other, workspace=ws).clone()
    s, begins, out = dw.spec, torch.from_numpy(kw["key_begins"]).cuda(), torch.zeros_like(dw.q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cwlib.shaped_attention(dw.q, dw.k_new, dw.v_new, dw.k_pool, dw.v_pool, dw.block_table, s.prefix_lens, s.suffix_lens, 2,
                               s.softmax_scale, score_cap=20.0, window=150, key_begins=begins, out=out, workspace=ws)
    for _ in range(4):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert torch.equal(call(dother, kw_other, workspace=ws), want_other)

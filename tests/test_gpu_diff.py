"""diff_attention against the oracle, element by element.

Tolerance, per element, from the kernels' arithmetic (u the operand rounding of the weights:
2^-8 in bf16, 2^-11 in fp16, which chunks over fp8 pools use):
  before the norm, x = sum_j (p1 - lam p2) v:  |dx| <= r mass, mass = sum (p1 + |lam| p2) |v|
    (oracle), r = 2 u (a weight's rounding in the numerator and in the sum) + 2^-10 for the fp32
    parts (dot products of up to 128 exact products: below 2^-13 of sum |q k| <= ~10 each; the
    exponent's argument; the sums), and for chunks over fp8 pools 2^-10 (the value: code x scale
    in fp16, scale rounded too) + 2 * 2^-10 scores (the same of the keys; scores = the
    largest scale sum |q k| of the row)
  norm, y = x w / sqrt(mean x^2 + eps) s:  |dy| <= |s w| / root (|dx| + |x| rms(dx) / root), root
    = sqrt(mean x^2 + eps), with 1.1 for the second order and the fp32 norm
  stored: + 2^-8 |y|."""
import numpy as np
import pytest
import torch

import cw_workloads as cw
import oracle
import paper_2606_16824_amd as cwlib
from conftest import paged_inputs
from gpu_util import to_gpu

pytestmark = pytest.mark.gpu


def _bound(inp, out, terms, weight, eps, after, single):
    """`single` per row: whether it is a sequence's only new token (the streaming kernel)."""
    fp8 = inp.kv_dtype == "fp8"
    chunk = 2 * 2.0 ** -11 + 2.0 ** -10 + 2.0 ** -10 + 2 * 2.0 ** -10 * terms["scores"] if fp8 else 2 * 2.0 ** -8 + 2.0 ** -10
    r = np.where(single[:, None, None], 2 * 2.0 ** -8 + 2.0 ** -10, chunk)
    dx, x = r * terms["mass"], terms["x"]
    if weight is None:
        dy = abs(after) * dx
    else:
        root = np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        rms = np.sqrt((dx * dx).mean(-1, keepdims=True))
        dy = 1.1 * np.abs(after * weight) / root * (dx + np.abs(x) * rms / root)
    return dy + 2.0 ** -8 * np.abs(out) + 1e-38


def _inputs(lp, ls, pairs, g, d, page, dt, seed=3, norm=True):
    spec = cw.custom_spec(lp, ls, num_kv_heads=2 * pairs, gqa_group=g, head_dim=d, page_size=page, kv_dtype=dt, seed=seed)
    w = cw.materialize(spec)
    rng = np.random.default_rng(seed)
    lam = rng.uniform(-0.3, 0.9, size=pairs * g).astype(np.float32)
    weight = rng.uniform(0.5, 1.5, size=2 * d).astype(np.float32) if norm else None
    return w, to_gpu(w), lam, weight


def _run(dw, lam, weight, eps=1e-5, after=0.6, **kw):
    s = dw.spec
    return cwlib.diff_attention(dw.q, dw.k_new, dw.v_new, dw.k_pool, dw.v_pool, dw.block_table, s.prefix_lens, s.suffix_lens,
                                s.gqa_group, s.softmax_scale, torch.from_numpy(lam).cuda(), k_scale=dw.k_scale,
                                v_scale=dw.v_scale, norm_weight=None if weight is None else torch.from_numpy(weight).cuda(),
                                norm_eps=eps, out_scale=after, **kw)


def _check(w, dw, lam, weight, what, eps=1e-5, after=0.6):
    out = torch.full((dw.q.shape[0], dw.q.shape[1] // 2, 2 * dw.q.shape[2]), float("nan"), dtype=torch.bfloat16, device="cuda")
    got = _run(dw, lam, weight, eps, after, out=out)
    torch.cuda.synchronize()
    assert got is out
    inp = paged_inputs(w)
    ref, terms = oracle.diff_attention(inp, lam, weight, eps, after)
    single = np.repeat(w.spec.suffix_lens == 1, w.spec.suffix_lens)
    tol = _bound(inp, ref, terms, weight, eps, after, single)
    g = out.cpu().double().numpy()
    assert np.isfinite(g).all(), what
    over = np.abs(g - ref) / tol
    print(f"[{what}] worst {over.max():.3f} of the tolerance, relative {np.linalg.norm(g - ref) / np.linalg.norm(ref):.2e}",
          flush=True)
    assert over.max() <= 1.0, what
    return out


CASES = [
    # lp, ls, pairs, g, d, page, dt
    ([0], [1], 1, 1, 64, 16, "bf16"),
    ([5], [1], 1, 4, 128, 16, "bf16"),
    ([0], [2], 1, 1, 128, 16, "bf16"),
    ([31, 32, 33, 0, 64, 200], [1, 1, 1, 1, 1, 1], 2, 3, 128, 16, "bf16"),
    ([31, 32, 33, 0, 64, 200], [1, 1, 1, 1, 1, 1], 2, 16, 64, 64, "bf16"),
    ([31, 32, 33, 0, 64, 200], [1, 1, 1, 1, 1, 1], 2, 4, 128, 64, "fp8"),
    ([17, 1000, 90], [1, 1, 1], 1, 5, 64, 16, "fp8"),
    ([3000, 777, 1999], [1, 1, 1], 2, 4, 128, 16, "bf16"),
    ([2500, 640], [1, 1], 4, 2, 64, 64, "bf16"),
    ([2900, 64], [1, 1], 2, 8, 128, 64, "fp8"),
    ([0, 16, 63, 64, 65, 31, 33], [33, 2, 64, 65, 31, 97, 3], 1, 4, 64, 16, "bf16"),
    ([0, 16, 63, 64, 65, 31, 33], [33, 2, 64, 65, 31, 97, 3], 1, 4, 128, 64, "bf16"),
    ([0, 16, 63, 64, 65, 31, 33], [33, 2, 64, 65, 31, 97, 3], 1, 3, 128, 16, "fp8"),
    ([0, 16, 63, 64, 65, 31, 33], [33, 2, 64, 65, 31, 97, 3], 2, 1, 64, 64, "fp8"),
    ([300, 0, 17, 500, 40], [1, 70, 1, 129, 0], 2, 4, 128, 16, "bf16"),
    ([300, 0, 17, 500, 40], [1, 70, 1, 129, 0], 3, 5, 64, 64, "bf16"),
    ([300, 0, 17, 500, 40], [1, 70, 1, 129, 0], 2, 2, 128, 64, "fp8"),
    ([300, 0, 17, 500, 40], [1, 70, 1, 129, 0], 1, 16, 64, 16, "fp8"),
    ([700, 90, 1500], [150, 64, 300], 2, 4, 128, 16, "bf16"),
    ([0, 0], [400, 131], 1, 1, 128, 64, "bf16"),
    ([0], [700], 2, 8, 64, 16, "bf16"),
    ([1], [600], 1, 2, 128, 16, "fp8"),
]


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_against_oracle(i, norm):
    lp, ls, pairs, g, d, page, dt = CASES[i]
    print(f"\n[case] diff {CASES[i]} norm={norm}", flush=True)
    w, dw, lam, weight = _inputs(lp, ls, pairs, g, d, page, dt, seed=50 + i, norm=norm)
    _check(w, dw, lam, weight, f"diff {CASES[i]} norm={norm}", after=0.6 if norm else 1.0)


@pytest.mark.parametrize("tiles", [1, 2, 5])
@pytest.mark.parametrize("dt", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
def test_split_keys(tiles, dt, d):
    """Every key range cut into pieces of `tiles` tiles: merges of two to some thirty partials."""
    print(f"\n[case] diff split {tiles} {dt} {d}", flush=True)
    w, dw, lam, weight = _inputs([900, 0, 333, 64], [40, 200, 1, 1], 2, 3, d, 16, dt, seed=90 + tiles)
    cwlib.set_tuning(0, tiles)
    try:
        _check(w, dw, lam, weight, f"diff split {tiles} {dt} {d}")
    finally:
        cwlib.set_tuning(0, 0)


@pytest.mark.parametrize("d,page,dt", [(64, 16, "bf16"), (128, 64, "fp8")])
def test_levelled_plan(d, page, dt):
    """More query tiles than CUs, and far from a multiple: some are cut into key ranges. Another
    plan than with whole tiles (a target of 256 workgroups), the same result within the bounds."""
    print(f"\n[case] diff levelled {d} {dt}", flush=True)
    w, dw, lam, weight = _inputs([1500, 1400, 900, 1600, 1300, 700, 1500], [700, 650, 640, 600, 690, 710, 500], 2, 4, d, page,
                                 dt, seed=29)  # 286 tiles
    got = _check(w, dw, lam, weight, f"diff levelled {d} {dt}")
    cwlib.set_tuning(1, 256)
    try:
        whole = _run(dw, lam, weight)
    finally:
        cwlib.set_tuning(1, 0)
    torch.cuda.synchronize()
    assert not torch.equal(got, whole)


@pytest.mark.parametrize("knob,value", [(4, 1), (6, 0), (7, 0)])
def test_plan_paths_give_the_same_bits(knob, value):
    """Plans read from the staging slot, uploaded in full, or not in the kernel arguments."""
    print(f"\n[case] diff plan path {knob}={value}", flush=True)
    for lens in (([900, 40, 333], [1, 1, 1]), ([900, 40, 333], [40, 200, 3]), ([900, 40, 333], [1, 200, 1])):
        w, dw, lam, weight = _inputs(*lens, 2, 3, 128, 16, "bf16", seed=7)
        want = _run(dw, lam, weight)
        cwlib.set_tuning(knob, value)
        try:
            got = _run(dw, lam, weight)
        finally:
            cwlib.set_tuning(knob, 1 if knob in (6, 7) else 0)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_first_map_alone_is_the_plain_attention():
    """lam = 0 and no norm: each half of the value against the framework's own attention."""
    print("\n[case] diff with lam 0", flush=True)
    w, dw, lam, _ = _inputs([300, 0, 17], [1, 70, 129], 2, 4, 128, 16, "bf16", seed=31, norm=False)
    s = dw.spec
    got = _run(dw, np.zeros_like(lam), None, after=1.0).view(-1, 2, 4, 2, 128)
    cols = lambda x, m: x.view(x.shape[0], 2, -1, *x.shape[2:])[:, :, m]
    q = dw.q.view(-1, 2, 4, 2, 128)[:, :, :, 0].reshape(-1, 8, 128).contiguous()
    k = dw.k_new.view(-1, 2, 2, 128)[:, :, 0].contiguous()
    kp = cols(dw.k_pool, 0).contiguous()
    for half in (0, 1):
        v = dw.v_new.view(-1, 2, 2, 128)[:, :, half].contiguous()
        vp = cols(dw.v_pool, half).contiguous()
        want = cwlib.extend_attention(q, k, v, kp, vp, dw.block_table, s.prefix_lens, s.suffix_lens, 4, s.softmax_scale)
        torch.cuda.synchronize()
        err = (got[:, :, :, half].reshape(-1, 8, 128).float() - want.float()).abs().max().item()
        assert err <= 4e-2, err  # two kernels, each within the 2e-2 that its tests allow


@pytest.mark.parametrize("d,dt", [(128, "bf16"), (64, "fp8")])
def test_rising_scores_raise_the_running_max(d, dt):
    """Keys that grow along the prefix: the running max is raised again and again."""
    print(f"\n[case] diff rising scores {d} {dt}", flush=True)
    w, dw, lam, weight = _inputs([700, 700], [1, 90], 1, 2, d, 16, dt, seed=77)
    heads = w.k_pool.shape[1]
    ramp = torch.ones(w.k_pool.shape[0])
    for b in range(2):
        for j in range(44):
            ramp[int(w.block_table[b, j])] = 1.0 + 0.25 * j
    if dt == "fp8":
        w.k_scale *= ramp[:, None]
    else:
        w.k_pool *= ramp[:, None, None, None].to(torch.bfloat16)
    dw = to_gpu(w)
    inp = paged_inputs(w)
    out = _run(dw, lam, weight)
    torch.cuda.synchronize()
    ref, terms = oracle.diff_attention(inp, lam, weight, 1e-5, 0.6)
    single = np.repeat(w.spec.suffix_lens == 1, w.spec.suffix_lens)
    # the fp32 dot products' part grows with the scores: 2^-17 of them, in numerator and sum
    terms["mass"] = terms["mass"] * (1 + 2.0 ** -16 * terms["scores"] / (2 * 2.0 ** -11))
    over = np.abs(out.cpu().double().numpy() - ref) / _bound(inp, ref, terms, weight, 1e-5, 0.6, single)
    assert float(terms["scores"].max()) > 40 and over.max() <= 1.0, over.max()
    assert heads == 2


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("where", ["all huge", "all tiny", "one prefix page huge", "a new token huge", "first tile tiny", "zeros"])
def test_values_of_any_size(where, d):
    """bf16 pools: values near the ends of bf16's range, alone and among others."""
    print(f"\n[case] diff values {where} {d}", flush=True)
    w, _, lam, weight = _inputs([300, 0, 70, 300], [90, 130, 33, 1], 1, 3, d, 16, "bf16", seed=66)
    big, small = 2.0 ** 60, 2.0 ** -60
    if where.startswith("all"):
        w.v_pool *= big if where == "all huge" else small
        w.v_new *= big if where == "all huge" else small
    elif where == "one prefix page huge":
        w.v_pool[int(w.block_table[0, 9]), 1] *= big
    elif where == "a new token huge":
        w.v_new[200, 0] *= big
    elif where == "first tile tiny":
        for j in range(4):
            w.v_pool[int(w.block_table[0, j])] *= small
    else:
        w.v_pool[:, 0] = 0
        w.v_new[:, 0] = 0
    dw = to_gpu(w)
    # without a norm (its mean of squares would pass fp32)
    _check(w, dw, lam, None, f"diff values {where} {d}", after=1.0)


@pytest.mark.parametrize("d,page", [(64, 64), (128, 16)])
def test_pages_of_zeros_have_scale_zero(d, page):
    """fp8 pages whose largest value is 0 and so their scale: a whole prefix, and last pages that
    are partly filled, of K, of V and of both."""
    print(f"\n[case] diff scale zero {d} {page}", flush=True)
    w, _, lam, weight = _inputs([300, 309, 300, 309, 5, 70], [1, 1, 1, 90, 1, 40], 2, 3, d, page, "fp8", seed=67)
    last = lambda b: int(w.block_table[b, (int(w.spec.prefix_lens[b]) - 1) // page])
    w.k_scale[last(0)] = 0
    w.v_scale[last(1)] = 0
    w.k_scale[last(2), 1] = w.v_scale[last(2), 2] = 0
    w.k_scale[last(3)] = w.v_scale[last(3)] = 0
    for b in (4, 5):
        for j in range(-(-int(w.spec.prefix_lens[b]) // page)):
            w.k_scale[int(w.block_table[b, j])] = w.v_scale[int(w.block_table[b, j])] = 0
    _check(w, to_gpu(w), lam, weight, f"diff scale zero {d}")


@pytest.mark.parametrize("d,page", [(64, 16), (128, 64)])
def test_value_scales_far_apart(d, page):
    """Single tokens over fp8 pages whose V scales lie up to 2^20 apart, with most of the weight
    on a page of small values.  (Scores reach 116: 2^-16 of them from the dot products, 2^-9 in all, is
    less than the bound's 2^-7 leaves beside fp16 weights.)"""
    print(f"\n[case] diff value scales {d} {page}", flush=True)
    lp = [900, 500, 37]
    w, _, lam, weight = _inputs(lp, [1, 1, 1], 2, 3, d, page, "fp8", seed=68)
    rng = np.random.default_rng(5)
    for b in range(3):
        n = -(-lp[b] // page)
        for j in range(n):
            w.v_scale[int(w.block_table[b, j])] *= float(2.0 ** -rng.integers(0, 17))
        pg = int(w.block_table[b, n // 2])
        w.k_scale[pg] *= 12.0
        w.v_scale[pg] = 2.0 ** -23  # (scales are at most 0.1)
    w.v_new *= 2.0 ** -20
    _check(w, to_gpu(w), lam, None, f"diff value scales {d}", after=1.0)


def test_other_stream_shared_workspace_and_repeat():
    print("\n[case] diff on another stream", flush=True)
    w, dw, lam, weight = _inputs([900, 40, 333], [1, 200, 3], 2, 3, 128, 16, "bf16", seed=12)
    s = dw.spec
    nb = cwlib.diff_workspace_bytes(s.prefix_lens, s.suffix_lens, 2, 3, 128, 16, "bf16")
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    a = _run(dw, lam, weight, workspace=ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        b = _run(dw, lam, weight, workspace=ws)
        c = _run(dw, lam, weight, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(a, c)


def test_pages_past_4_gib():
    """The same call with its pages moved past 4 GiB of the pools: the same bits."""
    print("\n[case] diff large pools", flush=True)
    w, dw, lam, weight = _inputs([500, 900], [1, 80], 2, 2, 128, 64, "bf16", seed=15)
    want = _run(dw, lam, weight)
    n = dw.k_pool.shape[0]
    far = 80000  # pages of 64 KB
    move = lambda x: torch.cat([torch.zeros(far, *x.shape[1:], dtype=x.dtype, device="cuda"), x])
    dw.k_pool, dw.v_pool = move(dw.k_pool), move(dw.v_pool)
    bt = dw.block_table
    dw.block_table = torch.where((bt >= 0) & (bt < n), bt + far, bt).contiguous()
    got = _run(dw, lam, weight)
    torch.cuda.synchronize()
    assert torch.equal(got, want)

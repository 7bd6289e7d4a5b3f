"""shaped_attention against the oracle, element by element (the bound: shaped_util)."""
import numpy as np
import pytest
import torch

import paper_2606_16824_amd as cwlib
from gpu_util import to_gpu
from shaped_util import call, check, inputs, shape_of

pytestmark = pytest.mark.gpu

SIZES = [
    # lp, ls, hkv, g, d, page, dt
    ([0], [1], 1, 1, 64, 16, "bf16"),
    ([5], [1], 1, 4, 128, 16, "bf16"),
    ([0], [2], 1, 1, 128, 16, "bf16"),
    ([31, 32, 33, 0, 64, 200], [1, 1, 1, 1, 1, 1], 2, 3, 128, 16, "bf16"),
    ([31, 32, 33, 0, 64, 200], [1, 1, 1, 1, 1, 1], 2, 16, 64, 64, "bf16"),
    ([31, 32, 33, 0, 64, 200], [1, 1, 1, 1, 1, 1], 2, 4, 128, 64, "fp8"),
    ([17, 1000, 90], [1, 1, 1], 1, 5, 64, 16, "fp8"),
    ([2500, 640], [1, 1], 2, 2, 64, 64, "bf16"),
    ([2900, 64, 1500], [1, 1, 1], 2, 8, 128, 64, "fp8"),
    ([0, 16, 63, 64, 65, 31, 33], [33, 2, 64, 65, 31, 97, 3], 1, 4, 64, 16, "bf16"),
    ([0, 16, 63, 64, 65, 31, 33], [33, 2, 64, 65, 31, 97, 3], 1, 4, 128, 64, "bf16"),
    ([0, 16, 63, 64, 65, 31, 33], [33, 2, 64, 65, 31, 97, 3], 1, 3, 128, 16, "fp8"),
    ([0, 16, 63, 64, 65, 31, 33], [33, 2, 64, 65, 31, 97, 3], 2, 1, 64, 64, "fp8"),
    ([300, 0, 17, 500, 40], [1, 70, 1, 129, 0], 2, 4, 128, 16, "bf16"),
    ([300, 0, 17, 500, 40], [1, 70, 1, 129, 0], 1, 16, 64, 16, "fp8"),
    ([700, 90, 1500], [150, 64, 300], 1, 4, 128, 16, "bf16"),
    ([700, 90, 1500], [150, 64, 300], 1, 4, 64, 64, "fp8"),
    ([0, 0], [400, 131], 1, 1, 128, 64, "bf16"),
    ([0], [700], 1, 8, 64, 16, "bf16"),
    ([1], [600], 1, 2, 128, 16, "fp8"),
    ([1000], [420], 1, 1, 128, 16, "fp8"),
]
SHAPES = {
    "plain": dict(),
    "cap": dict(cap=20.0),
    "slopes": dict(slopes=True),
    "window1": dict(window=1),
    "window7": dict(window=7, cap=5.0),
    "window100": dict(window=100),
    "window333": dict(window=333, slopes=True),
    "docs": dict(docs=6),
    "docs_window": dict(docs=3, window=150, cap=50.0),
    "empty": dict(docs=4, empty=True),
    "empty_cap_slopes": dict(empty=True, cap=30.0, slopes=True),
    "full": dict(full="most"),
    "full_slopes_window": dict(full="most", slopes=True, window=90),
    "full_docs_cap": dict(full="all", docs=3, cap=10.0, empty=True),
}


def _shape(w, name, seed):
    kw = dict(SHAPES[name])
    if kw.get("full"):
        n = w.spec.prefix_lens + w.spec.suffix_lens
        # three quarters of each sequence, or more than all of it; every third sequence has none
        kw["full"] = [0 if b % 3 == 2 else (3 * x // 4 if kw["full"] == "most" else x + 50) for b, x in enumerate(n)]
    return shape_of(w, seed=seed, **kw)


@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("i", range(len(SIZES)))
def test_against_oracle(i, name):
    print(f"\n[case] shaped {SIZES[i]} {name}", flush=True)
    w = inputs(*SIZES[i], seed=50 + i)
    check(w, _shape(w, name, 70 + i), f"shaped {SIZES[i]} {name}")


@pytest.mark.parametrize("tiles", [1, 2, 5])
@pytest.mark.parametrize("dt", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("name", ["cap", "window333", "docs_window", "empty_cap_slopes", "full"])
def test_split_keys(tiles, dt, d, name):
    """Every key range cut into pieces of `tiles` tiles: merges of two to some thirty partials, whole pieces
    without a visible key among them."""
    print(f"\n[case] shaped split {tiles} {dt} {d} {name}", flush=True)
    w = inputs([900, 0, 333, 64], [40, 200, 1, 1], 2, 3, d, 16, dt, seed=90 + tiles)
    cwlib.set_tuning(0, tiles)
    try:
        check(w, _shape(w, name, 5), f"shaped split {tiles} {dt} {d} {name}")
    finally:
        cwlib.set_tuning(0, 0)


@pytest.mark.parametrize("dt", ["bf16", "fp8"])
@pytest.mark.parametrize("d,page", [(64, 64), (128, 16)])
@pytest.mark.parametrize("window", [1, 16, 64, 65, 100, 500])
def test_pages_before_the_window_are_not_read(dt, d, page, window):
    """Table entries of pages wholly before every window are invalid, and what lies before the first
    visible key in the others is NaN: same bits as with everything in place."""
    print(f"\n[case] shaped freed {dt} {d} {page} {window}", flush=True)
    w = inputs([900, 61, 1333, 700, 256], [1, 130, 77, 1, 64], 2, 4, d, page, dt, seed=17)
    kw = shape_of(w, cap=20.0, window=window)
    dw = to_gpu(w)
    want, want_lse = check(w, kw, f"shaped freed {dt} {d} {page} {window}", dw=dw)
    nan = torch.full((), 0x7F if dt == "fp8" else float("nan"), dtype=dw.k_pool.dtype, device="cuda")
    for b, (lp, ls) in enumerate(zip(w.spec.prefix_lens.tolist(), w.spec.suffix_lens.tolist())):
        first = max(0, lp - window + 1)  # of the first new token's window
        for i in range((lp + ls + page - 1) // page):
            row = int(w.block_table[b, i])
            if (i + 1) * page <= first:
                dw.block_table[b, i] = 0x7FFFFFFF
            for pool in (dw.k_pool, dw.v_pool):
                pool[row, :, :max(0, min(page, first - i * page))] = nan
            if dt == "fp8" and (i + 1) * page <= first:
                dw.k_scale[row] = dw.v_scale[row] = float("nan")
    lse = torch.full_like(want_lse, 7.0)
    got = call(dw, kw, lse=lse)
    torch.cuda.synchronize()
    assert torch.equal(got.view(torch.int16), want.view(torch.int16)) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("dt", ["bf16", "fp8"])
def test_one_sided_shapes_agree(dt):
    """A cap that nothing reaches, slopes of 0, a window and documents that hide nothing and prefix masks that add
    nothing: the plain call's outputs but for rounding."""
    print(f"\n[case] shaped agree {dt}", flush=True)
    w = inputs([500, 0, 40], [90, 130, 1], 2, 4, 128, 16, dt, seed=7, sharp=1.0)
    dw = to_gpu(w)
    plain = call(dw, shape_of(w)).float()
    total = int(w.spec.suffix_lens.sum())
    for kw in (dict(window=4000), dict(begins=np.zeros(total, dtype=np.int32)), dict(full=[500, 0, 41]), dict(slopes=np.zeros(8, dtype=np.float32))):
        full = shape_of(w, window=kw.get("window", 0), full=kw.get("full"))
        full["key_begins"], full["slopes"] = kw.get("begins"), kw.get("slopes")
        got = call(dw, full).float()
        torch.cuda.synchronize()
        assert (got - plain).abs().max().item() <= 2.0 ** -7 * plain.abs().max().item(), kw.keys()


@pytest.mark.parametrize("d,page,dt,name", [(64, 16, "bf16", "cap"), (128, 64, "fp8", "window333"), (128, 16, "bf16", "full_slopes_window"),
                                            (64, 64, "fp8", "docs")])
def test_levelled_plan(d, page, dt, name):
    """More query tiles than CUs, and far from a multiple: some may be cut into key ranges."""
    print(f"\n[case] shaped levelled {d} {dt} {name}", flush=True)
    w = inputs([1500, 1400, 900], [700, 650, 640], 8, 4, d, page, dt, seed=29)
    # (rows of two tokens are compared: the oracle goes row by row)
    kw = _shape(w, name, 3)
    dw = to_gpu(w)
    got = call(dw, kw)
    cwlib.set_tuning(1, 256)
    try:
        whole = call(dw, kw)
    finally:
        cwlib.set_tuning(1, 0)
    torch.cuda.synchronize()
    assert torch.isfinite(got.float()).all()
    # two results within the bound of each other: 2 u of the mass each, mass at most sqrt(sum w v^2) <= 4.5 in magnitude here
    assert (got.float() - whole.float()).abs().max().item() <= 4 * 2.0 ** -8 * 4.5


def test_many_decodes():
    print("\n[case] shaped 300 decodes", flush=True)
    rng = np.random.default_rng(4)
    w = inputs(rng.integers(0, 300, size=300), np.ones(300, dtype=int), 1, 2, 64, 16, "bf16", seed=5)
    check(w, shape_of(w, cap=20.0, window=128, docs=2), "shaped 300 decodes")


def test_nothing_to_do():
    w = inputs([40, 0], [0, 0], 1, 2, 64, 16, "bf16")
    assert call(to_gpu(w), shape_of(w)).shape == (0, 2, 64)

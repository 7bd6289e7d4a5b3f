"""qk_norm_rope against the oracle, and its pools against the page write of its outputs.

Tolerance of q_out and k_out: fp32 throughout, one rounding to bf16 (2^-8 relative).  The
fp32 part: the sum of squares of up to 128 terms (all positive: relative (128 + 1) 2^-24 at
most, half of it after the root), root and quotient 2^-23 each, then four products and a sum:
below 2^-16 of |a cos| + |b sin| in all.  So |error| <= 2^-8 |y| + 2^-15 (|a| + |b|), the
second for the sum's cancellation and what the rounding sees of it."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_16824_amd as cwlib
from gpu_util import bits

pytestmark = pytest.mark.gpu
EPS = 1e-6


def _angles(n, rot):
    a = np.arange(n)[:, None] * 10000.0 ** (-np.arange(0, rot, 2) / rot)[None, :]
    return torch.from_numpy(np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)).cuda()


def _inputs(t, hq, hkv, d, rot, packed, seed, positions=5000):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=gen, device="cuda", dtype=torch.bfloat16)
    if packed:
        x = n(t, hq + 2 * hkv, d)
        q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    else:
        q, k, v = n(t, hq, d), n(t, hkv, d), n(t, hkv, d)
    w = [torch.rand(d, generator=gen, device="cuda") + 0.5 for _ in range(2)]
    pos = torch.randint(0, positions, (t,), generator=gen, device="cuda", dtype=torch.int32)
    return q, k, v, w, pos, _angles(positions, rot)


def _want(x, w, cs, pos, interleaved):
    """Oracle values and, of each element, the |a| + |b| that its tolerance goes by."""
    half = cs.shape[1] // 2
    angle = cs.cpu().double().numpy()[np.clip(pos.cpu().numpy(), 0, len(cs) - 1)]
    x = x.cpu().double().numpy()
    w = None if w is None else w.cpu().numpy()
    y = oracle.norm_rotate(x, w, EPS, angle[:, :half], angle[:, half:], interleaved)
    size = oracle.norm_rotate(np.abs(x), None if w is None else np.abs(w), EPS, np.ones_like(angle[:, :half]),
                              np.ones_like(angle[:, half:]), interleaved)
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    size[..., a] = size[..., b]  # |a| + |b|: the first of a pair came out as their difference
    return y, size


def _near(got, ref, what):
    y, size = ref
    err = np.abs(got.cpu().double().numpy() - y)
    over = err / (2.0 ** -8 * np.abs(y) + 2.0 ** -15 * size + 1e-30)
    print(f"[{what}] worst {over.max():.3f} of the tolerance", flush=True)
    assert over.max() <= 1.0, what


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("t,hq,hkv,d,rot,packed,norm", [
    (1, 8, 2, 128, 128, True, True), (1, 5, 1, 64, 64, False, True), (3, 1, 1, 64, 16, True, True),
    (17, 4, 1, 128, 64, True, True), (33, 20, 4, 128, 96, False, True), (130, 3, 3, 64, 48, True, False),
    (257, 32, 8, 128, 128, True, True), (9000, 2, 1, 64, 32, False, True), (2, 40, 8, 128, 112, True, False),
])
def test_against_oracle(t, hq, hkv, d, rot, packed, norm, interleaved):
    print(f"\n[case] norm and rotation t={t} {hq}q/{hkv}kv d={d} rot={rot} packed={packed}", flush=True)
    q, k, v, w, pos, cs = _inputs(t, hq, hkv, d, rot, packed, seed=t + d)
    if not norm:
        w = [None, None]
    qo, ko, vo = cwlib.qk_norm_rope(q, k, cs, pos, q_weight=w[0], k_weight=w[1], eps=EPS, interleaved=interleaved, v=v)
    torch.cuda.synchronize()
    _near(qo, _want(q, w[0], cs, pos, interleaved), "q")
    _near(ko, _want(k, w[1], cs, pos, interleaved), "k")
    assert torch.equal(vo, v)
    q2, k2, none = cwlib.qk_norm_rope(q, k, cs, pos, q_weight=w[0], k_weight=w[1], eps=EPS, interleaved=interleaved)
    assert none is None and torch.equal(q2, qo) and torch.equal(k2, ko)


@pytest.mark.parametrize("dt", ["bf16", "fp8"])
@pytest.mark.parametrize("d,page,hq,hkv", [(128, 16, 8, 2), (64, 64, 5, 1), (128, 64, 4, 4), (64, 16, 20, 10)])
def test_pages_are_those_of_the_page_write(dt, d, page, hq, hkv):
    """The pools, byte for byte, as kv_write_pages of k_out and v leaves them."""
    print(f"\n[case] page write {dt} d={d} page={page}", flush=True)
    lp, ls = [0, 37, 64, 5], [19, 1, 70, 0]
    t, num_pages = sum(ls), 40
    q, k, v, w, _, cs = _inputs(t, hq, hkv, d, d, True, seed=d + page)
    gen = torch.Generator(device="cuda").manual_seed(9)
    if dt == "fp8":
        pools = [torch.randint(0, 256, (num_pages, hkv, page, d), generator=gen, device="cuda", dtype=torch.uint8) for _ in "kv"]
        scales = [torch.rand(num_pages, hkv, generator=gen, device="cuda") * 0.02 + 0.001 for _ in "kv"]
    else:
        pools = [torch.randn(num_pages, hkv, page, d, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in "kv"]
        scales = [None, None]
    table = torch.randperm(num_pages, generator=gen, device="cuda").to(torch.int32)[:36].view(4, 9).contiguous()
    want = [x.clone() for x in pools]
    tables = cwlib.build_step_tables(torch.tensor(lp, dtype=torch.int32, device="cuda"),
                                     torch.tensor(ls, dtype=torch.int32, device="cuda"),
                                     torch.empty(0, dtype=torch.int32, device="cuda"), table.clone(), page, t)
    # (no free pages: the slots of held pages are real, those of new ones are made here)
    flat = []
    for b in range(4):
        flat += [int(table[b, p // page]) * page + p % page for p in range(lp[b], lp[b] + ls[b])]
    slots = torch.tensor(flat, dtype=torch.int64, device="cuda")
    qo, ko, vo = cwlib.qk_norm_rope(q, k, cs, tables.positions, q_weight=w[0], k_weight=w[1], v=v, k_pool=pools[0],
                                    v_pool=pools[1], slots=slots, k_scale=scales[0], v_scale=scales[1])
    cwlib.kv_write_pages(ko, vo, want[0], want[1], table, lp, ls, k_scale=scales[0], v_scale=scales[1])
    torch.cuda.synchronize()
    assert torch.equal(vo, v)
    raw = lambda x: x.view(torch.uint8)
    assert torch.equal(raw(pools[0]), raw(want[0])) and torch.equal(raw(pools[1]), raw(want[1]))


def test_padding_tokens_and_slots_outside():
    """Nothing is written of a token without a position, and no page of one without a slot."""
    print("\n[case] padding tokens", flush=True)
    t, hq, hkv, d, page = 12, 4, 2, 64, 16
    q, k, v, w, pos, cs = _inputs(t, hq, hkv, d, d, False, seed=4, positions=100)
    pos[3], pos[7], pos[11] = -1, 100, -(1 << 31)
    slots = torch.arange(t, dtype=torch.int64, device="cuda")
    slots[1], slots[2], slots[5] = -1, 2 * page, 1 << 40
    pools = [torch.full((2, hkv, page, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    outs = [torch.full((t, h, d), 3.0, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv)]
    cwlib.qk_norm_rope(q, k, cs, pos, v=v, k_pool=pools[0], v_pool=pools[1], slots=slots, q_out=outs[0], k_out=outs[1],
                       v_out=outs[2])
    torch.cuda.synchronize()
    good = [i for i in range(t) if i not in (3, 7, 11)]
    for i in (3, 7, 11):
        assert all(bool((o[i] == 3.0).all()) for o in outs)
    for x, o in ((q, outs[0]), (k, outs[1])):
        y, size = _want(x, None, cs, pos, False)
        _near(o[good], (y[good], size[good]), "tokens with a position")
    for pool, o in zip(pools, outs[1:]):
        for s in range(2 * page):
            row = pool[s // page, :, s % page]
            if s < t and s in good and s not in (1, 2, 5):
                assert torch.equal(row, o[s])
            else:
                assert bool((row == 7.0).all())


def test_in_place_and_other_stream():
    print("\n[case] in place", flush=True)
    q, k, v, w, pos, cs = _inputs(70, 8, 2, 128, 128, False, seed=8)
    want = cwlib.qk_norm_rope(q, k, cs, pos, q_weight=w[0], k_weight=w[1], v=v)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = cwlib.qk_norm_rope(q, k, cs, pos, q_weight=w[0], k_weight=w[1], v=v, q_out=q, k_out=k, v_out=v)
    torch.cuda.synchronize()
    assert got[0] is q and all(np.array_equal(bits(a), bits(b)) for a, b in zip(got, want))


def test_rows_of_zeros_infinities_and_nan_stay_their_own():
    print("\n[case] special rows", flush=True)
    q, k, v, w, pos, cs = _inputs(6, 4, 1, 128, 64, False, seed=11)
    want = cwlib.qk_norm_rope(q, k, cs, pos, q_weight=w[0], k_weight=w[1])[0].clone()
    q[1, 2] = 0
    q[2, 1, 5] = float("inf")
    q[4, 0, 9] = float("nan")
    got = cwlib.qk_norm_rope(q, k, cs, pos, q_weight=w[0], k_weight=w[1])[0]
    torch.cuda.synchronize()
    assert bool((got[1, 2] == 0).all()) and bool(got[4, 0].isnan().all()) and bool(got[2, 1, 5].isnan())
    odd = {(1, 2), (2, 1), (4, 0)}
    for t in range(6):
        for h in range(4):
            if (t, h) not in odd:
                assert torch.equal(got[t, h], want[t, h])


def test_offsets_past_32_bits():
    """Pool slots past 4 GiB and a projection of more than 2^31 elements."""
    print("\n[case] large pools and rows", flush=True)
    hkv, page, d, num_pages = 8, 64, 128, 50000
    pools = [torch.zeros(num_pages, hkv, page, d, dtype=torch.bfloat16, device="cuda") for _ in "kv"]  # 6.5 GB each
    t = 5
    x = torch.empty(t, (1 << 29) + 64, dtype=torch.bfloat16, device="cuda")  # tokens 1 GiB apart
    g = torch.Generator(device="cuda").manual_seed(2)
    parts = torch.randn(t, 6 * hkv, d, generator=g, device="cuda", dtype=torch.bfloat16)
    x[:, :6 * hkv * d] = parts.view(t, -1)
    view = lambda a, b: x[:, a * d:b * d].unflatten(1, (b - a, d))
    cs = _angles(10, d)
    pos = torch.arange(t, dtype=torch.int32, device="cuda")
    slots = torch.tensor([3, 49999 * page + 63, 33333 * page, 49998 * page + 1, 17 * page], dtype=torch.int64, device="cuda")
    got = cwlib.qk_norm_rope(view(0, 4 * hkv), view(4 * hkv, 5 * hkv), cs, pos, v=view(5 * hkv, 6 * hkv), k_pool=pools[0],
                             v_pool=pools[1], slots=slots)
    want = cwlib.qk_norm_rope(parts[:, :4 * hkv], parts[:, 4 * hkv:5 * hkv], cs, pos, v=parts[:, 5 * hkv:])
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    for pool, o in zip(pools, got[1:]):
        assert torch.equal(pool[slots // page, :, slots % page], o)
        assert int(torch.count_nonzero(pool.view(torch.int32)[::7])) <= t * hkv * d

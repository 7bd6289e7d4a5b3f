"""qk_norm_rope_axes against the oracle (its tolerance is that of qk_norm_rope: test_gpu_qk_norm_rope), against
qk_norm_rope where all axes agree, and its pools."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_16824_amd as cwlib

pytestmark = pytest.mark.gpu
EPS = 1e-6


def _angles(n, rot):
    a = np.arange(n)[:, None] * 10000.0 ** (-np.arange(0, rot, 2) / rot)[None, :]
    return torch.from_numpy(np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)).cuda()


def _inputs(t, hq, hkv, d, rot, axes, packed, seed, positions=3000):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=gen, device="cuda", dtype=torch.bfloat16)
    if packed:
        x = n(t, hq + 2 * hkv, d)
        q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    else:
        q, k, v = n(t, hq, d), n(t, hkv, d), n(t, hkv, d)
    w = [torch.rand(d, generator=gen, device="cuda") + 0.5 for _ in range(2)]
    pos = torch.randint(0, positions, (axes, t), generator=gen, device="cuda", dtype=torch.int32)
    return q, k, v, w, pos, _angles(positions, rot)


def _axis_of(kind, rot, axes):
    pairs = rot // 2
    if kind == "runs":
        return [i * axes // pairs for i in range(pairs)]
    if kind == "turns":
        return [i % axes for i in range(pairs)]
    if kind == "last":
        return [axes - 1] * pairs
    return np.random.default_rng(rot + axes).integers(0, axes, size=pairs).tolist()


def _near(got, x, w, cs, pos, axis_of, interleaved, what):
    cos, sin = oracle.axis_angles(cs.cpu().double().numpy(), pos.cpu().numpy(), axis_of)
    x = x.cpu().double().numpy()
    w = None if w is None else w.cpu().numpy()
    y = oracle.norm_rotate(x, w, EPS, cos, sin, interleaved)
    half = cos.shape[1]
    size = oracle.norm_rotate(np.abs(x), None if w is None else np.abs(w), EPS, np.ones_like(cos), np.ones_like(sin), interleaved)
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    size[..., a] = size[..., b]  # |a| + |b|: the first of a pair came out as their difference
    over = np.abs(got.cpu().double().numpy() - y) / (2.0 ** -8 * np.abs(y) + 2.0 ** -15 * size + 1e-30)
    print(f"[{what}] worst {over.max():.3f} of the tolerance", flush=True)
    assert over.max() <= 1.0, what


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("kind", ["runs", "turns", "random", "last"])
@pytest.mark.parametrize("t,hq,hkv,d,rot,axes,packed,norm", [
    (1, 8, 2, 128, 128, 3, True, True), (1, 5, 1, 64, 64, 2, False, True), (3, 1, 1, 64, 16, 3, True, True),
    (17, 4, 1, 128, 64, 4, True, True), (33, 20, 4, 128, 96, 3, False, False), (130, 3, 3, 64, 48, 1, True, True),
    (9000, 2, 1, 64, 32, 3, False, True), (257, 32, 8, 128, 112, 3, True, True)])
def test_against_oracle(t, hq, hkv, d, rot, axes, packed, norm, kind, interleaved):
    print(f"\n[case] axes t={t} {hq}q/{hkv}kv d={d} rot={rot} axes={axes} {kind}", flush=True)
    q, k, v, w, pos, cs = _inputs(t, hq, hkv, d, rot, axes, packed, seed=t + d)
    w = w if norm else [None, None]
    axis_of = _axis_of(kind, rot, axes)
    qo, ko, vo = cwlib.qk_norm_rope_axes(q, k, cs, pos, axis_of, q_weight=w[0], k_weight=w[1], eps=EPS, interleaved=interleaved, v=v)
    torch.cuda.synchronize()
    _near(qo, q, w[0], cs, pos, axis_of, interleaved, "q")
    _near(ko, k, w[1], cs, pos, axis_of, interleaved, "k")
    assert torch.equal(vo, v)
    # one position on all axes: the call without axes, bit for bit
    same = pos[:1].expand(axes, t).contiguous()
    got = cwlib.qk_norm_rope_axes(q, k, cs, same, axis_of, q_weight=w[0], k_weight=w[1], eps=EPS, interleaved=interleaved)
    want = cwlib.qk_norm_rope(q, k, cs, pos[0].contiguous(), q_weight=w[0], k_weight=w[1], eps=EPS, interleaved=interleaved)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dt", ["bf16", "fp8"])
@pytest.mark.parametrize("d,page,hq,hkv", [(128, 16, 8, 2), (64, 64, 5, 1), (128, 64, 4, 4), (64, 16, 20, 10)])
def test_pages_are_those_of_the_page_write(dt, d, page, hq, hkv):
    print(f"\n[case] axes page write {dt} d={d} page={page}", flush=True)
    lp, ls, num_pages = [0, 37, 64, 5], [19, 1, 70, 0], 40
    t = sum(ls)
    q, k, v, w, pos, cs = _inputs(t, hq, hkv, d, d, 3, True, seed=d + page)
    gen = torch.Generator(device="cuda").manual_seed(9)
    if dt == "fp8":
        pools = [torch.randint(0, 256, (num_pages, hkv, page, d), generator=gen, device="cuda", dtype=torch.uint8) for _ in "kv"]
        scales = [torch.rand(num_pages, hkv, generator=gen, device="cuda") * 0.02 + 0.001 for _ in "kv"]
    else:
        pools = [torch.randn(num_pages, hkv, page, d, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in "kv"]
        scales = [None, None]
    table = torch.randperm(num_pages, generator=gen, device="cuda").to(torch.int32)[:36].view(4, 9).contiguous()
    want = [x.clone() for x in pools]
    slots = torch.tensor([int(table[b, p // page]) * page + p % page for b in range(4) for p in range(lp[b], lp[b] + ls[b])],
                         dtype=torch.int64, device="cuda")
    qo, ko, vo = cwlib.qk_norm_rope_axes(q, k, cs, pos, _axis_of("runs", d, 3), q_weight=w[0], k_weight=w[1], v=v,
                                         k_pool=pools[0], v_pool=pools[1], slots=slots, k_scale=scales[0], v_scale=scales[1])
    cwlib.kv_write_pages(ko, vo, want[0], want[1], table, lp, ls, k_scale=scales[0], v_scale=scales[1])
    torch.cuda.synchronize()
    raw = lambda x: x.view(torch.uint8)
    assert torch.equal(vo, v) and torch.equal(raw(pools[0]), raw(want[0])) and torch.equal(raw(pools[1]), raw(want[1]))


def test_padding_tokens():
    """Nothing is written of a token one of whose positions lies outside, on whichever axis."""
    print("\n[case] axes padding", flush=True)
    t, hq, hkv, d, page = 12, 4, 2, 64, 16
    q, k, v, w, pos, cs = _inputs(t, hq, hkv, d, d, 4, False, seed=4, positions=100)
    pos[0, 3], pos[1, 5], pos[2, 7], pos[3, 11] = -1, 100, -(1 << 31), (1 << 31) - 1
    pools = [torch.full((2, hkv, page, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    outs = [torch.full((t, h, d), 3.0, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv)]
    axis_of = [0] * 32  # (also a position that no pair follows counts)
    cwlib.qk_norm_rope_axes(q, k, cs, pos, axis_of, v=v, k_pool=pools[0], v_pool=pools[1],
                            slots=torch.arange(t, dtype=torch.int64, device="cuda"), q_out=outs[0], k_out=outs[1], v_out=outs[2])
    torch.cuda.synchronize()
    good = [i for i in range(t) if i not in (3, 5, 7, 11)]
    for i in (3, 5, 7, 11):
        assert all(bool((o[i] == 3.0).all()) for o in outs) and bool((pools[0][0, :, i] == 7.0).all())
    _near(outs[0][good], q[good], None, cs, pos[:, good], axis_of, False, "tokens with positions")
    for pool, o in zip(pools, outs[1:]):
        for i in good:
            assert torch.equal(pool[0, :, i], o[i])


def test_in_place_other_stream_and_replays():
    print("\n[case] axes in place, graph", flush=True)
    q, k, v, w, pos, cs = _inputs(70, 8, 2, 128, 128, 3, False, seed=8)
    axis_of = _axis_of("turns", 128, 3)
    want = cwlib.qk_norm_rope_axes(q, k, cs, pos, axis_of, q_weight=w[0], k_weight=w[1], v=v)
    outs = [torch.empty_like(x) for x in want]
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        cwlib.qk_norm_rope_axes(q, k, cs, pos, axis_of, q_weight=w[0], k_weight=w[1], v=v, q_out=outs[0], k_out=outs[1], v_out=outs[2])
    for _ in range(3):
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    with torch.cuda.stream(s):
        got = cwlib.qk_norm_rope_axes(q, k, cs, pos, axis_of, q_weight=w[0], k_weight=w[1], v=v, q_out=q, k_out=k, v_out=v)
    torch.cuda.synchronize()
    assert got[0] is q and all(torch.equal(a, b) for a, b in zip(got, want))

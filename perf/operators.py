"""The operators around a serving step of a model whose layers use normalised, rotated
queries and keys and differential attention over the paged cache, as measurable cases.

A case is a dict of plain values; `op` says which operator:

  tables  build_step_tables: block-table entries of a step's new pages, and of every new
          token its sequence, position and pool slot, from lengths that lie on the GPU
  rope    qk_norm_rope: the RMS norm of every query and key head with the position
          rotation, and (with `pool`) the new K/V written into their pool slots
  diff    diff_attention: the difference of two softmax maps over a paged cache, prompts
          and chunks of new tokens mixed with single tokens, each head's result normed

Sequence lengths belong to the case (`lens_seed`); the data come from prepare's seed.
`own` False: the plain forms in elementary torch operations; True: the library's calls.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"

MAX_FLOPS = 6.8e12  # of a drawn diff case, below what `session` needs
MAX_KEYS = 1 << 20  # cached keys of a drawn diff case
EPS = 1e-5


def _tables(name, *, seqs, pre_hi, suf_hi, singles, page=16, spare=1.25, pad=0, lens_seed=1):
    """`singles`: share of sequences with one new token; `spare`: free pages per page
    needed (below 1 the list runs out); `pad`: tokens of the arrays behind the last one."""
    return {"name": name, "op": "tables", "seqs": seqs, "pre_hi": pre_hi, "suf_hi": suf_hi, "singles": singles,
            "page": page, "spare": spare, "pad": pad, "lens_seed": lens_seed}


def _rope(name, *, tokens, hq=32, hkv=8, d=128, rot=128, interleaved=False, norm=True, packed=True,
          pool="bf16", page=16, pos_hi=32768):
    """`packed`: q, k and v are columns of one projection's output; `pool`: "" for no page write."""
    return {"name": name, "op": "rope", "tokens": tokens, "hq": hq, "hkv": hkv, "d": d, "rot": rot,
            "interleaved": interleaved, "norm": norm, "packed": packed, "pool": pool, "page": page, "pos_hi": pos_hi}


def _diff(name, *, pairs=4, g=4, d=128, page=16, dtype="bf16", norm=True, decodes=0, dec_lo=0, dec_hi=0, extends=0,
          pre_lo=0, pre_hi=0, suf_lo=0, suf_hi=0, lens_seed=1):
    """`pairs`: pairs of key heads (a pair shares a value head of twice the width); `g`: query pairs of each."""
    return {"name": name, "op": "diff", "pairs": pairs, "g": g, "d": d, "page": page, "dtype": dtype, "norm": norm,
            "decodes": decodes, "dec_lo": dec_lo, "dec_hi": dec_hi, "extends": extends, "pre_lo": pre_lo,
            "pre_hi": pre_hi, "suf_lo": suf_lo, "suf_hi": suf_hi, "lens_seed": lens_seed}


def listed():
    return [
        # eight sessions generating: the tables of the smallest steps, launch latency counts
        _tables("tables_decodes", seqs=8, pre_hi=20000, suf_hi=1, singles=1.0, lens_seed=21),
        # chunked prefill: 31 chunks of up to 512 tokens among 33 decodes, arrays padded for a captured graph
        _tables("tables_chunked", seqs=64, pre_hi=32768, suf_hi=512, singles=0.5, pad=1024, lens_seed=22),
        # a node's whole queue: thousands of sessions, most of them generating, 64-token pages
        _tables("tables_queue", seqs=3500, pre_hi=65536, suf_hi=700, singles=0.75, page=64, lens_seed=23),
        # one session generating: one token through norm, rotation and page write
        _rope("rope_one", tokens=1),
        # 96 sessions generating on a model with 64-wide heads, half of each rotated in pairs of neighbours, fp8 pages
        _rope("rope_decodes_fp8", tokens=96, hq=16, hkv=4, d=64, rot=32, interleaved=True, pool="fp8", page=64),
        # an odd chunk of a prompt, queries and keys only, tensors of their own
        _rope("rope_chunk", tokens=1531, hq=64, hkv=8, packed=False, pool=""),
        # a full prefill batch into bf16 pages
        _rope("rope_prefill", tokens=16384),
        # one session generating: differential attention of one token over 1700 cached ones
        _diff("diff_one", decodes=1, dec_lo=1700, dec_hi=1700),
        # 48 sessions generating over fp8 pages
        _diff("diff_decodes_fp8", dtype="fp8", decodes=48, dec_lo=2048, dec_hi=32768, lens_seed=24),
        # chunked prefill on a model with 64-wide key heads: ragged chunks beside decodes, no norm
        _diff("diff_chunked_d64", pairs=8, g=2, d=64, page=64, norm=False, decodes=24, dec_lo=200, dec_hi=6000, extends=9,
              pre_lo=0, pre_hi=12000, suf_lo=37, suf_hi=1300, lens_seed=25),
        # an agent turn: 1024 new tokens on a 16384-token prefix
        _diff("diff_turn", extends=1, pre_lo=16384, pre_hi=16384, suf_lo=1024, suf_hi=1024),
        # a long session coming back with 4096 new tokens on 32768 cached ones
        _diff("diff_session", pairs=8, extends=1, pre_lo=32768, pre_hi=32768, suf_lo=4096, suf_hi=4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above."""
    op = rng.choice(["tables", "rope", "rope", "diff", "diff", "diff"])
    if op == "tables":
        while True:
            case = _tables("", seqs=_log_int(rng, 1, 4096), pre_hi=_log_int(rng, 1, 65536), suf_hi=_log_int(rng, 1, 4096),
                           singles=rng.choice([0.0, 0.5, 0.9, 1.0]), page=rng.choice([16, 64]),
                           spare=rng.choice([1.0, 1.25, 2.0, 0.6]), pad=rng.choice([0, _log_int(rng, 1, 2000)]),
                           lens_seed=rng.randrange(1, 1 << 30))
            if work(case)["bytes"] <= 8e6:
                break
    elif op == "rope":
        while True:
            hq, hkv = rng.choice([(32, 8), (64, 8), (32, 4), (16, 2), (4, 1), (16, 16), (20, 4)])
            d = rng.choice([128, 128, 64])
            case = _rope("", tokens=_log_int(rng, 1, 16384), hq=hq, hkv=hkv, d=d, rot=rng.choice([d, d, d // 2, 16]),
                         interleaved=rng.random() < 0.4, norm=rng.random() < 0.8, packed=rng.random() < 0.7,
                         pool=rng.choice(["", "bf16", "fp8"]), page=rng.choice([16, 64]), pos_hi=_log_int(rng, 100, 131072))
            if work(case)["bytes"] <= 4.5e8:
                break
    else:
        while True:
            pairs, g = rng.choice([(4, 4), (4, 4), (8, 2), (2, 8), (1, 4), (8, 1), (4, 5), (1, 16)])
            case = _diff("", pairs=pairs, g=g, d=rng.choice([128, 128, 64]), page=rng.choice([16, 64]),
                         dtype=rng.choice(["bf16", "bf16", "fp8"]), norm=rng.random() < 0.7, lens_seed=rng.randrange(1, 1 << 30))
            what = rng.choice(["decode", "extend", "mixed"])
            if what != "extend":
                case["decodes"] = _log_int(rng, 1, 64)
                case["dec_hi"] = _log_int(rng, 100, 65536)
                case["dec_lo"] = int(case["dec_hi"] * rng.uniform(0.0, 1.0))
            if what != "decode":
                case["extends"] = _log_int(rng, 1, 16)
                case["pre_hi"] = rng.choice([0, _log_int(rng, 100, 65536)])
                case["pre_lo"] = int(case["pre_hi"] * rng.uniform(0.0, 1.0))
                case["suf_hi"] = _log_int(rng, 2, 4096)
                case["suf_lo"] = max(2, int(case["suf_hi"] * rng.uniform(0.03, 1.0)))
            lp, ls = _lens(case)
            if work(case)["flops"] <= MAX_FLOPS and int((lp + ls).sum()) <= MAX_KEYS:
                break
    del case["name"]
    return case


# ---------------------------------------------------------------------------- sizes


def _lens(case):
    """Prefix and suffix lengths of every sequence, int64, in a mixed order."""
    rng = np.random.default_rng(case["lens_seed"])
    if case["op"] == "tables":
        n = case["seqs"]
        lp = rng.integers(0, case["pre_hi"] + 1, size=n)
        ls = rng.integers(0, case["suf_hi"] + 1, size=n)  # a sequence may have no new token in this step
        ls[rng.random(n) < case["singles"]] = 1
        return lp, ls
    nd, ne = case["decodes"], case["extends"]
    lp = np.concatenate([rng.integers(case["dec_lo"], case["dec_hi"] + 1, size=nd),
                         rng.integers(case["pre_lo"], case["pre_hi"] + 1, size=ne)])
    ls = np.concatenate([np.ones(nd, dtype=np.int64), rng.integers(case["suf_lo"], case["suf_hi"] + 1, size=ne)])
    order = rng.permutation(nd + ne)
    return lp[order], ls[order]


def _pages(lp, ls, p):
    held = (lp + p - 1) // p
    return held, (lp + ls + p - 1) // p


def work(case):
    if case["op"] == "tables":
        lp, ls = _lens(case)
        held, need = _pages(lp, ls, case["page"])
        tokens = int(ls.sum()) + case["pad"]
        # lengths read, free pages read and written to the table, per token three indices (4, 4 and 8 bytes); a token's
        # page is read from the table unless it is new
        old = int(((held > lp // case["page"]) & (ls > 0)).sum())
        return {"bytes": 12 * len(lp) + 8 * int((need - held).sum()) + 16 * tokens + 4 * old, "flops": 0}
    if case["op"] == "rope":
        t, hq, hkv, d = case["tokens"], case["hq"], case["hkv"], case["d"]
        heads = hq + hkv + (hkv if case["pool"] else 0)
        byts = 2 * t * heads * d * 2 + t * (4 + case["rot"] * 4)
        if case["pool"]:
            byts += t * (2 * hkv * d * (1 if case["pool"] == "fp8" else 2) + 8)
        return {"bytes": byts, "flops": t * (hq + hkv) * d * 7}
    pairs, g, d, p = case["pairs"], case["g"], case["d"], case["page"]
    fp8 = case["dtype"] == "fp8"
    lp, ls = _lens(case)
    new = int(ls.sum())
    n_pages = int(((lp + p - 1) // p).sum())
    kv = 4 * int(lp.sum()) * pairs * d * (1 if fp8 else 2) + n_pages * (4 + (16 * pairs if fp8 else 0))
    byts = kv + 4 * new * pairs * d * 2 + 2 * new * pairs * g * 2 * d * 2
    seen = int((ls * lp + ls * (ls + 1) // 2).sum())
    return {"bytes": byts, "flops": 12 * d * pairs * g * seen}


# ---------------------------------------------------------------------------- inputs


class _State:
    pass


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.bfloat16)


def _codes(x, scale):
    """e4m3fn codes of x / scale, as bytes."""
    return (x / scale).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


def _pool(gen, pages, heads, p, d, dtype, scale):
    if dtype != "fp8":
        return _normal(gen, pages, heads, p, d)
    return _codes(torch.randn(pages, heads, p, d, generator=gen, device=DEV), scale[:, :, None, None])


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = _State()
    s.case, s.op = case, case["op"]
    return {"tables": _prepare_tables, "rope": _prepare_rope, "diff": _prepare_diff}[s.op](case, gen, s)


def _prepare_tables(case, gen, s):
    lp, ls = _lens(case)
    held, need = _pages(lp, ls, case["page"])
    new, n = int((need - held).sum()), len(lp)
    total = int(held.sum()) + max(1, int(new * case["spare"])) + 7
    ids = torch.randperm(total, generator=gen, device=DEV).to(torch.int32)
    s.stride = int(need.max()) + 3
    s.table = torch.full((n, s.stride), 1 << 30, dtype=torch.int32, device=DEV)
    old = torch.arange(s.stride, device=DEV)[None, :] < torch.from_numpy(held).to(DEV)[:, None]
    s.table[old] = ids[:int(held.sum())]
    s.free = ids[int(held.sum()):].clone()
    s.lp = torch.from_numpy(lp.astype(np.int32)).to(DEV)
    s.ls = torch.from_numpy(ls.astype(np.int32)).to(DEV)
    s.tokens = max(1, int(ls.sum()) + case["pad"])
    s.page = case["page"]
    s.cu = torch.empty(n + 1, dtype=torch.int32, device=DEV)
    s.seq = torch.empty(s.tokens, dtype=torch.int32, device=DEV)
    s.pos = torch.empty(s.tokens, dtype=torch.int32, device=DEV)
    s.slot = torch.empty(s.tokens, dtype=torch.int64, device=DEV)
    s.info = torch.empty(3, dtype=torch.int64, device=DEV)
    return s


def _angles(rows, rot):
    """cos and sin of every position's rotations, fp32 [rows, rot] (the cosines first)."""
    freq = 10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
    a = torch.arange(rows, device=DEV, dtype=torch.float64)[:, None] * freq[None, :]
    return torch.cat([a.cos(), a.sin()], 1).float()


def _prepare_rope(case, gen, s):
    t, hq, hkv, d, p = case["tokens"], case["hq"], case["hkv"], case["d"], case["page"]
    if case["packed"]:
        x = _normal(gen, t, hq + 2 * hkv, d)
        s.q, s.k, s.v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    else:
        s.q, s.k, s.v = _normal(gen, t, hq, d), _normal(gen, t, hkv, d), _normal(gen, t, hkv, d)
    s.wq = s.wk = None
    if case["norm"]:
        s.wq = torch.rand(d, generator=gen, device=DEV) + 0.5
        s.wk = torch.rand(d, generator=gen, device=DEV) + 0.5
    s.table = _angles(case["pos_hi"], case["rot"])
    s.pos = torch.randint(0, case["pos_hi"], (t,), generator=gen, device=DEV, dtype=torch.int32)
    s.q_out, s.k_out, s.v_out = (torch.empty(t, h, d, dtype=torch.bfloat16, device=DEV) for h in (hq, hkv, hkv))
    s.k_pool = s.v_pool = s.slots = s.k_scale = s.v_scale = None
    if case["pool"]:
        pages = (t + p - 1) // p + 5
        if case["pool"] == "fp8":
            s.k_scale = torch.rand(pages, hkv, generator=gen, device=DEV) * 0.09 + 0.01
            s.v_scale = torch.rand(pages, hkv, generator=gen, device=DEV) * 0.09 + 0.01
        s.k_pool = _pool(gen, pages, hkv, p, d, case["pool"], s.k_scale)
        s.v_pool = _pool(gen, pages, hkv, p, d, case["pool"], s.v_scale)
        # runs of consecutive slots within pages in any order, as sequences have them
        s.slots = (torch.randperm(pages, generator=gen, device=DEV)[:, None] * p + torch.arange(p, device=DEV)).reshape(-1)[:t].contiguous()
    return s


def _prepare_diff(case, gen, s):
    pairs, g, d, p = case["pairs"], case["g"], case["d"], case["page"]
    lp, ls = _lens(case)
    s.lp, s.ls = lp.astype(np.int32), ls.astype(np.int32)
    need = _pages(lp, ls, p)[1]
    pages = int(need.sum()) * 5 // 4 + 8
    s.k_scale = s.v_scale = None
    if case["dtype"] == "fp8":
        s.k_scale = torch.rand(pages, 2 * pairs, generator=gen, device=DEV) * 0.09 + 0.01
        s.v_scale = torch.rand(pages, 2 * pairs, generator=gen, device=DEV) * 0.09 + 0.01
    s.k_pool = _pool(gen, pages, 2 * pairs, p, d, case["dtype"], s.k_scale)
    s.v_pool = _pool(gen, pages, 2 * pairs, p, d, case["dtype"], s.v_scale)
    ids = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32)
    n, t = len(lp), int(ls.sum())
    s.table = torch.zeros(n, max(1, int(need.max())), dtype=torch.int32, device=DEV)
    at = 0
    for b in range(n):
        s.table[b, :int(need[b])] = ids[at:at + int(need[b])]
        at += int(need[b])
    s.k_new, s.v_new = _normal(gen, t, 2 * pairs, d), _normal(gen, t, 2 * pairs, d)
    # heads range from nearly uniform attention to peaked
    sharp = torch.rand(1, 2 * pairs * g, 1, generator=gen, device=DEV) * 1.5 + 0.5
    s.q = (_normal(gen, t, 2 * pairs * g, d) * sharp).to(torch.bfloat16)
    s.lam = torch.rand(pairs * g, generator=gen, device=DEV) * 0.6 + 0.2
    s.weight = torch.rand(2 * d, generator=gen, device=DEV) + 0.5 if case["norm"] else None
    s.after = 0.4 if case["norm"] else 1.0  # one minus the layer's initial weight of the second map
    s.scale = 1.0 / math.sqrt(d)
    s.out, s.ws = torch.empty(t, pairs * g, 2 * d, dtype=torch.bfloat16, device=DEV), None
    return s


# ---------------------------------------------------------------------------- one pass


def run(s):
    return {"tables": _run_tables, "rope": _run_rope, "diff": _run_diff}[s.op](s)


def _run_tables(s):
    if own:
        import paper_2606_16824_amd as cw

        cw.build_step_tables(s.lp, s.ls, s.free, s.table, s.page, s.tokens, cu_rows=s.cu, seq_ids=s.seq, positions=s.pos,
                             slots=s.slot, info=s.info)
        return {"table": s.table, "cu": s.cu, "seq": s.seq, "pos": s.pos, "slot": s.slot, "info": s.info}
    p = s.page
    lp, ls = s.lp.long(), s.ls.long()
    held, need = (lp + p - 1) // p, (lp + ls + p - 1) // p
    end, taken = torch.cumsum(ls, 0), torch.cumsum(need - held, 0)
    first = taken - (need - held)
    col = torch.arange(s.stride, device=DEV)[None, :]
    at = first[:, None] + col - held[:, None]
    fresh = torch.where(at < s.free.numel(), s.free[at.clamp(0, s.free.numel() - 1)], -1)
    s.table.copy_(torch.where((col >= held[:, None]) & (col < need[:, None]), fresh, s.table))
    t = torch.arange(s.tokens, device=DEV)
    seq = torch.searchsorted(end, t, right=True)
    real = t < end[-1]
    b = seq.clamp(max=lp.numel() - 1)
    pos = lp[b] + t - (end - ls)[b]
    page = s.table[b, (pos // p).clamp(0, s.stride - 1)].long()
    s.cu.copy_(torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), end]))
    s.seq.copy_(torch.where(real, seq, -1))
    s.pos.copy_(torch.where(real, pos, -1))
    s.slot.copy_(torch.where(real & (page >= 0), page * p + pos % p, -1))
    s.info.copy_(torch.stack([taken[-1], end[-1], (need > s.stride).sum()]))
    return {"table": s.table, "cu": s.cu, "seq": s.seq, "pos": s.pos, "slot": s.slot, "info": s.info}


def _norm_rotate(x, w, cos, sin, rot, interleaved):
    """One head row in 32 bits: RMS norm with weights (if any), then the rotation of its first `rot` elements."""
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., rot:]], -1).to(torch.bfloat16)


def _run_rope(s):
    c = s.case
    if own:
        import paper_2606_16824_amd as cw

        if c["pool"]:
            cw.qk_norm_rope(s.q, s.k, s.table, s.pos, q_weight=s.wq, k_weight=s.wk, eps=EPS, interleaved=c["interleaved"],
                            v=s.v, k_pool=s.k_pool, v_pool=s.v_pool, slots=s.slots, k_scale=s.k_scale, v_scale=s.v_scale,
                            q_out=s.q_out, k_out=s.k_out, v_out=s.v_out)
        else:
            cw.qk_norm_rope(s.q, s.k, s.table, s.pos, q_weight=s.wq, k_weight=s.wk, eps=EPS, interleaved=c["interleaved"],
                            q_out=s.q_out, k_out=s.k_out)
    else:
        cs = s.table[s.pos.long()]
        cos, sin = (x[:, None, :] for x in cs.chunk(2, 1))
        s.q_out.copy_(_norm_rotate(s.q, s.wq, cos, sin, c["rot"], c["interleaved"]))
        s.k_out.copy_(_norm_rotate(s.k, s.wk, cos, sin, c["rot"], c["interleaved"]))
        if c["pool"]:
            s.v_out.copy_(s.v)
            pg, at = s.slots // c["page"], s.slots % c["page"]
            if c["pool"] == "fp8":
                s.k_pool[pg, :, at] = _codes(s.k_out.float(), s.k_scale[pg][:, :, None])
                s.v_pool[pg, :, at] = _codes(s.v_out.float(), s.v_scale[pg][:, :, None])
            else:
                s.k_pool[pg, :, at] = s.k_out
                s.v_pool[pg, :, at] = s.v_out
    if not c["pool"]:
        return {"q": s.q_out, "k": s.k_out}
    kind = torch.float8_e4m3fn if c["pool"] == "fp8" else torch.bfloat16
    return {"q": s.q_out, "k": s.k_out, "v": s.v_out, "k_pool": s.k_pool.view(kind), "v_pool": s.v_pool.view(kind)}


def _cached(pool, scale, ids, lp):
    """The first lp rows of a sequence's pages in 32 bits, [heads, lp, d]."""
    x = pool[ids].float() if scale is None else pool[ids].view(torch.float8_e4m3fn).float() * scale[ids][:, :, None, None]
    return x.transpose(0, 1).reshape(x.shape[1], -1, x.shape[3])[:, :lp]


def _run_diff(s):
    c = s.case
    if own:
        import paper_2606_16824_amd as cw

        if s.ws is None:  # a user's program keeps one for the lengths that it serves
            n_ws = cw.diff_workspace_bytes(s.lp, s.ls, c["pairs"], c["g"], c["d"], c["page"], c["dtype"])
            s.ws = torch.empty(max(256, n_ws), dtype=torch.uint8, device=DEV)
        cw.diff_attention(s.q, s.k_new, s.v_new, s.k_pool, s.v_pool, s.table, s.lp, s.ls, c["g"], s.scale, s.lam,
                          k_scale=s.k_scale, v_scale=s.v_scale, norm_weight=s.weight, norm_eps=EPS, out_scale=s.after,
                          out=s.out, workspace=s.ws)
        return {"out": s.out}
    pairs, g, d, p = c["pairs"], c["g"], c["d"], c["page"]
    lam = s.lam.view(pairs, 1, g, 1)
    cu = 0
    for lp, ls, row in zip(s.lp.tolist(), s.ls.tolist(), s.table):
        ids, n = row[:(lp + p - 1) // p].long(), lp + ls
        k = torch.cat([_cached(s.k_pool, s.k_scale, ids, lp), s.k_new[cu:cu + ls].float().transpose(0, 1)], 1)
        v = torch.cat([_cached(s.v_pool, s.v_scale, ids, lp), s.v_new[cu:cu + ls].float().transpose(0, 1)], 1)
        v = v.view(pairs, 2, n, d).transpose(1, 2).reshape(pairs, n, 2 * d)
        step = max(1, (1 << 28) // (2 * pairs * g * n))
        for t0 in range(0, ls, step):
            t1 = min(ls, t0 + step)
            q = s.q[cu + t0:cu + t1].float().view(-1, pairs, g, 2, d).permute(1, 3, 0, 2, 4).reshape(2 * pairs, -1, d)
            x = torch.matmul(q, k.transpose(1, 2).contiguous()).mul_(s.scale).view(2 * pairs, t1 - t0, g, n)
            hide = torch.arange(n, device=DEV)[None, :] > lp + torch.arange(t0, t1, device=DEV)[:, None]
            x.masked_fill_(hide[None, :, None, :], -math.inf)
            x.sub_(x.amax(-1, keepdim=True)).exp_()
            x.div_(x.sum(-1, keepdim=True))
            x = x.view(pairs, 2, t1 - t0, g, n)
            x = x[:, 0] - lam * x[:, 1]
            o = torch.matmul(x.reshape(pairs, -1, n), v).view(pairs, t1 - t0, g, 2 * d)
            if s.weight is not None:
                o = o * torch.rsqrt(o.square().mean(-1, keepdim=True) + EPS) * s.weight
            s.out[cu + t0:cu + t1] = (o * s.after).permute(1, 0, 2, 3).reshape(t1 - t0, pairs * g, 2 * d).to(torch.bfloat16)
        cu += ls
    return {"out": s.out}


# ---------------------------------------------------------------------------- what is right


def exact(case, seed):
    """The definitions in 64 bits. Pages move or round values and tables are whole numbers: those have no such value."""
    if case["op"] == "tables":
        return None
    s = prepare(case, seed)
    return _exact_rope(case, s) if case["op"] == "rope" else _exact_diff(case, s)


def _exact_rope(case, s):
    rot = case["rot"]
    half = rot // 2
    i = torch.arange(half, device=DEV)
    lo, hi = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half)
    angle = s.table[s.pos.long()].double()
    cos, sin = angle[:, None, :half], angle[:, None, half:]
    res = {}
    for name, x, w in (("q", s.q, s.wq), ("k", s.k, s.wk)):
        y = x.double()
        if w is not None:
            y = y / (y.pow(2).sum(-1, keepdim=True) / case["d"] + EPS).sqrt() * w.double()
        z = y.clone()
        z[..., lo] = y[..., lo] * cos - y[..., hi] * sin
        z[..., hi] = y[..., lo] * sin + y[..., hi] * cos
        res[name] = z
    if case["pool"]:
        res.update(v=s.v.double(), k_pool=None, v_pool=None)
    return res


def _exact_diff(case, s):
    pairs, g, d, p = case["pairs"], case["g"], case["d"], case["page"]
    out = torch.empty(s.out.shape, dtype=torch.float64, device=DEV)
    cu = np.concatenate([[0], np.cumsum(s.ls)]).tolist()
    key = torch.arange(int((s.lp.astype(np.int64) + s.ls).max()), device=DEV)
    for b in range(len(s.lp)):
        lp, ls = int(s.lp[b]), int(s.ls[b])
        n = lp + ls
        slot = s.table[b, key[:lp] // p].long() * p + key[:lp] % p

        def rows(pool, scale, new, head):
            old = pool[slot // p, head, slot % p]
            old = old.double() if scale is None else old.view(torch.float8_e4m3fn).double() * scale[slot // p, head].double()[:, None]
            return torch.cat([old, new[cu[b]:cu[b] + ls, head].double()])

        step = max(1, (1 << 27) // n)
        for j in range(pairs):
            value = torch.cat([rows(s.v_pool, s.v_scale, s.v_new, 2 * j + i) for i in (0, 1)], 1)
            keys = [rows(s.k_pool, s.k_scale, s.k_new, 2 * j + i).t().contiguous() for i in (0, 1)]
            for h in range(j * g, (j + 1) * g):
                for t0 in range(0, ls, step):
                    t1 = min(ls, t0 + step)
                    seen = key[None, :n] <= lp + torch.arange(t0, t1, device=DEV)[:, None]
                    o = 0.0
                    for i, weight in ((0, 1.0), (1, -s.lam[h].double())):
                        x = torch.mm(s.q[cu[b] + t0:cu[b] + t1, 2 * h + i].double(), keys[i]) * s.scale
                        x = x.masked_fill(~seen, -math.inf)
                        e = (x - x.amax(1, keepdim=True)).exp()
                        o = o + weight * torch.mm(e, value) / e.sum(1, keepdim=True)
                    if s.weight is not None:
                        o = o / (o.pow(2).mean(1, keepdim=True) + EPS).sqrt() * s.weight.double()
                    out[cu[b] + t0:cu[b] + t1, h] = o * s.after
    return {"out": out}

"""What a layer does around its attention, by its plain definition (float64, or integers).

Test infrastructure (see the package docstring): not used by the library.

step_tables      new block-table entries and the token arrays of a serving step
norm_rotate      RMS norm of head rows and their position rotation
diff_attention   the difference of two softmax maps per query pair over a paged cache:
                 query heads 2h, 2h+1 against key heads 2j, 2j+1 of pair j = h // G, the value
                 of pair j being value heads 2j and 2j+1 side by side
axis_angles      cos and sin of every token's rotated pairs where the pairs follow several position axes
residual_norm    the norm of a block's output, its gate, the residual stream and the next norm
shaped_attention softmax attention over a paged cache with capped, biased and masked scores
"""
from __future__ import annotations

from typing import Optional

import numpy as np

from .codecs import bf16_bits_to_f64
from .paged_attention import PagedInputs, gather_sequence_kv


def step_tables(prefix_lens, suffix_lens, free_pages, block_table, page_size: int, max_tokens: int):
    """(block_table, cu_rows, seq_ids, positions, slots, info) after the step, one entry at a time."""
    table = np.array(block_table, dtype=np.int64)
    stride = table.shape[1]
    lp = [max(int(x), 0) for x in prefix_lens]
    ls = [max(int(x), 0) for x in suffix_lens]
    pages = over = 0
    cu, seq, pos, slot = [0], [], [], []
    for b in range(len(lp)):
        held, need = -(-lp[b] // page_size), -(-(lp[b] + ls[b]) // page_size)
        over += need > stride
        for col in range(min(held, stride), min(need, stride)):
            table[b, col] = free_pages[pages] if pages < len(free_pages) else -1
            pages += 1
        for i in range(ls[b]):
            at = lp[b] + i
            page = table[b, at // page_size] if at // page_size < stride else -1
            seq.append(b)
            pos.append(at)
            slot.append(page * page_size + at % page_size if page >= 0 else -1)
        cu.append(cu[-1] + ls[b])

    def fit(x):
        return np.array((x + [-1] * max_tokens)[:max_tokens], dtype=np.int64)

    return table, np.array(cu), fit(seq), fit(pos), fit(slot), np.array([pages, cu[-1], over])


def norm_rotate(x: np.ndarray, weight: Optional[np.ndarray], eps: float, cos: np.ndarray, sin: np.ndarray,
                interleaved: bool) -> np.ndarray:
    """x float64 [T, H, D]; weight [D] or None; cos, sin float64 [T, R / 2]."""
    y = np.array(x, dtype=np.float64)
    if weight is not None:
        y = y / np.sqrt((y * y).mean(axis=-1, keepdims=True) + eps) * weight.astype(np.float64)
    half = cos.shape[1]
    out = y.copy()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        c, s = cos[:, i, None], sin[:, i, None]
        out[:, :, a] = y[:, :, a] * c - y[:, :, b] * s
        out[:, :, b] = y[:, :, b] * c + y[:, :, a] * s
    return out


def diff_attention(inp: PagedInputs, lam: np.ndarray, weight: Optional[np.ndarray] = None, eps: float = 0.0,
                   out_scale: float = 1.0):
    """(out [T, Hp, 2D], terms): terms holds, for error bounds, `x` (the difference before the
    norm), `mass` (sum of |weights| |values| of both maps) and `scores` (per row, the largest
    scale * sum |q| |k| of a visible key of either map)."""
    total, heads, d = inp.q.shape
    hp, g = heads // 2, inp.gqa_group
    x = np.zeros((total, hp, 2 * d))
    mass, scores = np.zeros_like(x), np.zeros((total, hp, 1))
    cu = inp.cu()
    q = bf16_bits_to_f64(inp.q)
    for b in range(len(inp.prefix_lens)):
        k, v = gather_sequence_kv(inp, b)
        lp, ls = int(inp.prefix_lens[b]), int(inp.suffix_lens[b])
        if ls == 0:
            continue
        rows = slice(int(cu[b]), int(cu[b]) + ls)
        seen = np.arange(lp + ls)[None, :] <= lp + np.arange(ls)[:, None]
        for h in range(hp):
            j = h // g
            value = np.concatenate([v[:, 2 * j], v[:, 2 * j + 1]], axis=1)
            for m, sign in ((0, 1.0), (1, -float(lam[h]))):
                qh, kh = q[rows, 2 * h + m], k[:, 2 * j + m]
                s = np.where(seen, inp.softmax_scale * (qh @ kh.T), -np.inf)
                p = np.exp(s - s.max(axis=1, keepdims=True))
                p /= p.sum(axis=1, keepdims=True)
                x[rows, h] += sign * (p @ value)
                mass[rows, h] += abs(sign) * (p @ np.abs(value))
                big = np.where(seen, inp.softmax_scale * (np.abs(qh) @ np.abs(kh).T), 0.0).max(axis=1)
                scores[rows, h, 0] = np.maximum(scores[rows, h, 0], big)
    out = x
    if weight is not None:
        out = x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps) * weight.astype(np.float64)
    return out * out_scale, {"x": x, "mass": mass, "scores": scores}


def axis_angles(cos_sin: np.ndarray, positions: np.ndarray, axis_of):
    """(cos, sin) float64 [T, R / 2] from the table [positions, R], the positions [axes, T] and each pair's axis."""
    half = cos_sin.shape[1] // 2
    cos, sin = np.empty((positions.shape[1], half)), np.empty((positions.shape[1], half))
    for i in range(half):
        row = positions[axis_of[i]]
        cos[:, i], sin[:, i] = cos_sin[row, i], cos_sin[row, half + i]
    return cos, sin


def residual_norm(x, residual, post=None, gate=None, scale: float = 1.0, pre=None, eps: float = 0.0):
    """(residual, y) in float64, not rounded; y None without pre."""
    def normed(z, w):
        return z / np.sqrt((z * z).mean(axis=-1, keepdims=True) + eps) * np.asarray(w, dtype=np.float64)

    u = np.asarray(x, dtype=np.float64)
    u = u if post is None else normed(u, post)
    r = scale * np.asarray(residual, dtype=np.float64) + (u if gate is None else np.asarray(gate, dtype=np.float64) * u)
    return r, None if pre is None else normed(r, pre)


def shaped_attention(inp: PagedInputs, cap: float = 0.0, slopes: Optional[np.ndarray] = None, window: int = 0,
                     begins: Optional[np.ndarray] = None, full: Optional[np.ndarray] = None):
    """(out [T, Hq, D], lse [T, Hq], terms): terms holds, for error bounds, `mass` (sum of weights times
    |values|), `scores` (per row, the largest scale * sum |q| |k| of a visible key) and `bias` (per row, the
    largest |bias| of one).  A row that sees nothing: 0 and -inf."""
    total, hq, d = inp.q.shape
    g = inp.gqa_group
    out, lse = np.zeros((total, hq, d)), np.full((total, hq), -np.inf)
    mass, scores, biases = np.zeros_like(out), np.zeros((total, hq, 1)), np.zeros((total, hq, 1))
    cu = inp.cu()
    q = bf16_bits_to_f64(inp.q)
    for b in range(len(inp.prefix_lens)):
        k, v = gather_sequence_kv(inp, b)
        lp, ls = int(inp.prefix_lens[b]), int(inp.suffix_lens[b])
        for i in range(ls):
            row, p = int(cu[b]) + i, lp + i
            j = np.arange(lp + ls)
            seen = j <= p
            if full is not None:
                seen |= j < int(full[b])
            if window:
                seen &= j > p - window
            if begins is not None:
                seen &= j >= int(begins[row])
            j = j[seen]
            if len(j) == 0:
                continue
            for h in range(hq):
                kj, vj = k[j, h // g], v[j, h // g]
                x = inp.softmax_scale * (kj @ q[row, h])
                if cap:
                    x = cap * np.tanh(x / cap)
                away = np.zeros(len(j)) if slopes is None else float(slopes[h]) * np.abs(p - j)
                x = x - away
                top = x.max()
                w = np.exp(x - top)
                lse[row, h] = top + np.log(w.sum())
                w /= w.sum()
                out[row, h], mass[row, h] = w @ vj, w @ np.abs(vj)
                scores[row, h, 0] = (inp.softmax_scale * (np.abs(kj) @ np.abs(q[row, h]))).max()
                biases[row, h, 0] = np.abs(away).max()
    return out, lse, {"mass": mass, "scores": scores, "bias": biases}

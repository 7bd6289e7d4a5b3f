"""Differential attention of single tokens in 64 bits, but for one thing: the weights of the second
product are rounded to `terms` terms of a type.  For tests that tell how far that moves a result."""
import numpy as np
import torch

from oracle.codecs import bf16_bits_to_f64
from oracle.paged_attention import gather_sequence_kv


def _rounded(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).to(dtype).double().numpy()


def singles_with_rounded_weights(inp, lam, dtype, terms):
    """out [B, Hp, 2 D], stored as bf16; every suffix is one token."""
    heads, d, g = inp.q.shape[1], inp.q.shape[2], inp.gqa_group
    out = np.zeros((len(inp.prefix_lens), heads // 2, 2 * d))
    q = bf16_bits_to_f64(inp.q)
    for b in range(len(out)):
        k, v = gather_sequence_kv(inp, b)
        for h in range(heads // 2):
            j = h // g
            value = np.concatenate([v[:, 2 * j], v[:, 2 * j + 1]], axis=1)
            for m, sign in ((0, 1.0), (1, -float(lam[h]))):
                s = inp.softmax_scale * (k[:, 2 * j + m] @ q[b, 2 * h + m])
                p = 256.0 * np.exp(s - s.max())
                w = _rounded(p, dtype)
                if terms == 2:
                    w = w + _rounded(p - w, dtype)
                out[b, h] += sign * (w @ value) / p.sum()
    return _rounded(out, torch.bfloat16)

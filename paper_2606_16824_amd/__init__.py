"""Prefix-cached paged extend attention on MI355X: Python binding of libcw.so.

Thin argument marshalling over the C ABI of include/cw.h: every function
passes device pointers (``tensor.data_ptr()``), host length arrays and torch's
current HIP stream to the library, which runs the HIP kernels.  There is no
fallback: without the built library every call raises.

    extend_attention(q, k_new, v_new, k_pool, v_pool, block_table, prefix_lens,
                     suffix_lens, gqa_group, softmax_scale, k_scale=None,
                     v_scale=None, out=None, lse=None, workspace=None)
    decode_attention(q, k_new, v_new, k_pool, v_pool, block_table, prefix_lens,
                     gqa_group, softmax_scale, ...)
    kv_write_pages(k_new, v_new, k_pool, v_pool, block_table, prefix_lens,
                   suffix_lens, k_scale=None, v_scale=None, workspace=None)

and, of include/cw_layer.h, what a layer does around its attention: build_step_tables
(block table and slots from lengths on the GPU), qk_norm_rope and qk_norm_rope_axes (norm,
rotation by one or several position axes, and page write), residual_norm (the norms around the
residual stream), diff_attention (differential attention over pools of paired heads) and
shaped_attention (capped, biased and masked scores).

Page size and head dim are read from the pool shape [num_pages, Hkv, P, D];
an fp8 pool is a uint8 (or float8_e4m3fn) tensor of e4m3fn codes.

The C side sees only pointers, so the binding checks every tensor's dtype and
shape against the call's lengths before passing a pointer (ValueError on a
mismatch): block_table 2-D int32 with a row per sequence; q and out bf16
[T, Hkv*G, D]; k_new, v_new bf16 [T, Hkv, D]; lse fp32 [T, Hkv*G]; v_pool like
k_pool; fp8 scales fp32 [num_pages, Hkv] (and absent for bf16 pools); every
tensor on one GPU and contiguous.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional

import numpy as np
import torch

from . import _lib as L

__all__ = ["CWError", "init", "pinned_allocations", "arg_plan_calls", "extend_attention", "extend_attention_noalloc", "write_extend_attention", "decode_attention", "kv_write_pages",
           "extend_workspace_bytes", "decode_workspace_bytes", "write_pages_workspace_bytes",
           "set_tuning", "plan_items", "decode_plan", "library", "kv_swap_out", "kv_swap_in", "swap_workspace_bytes",
           "step_attention", "step_workspace_bytes", "check_block_table", "ceiling_mfma_bf16", "ceiling_stream_read",
           "ceiling_stream_copy", "build_step_tables", "step_tables_workspace_bytes", "StepTables", "qk_norm_rope",
           "diff_attention", "diff_workspace_bytes", "qk_norm_rope_axes", "residual_norm", "shaped_attention",
           "shaped_workspace_bytes"]


class CWError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"status {status}: {message}")
        self.status = status


def library():
    return L.load()


def _check(status: int):
    if status != L.CW_OK:
        lib = library()
        raise CWError(status, lib.cw_last_error_message().decode(errors="replace"))


def _lens(x) -> np.ndarray:
    a = np.ascontiguousarray(np.asarray(x, dtype=np.int32))
    return a


def _ptr(a: Optional[np.ndarray]):
    return None if a is None or a.size == 0 else a.__array_interface__["data"][0]


def _dptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("tensors must be on the GPU")
    if not t.is_contiguous():
        raise ValueError("tensors must be contiguous")
    return t.data_ptr()


def _want(t, name, dtypes, shape):
    """Marshalling check: `t` has one of `dtypes` and exactly `shape`."""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a torch.Tensor, got {type(t).__name__}")
    if t.dtype not in dtypes:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {' or '.join(map(str, dtypes))}")
    if tuple(t.shape) != tuple(int(x) for x in shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(int(x) for x in shape)}")


_BF16 = (torch.bfloat16,)
_FP8 = (torch.uint8, torch.float8_e4m3fn)


def _check_pools(k_pool, v_pool, k_scale, v_scale):
    """Pool, scale and their dtypes; returns (num_pages, Hkv, P, D)."""
    if not isinstance(k_pool, torch.Tensor) or k_pool.dim() != 4:
        raise ValueError("k_pool must be a 4-D tensor [num_pages, Hkv, P, D]")
    _kv_dtype(k_pool)
    _want(v_pool, "v_pool", (k_pool.dtype,), k_pool.shape)
    num_pages, hkv, page, d = k_pool.shape
    if k_pool.dtype == torch.bfloat16:
        if k_scale is not None or v_scale is not None:
            raise ValueError("k_scale / v_scale are for fp8 pools only")
    else:
        if k_scale is None or v_scale is None:
            raise ValueError("an fp8 pool needs k_scale and v_scale")
        _want(k_scale, "k_scale", (torch.float32,), (num_pages, hkv))
        _want(v_scale, "v_scale", (torch.float32,), (num_pages, hkv))
    return num_pages, hkv, page, d


def _quick_check(q, k_new, v_new, k_pool, v_pool, block_table, num_seqs, total, g, k_scale, v_scale,
                 out, lse):
    """The pool dimensions if every check of _check_call passes, else None (which of
    them failed is then found out, and raised, one check at a time).  A small call's
    own work takes 10 us on the GPU, and checking it argument by argument took 5."""
    try:
        pool_shape = k_pool.shape
        num_pages, hkv, page, d = pool_shape
        dt = k_pool.dtype
        dev = k_pool.get_device()
        if dev < 0 or v_pool.dtype is not dt or v_pool.shape != pool_shape or v_pool.get_device() != dev:
            return None
        if dt is torch.bfloat16:
            if k_scale is not None or v_scale is not None:
                return None
        elif dt in _FP8:
            pair = (num_pages, hkv)
            if not (k_scale.dtype is torch.float32 and k_scale.shape == pair and k_scale.get_device() == dev
                    and v_scale.dtype is torch.float32 and v_scale.shape == pair and v_scale.get_device() == dev):
                return None
        else:
            return None
        if type(g) is not int or g < 1:
            return None
        rows = (total, hkv * g, d)
        new = (total, hkv, d)
        if not (block_table.dtype is torch.int32 and block_table.dim() == 2 and block_table.shape[0] >= num_seqs
                and block_table.get_device() == dev
                and k_new.dtype is torch.bfloat16 and k_new.shape == new and k_new.get_device() == dev
                and v_new.dtype is torch.bfloat16 and v_new.shape == new and v_new.get_device() == dev):
            return None
        for t in (q, out):
            if t is not None and not (t.dtype is torch.bfloat16 and t.shape == rows and t.get_device() == dev):
                return None
        if lse is not None and not (lse.dtype is torch.float32 and lse.shape == rows[:2] and lse.get_device() == dev):
            return None
        return num_pages, hkv, page, d
    except (AttributeError, TypeError, ValueError):
        return None


def _check_call(q, k_new, v_new, k_pool, v_pool, block_table, num_seqs, total, gqa_group,
                k_scale=None, v_scale=None, out=None, lse=None):
    """dtype and shape of every tensor of an attention call against its lengths
    (`total` packed rows, `num_seqs` sequences); returns the pool dimensions."""
    dims = _quick_check(q, k_new, v_new, k_pool, v_pool, block_table, num_seqs, total, gqa_group,
                        k_scale, v_scale, out, lse)
    if dims is not None:
        return dims
    num_pages, hkv, page, d = _check_pools(k_pool, v_pool, k_scale, v_scale)
    if not isinstance(block_table, torch.Tensor) or block_table.dim() != 2 \
            or block_table.dtype != torch.int32:
        raise ValueError("block_table must be a 2-D int32 tensor [num_seqs, bt_stride]")
    if block_table.shape[0] < num_seqs:
        raise ValueError(f"block_table has {block_table.shape[0]} rows for {num_seqs} sequences")
    if int(gqa_group) < 1:
        raise ValueError(f"gqa_group = {gqa_group} must be >= 1")
    hq = hkv * int(gqa_group)
    if q is not None:
        _want(q, "q", _BF16, (total, hq, d))
    if out is not None:
        _want(out, "out", _BF16, (total, hq, d))
    _want(k_new, "k_new", _BF16, (total, hkv, d))
    _want(v_new, "v_new", _BF16, (total, hkv, d))
    if lse is not None:
        _want(lse, "lse", (torch.float32,), (total, hq))
    devs = {t.device for t in (q, out, k_new, v_new, k_pool, v_pool, k_scale, v_scale, block_table, lse)
            if t is not None}
    if len(devs) > 1:
        raise ValueError(f"tensors are on different devices: {sorted(map(str, devs))}")
    return num_pages, hkv, page, d


def _lens_pair(prefix_lens, suffix_lens):
    lp, ls = _lens(prefix_lens), _lens(suffix_lens)
    if lp.ndim != 1 or lp.shape != ls.shape:
        raise ValueError(f"prefix_lens {lp.shape} and suffix_lens {ls.shape} must be 1-D of one length")
    return lp, ls


def init():
    """cw_init on the current device (the one-time pinned staging set-up)."""
    _check(library().cw_init())


def pinned_allocations() -> int:
    """Pinned host allocations the library has made in this process."""
    return int(library().cw_pinned_allocations())


def arg_plan_calls() -> int:
    """Calls whose plan travelled in the kernel arguments, in this process."""
    return int(library().cw_arg_plan_calls())


def _stream():
    """torch's current HIP stream on the current device, as an integer."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _total(ls: np.ndarray) -> int:
    return sum(ls.tolist()) if ls.size <= 64 else int(ls.sum())


def _kv_dtype(pool: torch.Tensor) -> int:
    if pool.dtype == torch.bfloat16:
        return L.CW_KV_BF16
    if pool.dtype in (torch.uint8, torch.float8_e4m3fn):
        return L.CW_KV_FP8_E4M3FN
    raise ValueError(f"unsupported pool dtype {pool.dtype}")


def _workspace(nbytes: int, device, workspace: Optional[torch.Tensor]):
    if workspace is None:
        return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)
    return workspace


def write_pages_workspace_bytes(num_seqs: int) -> int:
    return int(library().cw_write_pages_workspace_bytes(num_seqs))


def _dtype_code(kv_dtype) -> int:
    if kv_dtype in ("bf16", L.CW_KV_BF16):
        return L.CW_KV_BF16
    if kv_dtype in ("fp8", "fp8_e4m3fn", L.CW_KV_FP8_E4M3FN):
        return L.CW_KV_FP8_E4M3FN
    raise ValueError(f"unsupported kv dtype {kv_dtype!r}")


def extend_workspace_bytes(prefix_lens, suffix_lens, num_kv_heads, gqa_group, head_dim,
                           page_size) -> int:
    lp, ls = _lens(prefix_lens), _lens(suffix_lens)
    return int(library().cw_extend_workspace_bytes(_ptr(lp), _ptr(ls), len(lp), num_kv_heads,
                                                   gqa_group, head_dim, page_size))


def decode_workspace_bytes(prefix_lens, num_kv_heads, gqa_group, head_dim, page_size,
                           kv_dtype="bf16") -> int:
    lp = _lens(prefix_lens)
    return int(library().cw_decode_workspace_bytes(_ptr(lp), len(lp), num_kv_heads, gqa_group,
                                                   head_dim, page_size, _dtype_code(kv_dtype)))


def set_tuning(key: int, value: int):
    _check(library().cw_set_tuning(key, value))


def plan_items(prefix_lens, suffix_lens, num_kv_heads, gqa_group, head_dim, page_size) -> np.ndarray:
    """The extend work list in launch order, int32 [n, 8] (see cw_extend_plan_items)."""
    lp, ls = _lens(prefix_lens), _lens(suffix_lens)
    lib = library()
    n = lib.cw_extend_plan_items(_ptr(lp), _ptr(ls), len(lp), num_kv_heads, gqa_group, head_dim,
                                 page_size, None, 0)
    if n < 0:
        raise CWError(L.CW_ERR_UNSUPPORTED, "invalid plan arguments")
    out = np.zeros((max(n, 1), 8), dtype=np.int32)
    lib.cw_extend_plan_items(_ptr(lp), _ptr(ls), len(lp), num_kv_heads, gqa_group, head_dim,
                             page_size, out.ctypes.data, n)
    return out[:n]


def decode_plan(prefix_lens, num_kv_heads, gqa_group, head_dim, page_size, kv_dtype="bf16",
                rebuilt=False):
    """The decode work list and merge groups, int32 [n, 8] each (see
    cw_decode_plan_items): as planned, or as rebuilt from the compact form."""
    lp = _lens(prefix_lens)
    lib = library()
    ng = C.c_int64()
    dt = {"bf16": L.CW_KV_BF16, "fp8": L.CW_KV_FP8_E4M3FN}[kv_dtype]
    n = lib.cw_decode_plan_items(_ptr(lp), len(lp), num_kv_heads, gqa_group, head_dim, page_size, dt,
                                 int(rebuilt), None, 0, None, 0, C.byref(ng))
    if n < 0:
        raise CWError(L.CW_ERR_UNSUPPORTED, "invalid plan arguments")
    items = np.zeros((max(n, 1), 8), dtype=np.int32)
    groups = np.zeros((max(ng.value, 1), 8), dtype=np.int32)
    lib.cw_decode_plan_items(_ptr(lp), len(lp), num_kv_heads, gqa_group, head_dim, page_size, dt,
                             int(rebuilt), items.ctypes.data, n, groups.ctypes.data, ng.value, C.byref(ng))
    return items[:n], groups[:ng.value]


def kv_write_pages(k_new, v_new, k_pool, v_pool, block_table, prefix_lens, suffix_lens,
                   k_scale=None, v_scale=None, workspace=None):
    lp, ls = _lens_pair(prefix_lens, suffix_lens)
    num_pages, hkv, page, d = _check_call(None, k_new, v_new, k_pool, v_pool, block_table, len(lp),
                                          _total(ls), 1, k_scale, v_scale)
    ws = _workspace(write_pages_workspace_bytes(len(lp)), k_pool.device, workspace)
    _check(library().cw_kv_write_pages(
        _dptr(k_new), _dptr(v_new), _dptr(k_pool), _dptr(v_pool), _dptr(k_scale), _dptr(v_scale),
        _dptr(block_table), block_table.shape[1], num_pages, _ptr(lp), _ptr(ls), len(lp), hkv, d,
        page, _kv_dtype(k_pool), _dptr(ws), ws.numel(), _stream()))


def extend_attention(q, k_new, v_new, k_pool, v_pool, block_table, prefix_lens, suffix_lens,
                     gqa_group, softmax_scale, k_scale=None, v_scale=None, out=None, lse=None,
                     workspace=None):
    lp, ls = _lens_pair(prefix_lens, suffix_lens)
    num_pages, hkv, page, d = _check_call(q, k_new, v_new, k_pool, v_pool, block_table, len(lp),
                                          _total(ls), gqa_group, k_scale, v_scale, out, lse)
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        workspace = _workspace(extend_workspace_bytes(lp, ls, hkv, gqa_group, d, page),
                               q.device, None)
    _check(library().cw_extend_attention(
        _dptr(q), _dptr(k_new), _dptr(v_new), _dptr(k_pool), _dptr(v_pool), _dptr(k_scale),
        _dptr(v_scale), _dptr(block_table), block_table.shape[1], num_pages, _ptr(lp), _ptr(ls),
        len(lp), hkv, gqa_group, d, page, float(softmax_scale), _kv_dtype(k_pool), _dptr(out),
        _dptr(lse), _dptr(workspace), workspace.numel(), _stream()))
    return out


def extend_attention_noalloc(q, k_new, v_new, k_pool, v_pool, block_table, prefix_lens, suffix_lens,
                             gqa_group, softmax_scale, k_scale=None, v_scale=None, out=None,
                             lse=None):
    """extend_attention with the library's static scratch instead of a workspace
    (cw_extend_attention_noalloc; init() must have run on this device).  With
    `out` given, the call allocates nothing."""
    lp, ls = _lens_pair(prefix_lens, suffix_lens)
    num_pages, hkv, page, d = _check_call(q, k_new, v_new, k_pool, v_pool, block_table, len(lp),
                                          _total(ls), gqa_group, k_scale, v_scale, out, lse)
    if out is None:
        out = torch.empty_like(q)
    _check(library().cw_extend_attention_noalloc(
        _dptr(q), _dptr(k_new), _dptr(v_new), _dptr(k_pool), _dptr(v_pool), _dptr(k_scale),
        _dptr(v_scale), _dptr(block_table), block_table.shape[1], num_pages, _ptr(lp), _ptr(ls),
        len(lp), hkv, gqa_group, d, page, float(softmax_scale), _kv_dtype(k_pool), _dptr(out),
        _dptr(lse), _stream()))
    return out


def write_extend_attention(q, k_new, v_new, k_pool, v_pool, block_table, prefix_lens, suffix_lens,
                           gqa_group, softmax_scale, k_scale=None, v_scale=None, out=None,
                           lse=None, workspace=None):
    """kv_write_pages + extend_attention in one launch (the pools are written)."""
    lp, ls = _lens_pair(prefix_lens, suffix_lens)
    num_pages, hkv, page, d = _check_call(q, k_new, v_new, k_pool, v_pool, block_table, len(lp),
                                          _total(ls), gqa_group, k_scale, v_scale, out, lse)
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        workspace = _workspace(extend_workspace_bytes(lp, ls, hkv, gqa_group, d, page),
                               q.device, None)
    _check(library().cw_write_extend_attention(
        _dptr(q), _dptr(k_new), _dptr(v_new), _dptr(k_pool), _dptr(v_pool), _dptr(k_scale),
        _dptr(v_scale), _dptr(block_table), block_table.shape[1], num_pages, _ptr(lp), _ptr(ls),
        len(lp), hkv, gqa_group, d, page, float(softmax_scale), _kv_dtype(k_pool), _dptr(out),
        _dptr(lse), _dptr(workspace), workspace.numel(), _stream()))
    return out


def step_workspace_bytes(prefix_lens, suffix_lens, num_kv_heads, gqa_group, head_dim, page_size,
                         kv_dtype="bf16") -> int:
    lp, ls = _lens(prefix_lens), _lens(suffix_lens)
    return int(library().cw_step_workspace_bytes(_ptr(lp), _ptr(ls), len(lp), num_kv_heads, gqa_group,
                                                 head_dim, page_size, _dtype_code(kv_dtype)))


def step_attention(q, k_new, v_new, k_pool, v_pool, block_table, prefix_lens, suffix_lens,
                   gqa_group, softmax_scale, k_scale=None, v_scale=None, out=None, lse=None,
                   workspace=None):
    """One serving step: page write + attention, decodes on the decode kernel."""
    lp, ls = _lens_pair(prefix_lens, suffix_lens)
    num_pages, hkv, page, d = _check_call(q, k_new, v_new, k_pool, v_pool, block_table, len(lp),
                                          _total(ls), gqa_group, k_scale, v_scale, out, lse)
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        workspace = _workspace(step_workspace_bytes(lp, ls, hkv, gqa_group, d, page, _kv_dtype(k_pool)),
                               q.device, None)
    _check(library().cw_step_attention(
        _dptr(q), _dptr(k_new), _dptr(v_new), _dptr(k_pool), _dptr(v_pool), _dptr(k_scale),
        _dptr(v_scale), _dptr(block_table), block_table.shape[1], num_pages, _ptr(lp), _ptr(ls),
        len(lp), hkv, gqa_group, d, page, float(softmax_scale), _kv_dtype(k_pool), _dptr(out),
        _dptr(lse), _dptr(workspace), workspace.numel(), _stream()))
    return out


def swap_workspace_bytes(n: int) -> int:
    return int(library().cw_swap_workspace_bytes(n))


def _hptr(t: Optional[torch.Tensor]):
    """Pointer to a host-pool tensor: device memory or pinned (device-mapped) host memory."""
    if t is None:
        return None
    if not (t.is_cuda or t.is_pinned()):
        raise ValueError("host pools must be pinned host tensors (pin_memory=True) or on the GPU")
    if not t.is_contiguous():
        raise ValueError("tensors must be contiguous")
    return t.data_ptr()


def _swap_dims(k_pool, k_host):
    num_pages, hkv, page, d = k_pool.shape
    if tuple(k_host.shape[1:]) != (hkv, page, d):
        raise ValueError(f"host pool blocks {tuple(k_host.shape[1:])} differ from pool blocks {(hkv, page, d)}")
    return num_pages, k_host.shape[0], hkv, page, d


def kv_swap_out(k_pool, v_pool, k_host, v_host, pages, host_blocks, k_scale=None, v_scale=None,
                k_scale_host=None, v_scale_host=None, workspace=None):
    """Pool page pages[i] -> host block host_blocks[i] (K, V and fp8 scales)."""
    pg, hb = _lens(pages), _lens(host_blocks)
    num_pages, n_host, hkv, page, d = _swap_dims(k_pool, k_host)
    ws = _workspace(swap_workspace_bytes(len(pg)), k_pool.device, workspace)
    _check(library().cw_kv_swap_out(
        _dptr(k_pool), _dptr(v_pool), _dptr(k_scale), _dptr(v_scale), num_pages, _hptr(k_host),
        _hptr(v_host), _hptr(k_scale_host), _hptr(v_scale_host), n_host, _ptr(pg), _ptr(hb), len(pg),
        hkv, d, page, _kv_dtype(k_pool), _dptr(ws), ws.numel(), _stream()))


def kv_swap_in(k_host, v_host, k_pool, v_pool, host_blocks, pages, k_scale_host=None,
               v_scale_host=None, k_scale=None, v_scale=None, workspace=None):
    """Host block host_blocks[i] -> pool page pages[i] (K, V and fp8 scales)."""
    pg, hb = _lens(pages), _lens(host_blocks)
    num_pages, n_host, hkv, page, d = _swap_dims(k_pool, k_host)
    ws = _workspace(swap_workspace_bytes(len(pg)), k_pool.device, workspace)
    _check(library().cw_kv_swap_in(
        _hptr(k_host), _hptr(v_host), _hptr(k_scale_host), _hptr(v_scale_host), n_host,
        _dptr(k_pool), _dptr(v_pool), _dptr(k_scale), _dptr(v_scale), num_pages, _ptr(hb), _ptr(pg),
        len(pg), hkv, d, page, _kv_dtype(k_pool), _dptr(ws), ws.numel(), _stream()))


def decode_attention(q, k_new, v_new, k_pool, v_pool, block_table, prefix_lens, gqa_group,
                     softmax_scale, k_scale=None, v_scale=None, out=None, lse=None, workspace=None):
    lp = _lens(prefix_lens)
    if lp.ndim != 1:
        raise ValueError("prefix_lens must be 1-D")
    num_pages, hkv, page, d = _check_call(q, k_new, v_new, k_pool, v_pool, block_table, len(lp),
                                          len(lp), gqa_group, k_scale, v_scale, out, lse)
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        workspace = _workspace(decode_workspace_bytes(lp, hkv, gqa_group, d, page,
                                                      _kv_dtype(k_pool)), q.device, None)
    _check(library().cw_decode_attention(
        _dptr(q), _dptr(k_new), _dptr(v_new), _dptr(k_pool), _dptr(v_pool), _dptr(k_scale),
        _dptr(v_scale), _dptr(block_table), block_table.shape[1], num_pages, _ptr(lp), len(lp),
        hkv, gqa_group, d, page, float(softmax_scale), _kv_dtype(k_pool), _dptr(out), _dptr(lse),
        _dptr(workspace), workspace.numel(), _stream()))
    return out


def check_block_table(block_table, prefix_lens, suffix_lens, num_pages: int, page_size: int,
                      workspace=None) -> np.ndarray:
    """Per sequence, the number of block-table entries a call with these lengths
    would read that lie outside [0, num_pages) (waits for the result)."""
    lp, ls = _lens(prefix_lens), _lens(suffix_lens)
    bad = torch.empty(max(len(lp), 1), dtype=torch.int32, device=block_table.device)
    if workspace is None:
        workspace = _workspace(write_pages_workspace_bytes(len(lp)), block_table.device, None)
    _check(library().cw_check_block_table(
        _dptr(block_table), block_table.shape[1], int(num_pages), _ptr(lp), _ptr(ls), len(lp),
        int(page_size), _dptr(bad), _dptr(workspace), workspace.numel(), _stream()))
    return bad[:len(lp)].cpu().numpy()


# around the attention (include/cw_layer.h)

def step_tables_workspace_bytes(num_seqs: int) -> int:
    return int(library().cw_step_tables_workspace_bytes(int(num_seqs)))


class StepTables(NamedTuple):
    """What build_step_tables wrote besides the block table: cu_rows int32 [B + 1], seq_ids and
    positions int32 [max_tokens], slots int64 [max_tokens], info int64 [3] (pages taken, new
    tokens, sequences that need more pages than a table row holds)."""
    cu_rows: torch.Tensor
    seq_ids: torch.Tensor
    positions: torch.Tensor
    slots: torch.Tensor
    info: torch.Tensor


def build_step_tables(prefix_lens, suffix_lens, free_pages, block_table, page_size: int, max_tokens: int,
                      cu_rows=None, seq_ids=None, positions=None, slots=None, info=None, workspace=None) -> StepTables:
    """The step's new block-table entries (in place) and its tokens' index arrays, from int32
    lengths on the GPU (cw_build_step_tables); waits for nothing."""
    t = int(max_tokens)
    if not isinstance(prefix_lens, torch.Tensor) or prefix_lens.dim() != 1:
        raise ValueError("prefix_lens must be a 1-D int32 tensor")
    num = prefix_lens.shape[0]
    if t < 0:
        raise ValueError(f"max_tokens = {t} is negative")
    if cu_rows is None or seq_ids is None or positions is None or slots is None or info is None:
        new = lambda n, dt: torch.empty(n, dtype=dt, device=prefix_lens.device)
        cu_rows = new(num + 1, torch.int32) if cu_rows is None else cu_rows
        seq_ids = new(t, torch.int32) if seq_ids is None else seq_ids
        positions = new(t, torch.int32) if positions is None else positions
        slots = new(t, torch.int64) if slots is None else slots
        info = new(3, torch.int64) if info is None else info
    nb = 0
    if num > _TABLES_WITHOUT_WORKSPACE and workspace is None:
        workspace = _workspace(step_tables_workspace_bytes(num), prefix_lens.device, None)
    if workspace is not None:
        nb = workspace.numel() * workspace.element_size()
    dev = torch._C._cuda_getDevice()
    if not _quick_tables(dev, num, t, prefix_lens, suffix_lens, free_pages, block_table, cu_rows, seq_ids, positions, slots,
                         info):
        i32, i64 = (torch.int32,), (torch.int64,)
        _want(prefix_lens, "prefix_lens", i32, (num,))
        _want(suffix_lens, "suffix_lens", i32, (num,))
        if not isinstance(free_pages, torch.Tensor) or free_pages.dim() != 1 or free_pages.dtype != torch.int32:
            raise ValueError("free_pages must be a 1-D int32 tensor")
        if not isinstance(block_table, torch.Tensor) or block_table.dim() != 2 or block_table.dtype != torch.int32:
            raise ValueError("block_table must be a 2-D int32 tensor [num_seqs, bt_stride]")
        if block_table.shape[0] < num:
            raise ValueError(f"block_table has {block_table.shape[0]} rows for {num} sequences")
        _want(cu_rows, "cu_rows", i32, (num + 1,))
        _want(seq_ids, "seq_ids", i32, (t,))
        _want(positions, "positions", i32, (t,))
        _want(slots, "slots", i64, (t,))
        _want(info, "info", i64, (3,))
        for x in (prefix_lens, suffix_lens, free_pages, block_table, cu_rows, seq_ids, positions, slots, info):
            _dptr(x)
        _one_device(prefix_lens, suffix_lens, free_pages, block_table, cu_rows, seq_ids, positions, slots, info)
    _check(library().cw_build_step_tables(
        prefix_lens.data_ptr(), suffix_lens.data_ptr(), num, free_pages.data_ptr(), free_pages.shape[0], int(page_size),
        block_table.data_ptr(), block_table.shape[1], t, cu_rows.data_ptr(), seq_ids.data_ptr(), positions.data_ptr(),
        slots.data_ptr(), info.data_ptr(), _dptr(workspace), nb, torch._C._cuda_getCurrentRawStream(dev)))
    return StepTables(cu_rows, seq_ids, positions, slots, info)


_TABLES_WITHOUT_WORKSPACE = 4096  # cw_step_tables_workspace_bytes is 0 up to here


def _quick_tables(dev, num, t, prefix_lens, suffix_lens, free_pages, block_table, cu_rows, seq_ids, positions, slots, info):
    """Whether every check of build_step_tables passes (else they are made one at a time): the
    call's own work takes 3 us on the GPU."""
    i32, i64, row = torch.int32, torch.int64, (1,)
    try:
        for x, n in ((prefix_lens, num), (suffix_lens, num), (cu_rows, num + 1), (seq_ids, t), (positions, t)):
            if not (x.dtype is i32 and x.stride() == row and x.numel() == n and x.get_device() == dev):
                return False
        return (slots.dtype is i64 and slots.stride() == row and slots.numel() == t and slots.get_device() == dev
                and info.dtype is i64 and info.stride() == row and info.numel() == 3 and info.get_device() == dev
                and free_pages.dtype is i32 and free_pages.stride() == row and free_pages.get_device() == dev
                and block_table.dtype is i32 and block_table.dim() == 2 and block_table.shape[0] >= num
                and block_table.get_device() == dev and block_table.is_contiguous())
    except AttributeError:
        return False


def _one_device(*tensors):
    """Every tensor on the current device, whose stream the call goes to."""
    devs = {t.device for t in tensors if t is not None}
    if len(devs) > 1:
        raise ValueError(f"tensors are on different devices: {sorted(map(str, devs))}")
    for dev in devs:
        if dev.type != "cuda":
            raise ValueError("tensors must be on the GPU")
        if dev.index != torch.cuda.current_device():
            raise ValueError(f"tensors are on {dev}, the current device is cuda:{torch.cuda.current_device()}")


def _head_rows(t, name, total, heads, d):
    """Pointer and token stride of a bf16 [T, H, D] tensor whose tokens' heads are contiguous."""
    _want(t, name, _BF16, (total, heads, d))
    if not t.is_cuda:
        raise ValueError("tensors must be on the GPU")
    if t.stride(2) != 1 or (heads > 1 and t.stride(1) != d):
        raise ValueError(f"{name}: the heads of a token must be contiguous (strides {t.stride()})")
    return t.data_ptr(), t.stride(0) if total > 1 else heads * d


def _quick_rope(dev, total, hq, hkv, d, q, k, v, cos_sin, positions, weights, q_out, k_out, v_out, k_pool, v_pool, slots,
                k_scale, v_scale, pos_shape):
    """Whether every check of qk_norm_rope passes (else they are made one at a time)."""
    bf, f32 = torch.bfloat16, torch.float32
    rows_q, rows = (total, hq, d), (total, hkv, d)
    try:
        _, q1, q2 = q.stride()
        _, k1, k2 = k.stride()
        if not (q.dtype is bf and q2 == 1 and (q1 == d or hq == 1) and q.get_device() == dev
                and k.dtype is bf and k2 == 1 and (k1 == d or hkv == 1) and k.get_device() == dev and k.shape == rows
                and q_out.dtype is bf and q_out.shape == rows_q and q_out.get_device() == dev and q_out.is_contiguous()
                and k_out.dtype is bf and k_out.shape == rows and k_out.get_device() == dev and k_out.is_contiguous()
                and cos_sin.dtype is f32 and cos_sin.dim() == 2 and cos_sin.get_device() == dev and cos_sin.is_contiguous()
                and positions.dtype is torch.int32 and positions.shape == pos_shape and positions.get_device() == dev
                and positions.is_contiguous()):
            return False
        if v is not None:
            _, v1, v2 = v.stride()
            if not (v.dtype is bf and v2 == 1 and (v1 == d or hkv == 1) and v.get_device() == dev and v.shape == rows
                    and v_out.dtype is bf and v_out.shape == rows and v_out.get_device() == dev and v_out.is_contiguous()):
                return False
        elif v_out is not None:
            return False
        for x in weights:
            if x is not None and not (x.dtype is f32 and x.shape == (d,) and x.get_device() == dev and x.is_contiguous()):
                return False
        if k_pool is None:
            return v_pool is None and slots is None and k_scale is None and v_scale is None
        shape, dt = k_pool.shape, k_pool.dtype
        if not (len(shape) == 4 and shape[1] == hkv and shape[3] == d and v_pool.shape == shape and v_pool.dtype is dt
                and k_pool.get_device() == dev and v_pool.get_device() == dev and k_pool.is_contiguous()
                and v_pool.is_contiguous() and v is not None and slots.dtype is torch.int64 and slots.shape == (total,)
                and slots.get_device() == dev and slots.is_contiguous()):
            return False
        if dt is bf:
            return k_scale is None and v_scale is None
        pair = (shape[0], hkv)
        return (dt in _FP8 and k_scale.dtype is f32 and k_scale.shape == pair and k_scale.get_device() == dev
                and k_scale.is_contiguous() and v_scale.dtype is f32 and v_scale.shape == pair
                and v_scale.get_device() == dev and v_scale.is_contiguous())
    except (AttributeError, TypeError, ValueError):
        return False


def _check_rope(total, hq, hkv, d, q, k, v, cos_sin, positions, q_weight, k_weight, q_out, k_out, v_out, k_pool, v_pool,
                slots, k_scale, v_scale, pos_shape):
    """The checks of qk_norm_rope, one at a time."""
    for x, name, h in ((q, "q", hq), (k, "k", hkv), (v, "v", hkv)):
        if x is not None:
            _head_rows(x, name, total, h, d)
    if not isinstance(cos_sin, torch.Tensor) or cos_sin.dim() != 2 or cos_sin.dtype != torch.float32:
        raise ValueError("cos_sin must be a 2-D float32 tensor [positions, rotary_dim]")
    _want(positions, "positions", (torch.int32,), pos_shape)
    for w, name in ((q_weight, "q_weight"), (k_weight, "k_weight")):
        if w is not None:
            _want(w, name, (torch.float32,), (d,))
    if k_pool is not None or v_pool is not None:
        if k_pool is None or v_pool is None or v is None or slots is None:
            raise ValueError("a page write needs k_pool, v_pool, slots and v")
        _, pool_heads, _, pool_d = _check_pools(k_pool, v_pool, k_scale, v_scale)
        if (pool_heads, pool_d) != (hkv, d):
            raise ValueError(f"pools of {pool_heads} heads of {pool_d} for k of {hkv} heads of {d}")
        _want(slots, "slots", (torch.int64,), (total,))
    elif slots is not None or k_scale is not None or v_scale is not None:
        raise ValueError("slots, k_scale and v_scale are for a page write (k_pool and v_pool)")
    _want(q_out, "q_out", _BF16, (total, hq, d))
    _want(k_out, "k_out", _BF16, (total, hkv, d))
    if v_out is not None:
        if v is None:
            raise ValueError("v_out without v")
        _want(v_out, "v_out", _BF16, (total, hkv, d))
    for x in (cos_sin, positions, q_weight, k_weight, q_out, k_out, v_out, k_pool, v_pool, k_scale, v_scale, slots):
        _dptr(x)
    _one_device(q, k, v, cos_sin, positions, q_weight, k_weight, k_pool, v_pool, slots, k_scale, v_scale, q_out, k_out,
                v_out)


def qk_norm_rope(q, k, cos_sin, positions, q_weight=None, k_weight=None, eps=1e-6, interleaved=False, v=None,
                 k_pool=None, v_pool=None, slots=None, k_scale=None, v_scale=None, q_out=None, k_out=None, v_out=None):
    """Norm of every query and key head, position rotation and (with pools) page write in one
    pass (cw_qk_norm_rope).  q [T, Hq, D], k, v [T, Hkv, D] may be columns of one projection's
    output.  Returns (q_out, k_out, v_out), contiguous; v_out is None without v."""
    return _norm_rope(None, q, k, cos_sin, positions, q_weight, k_weight, eps, interleaved, v, k_pool, v_pool, slots, k_scale,
                      v_scale, q_out, k_out, v_out)


def qk_norm_rope_axes(q, k, cos_sin, positions, axis_of, q_weight=None, k_weight=None, eps=1e-6, interleaved=False, v=None,
                      k_pool=None, v_pool=None, slots=None, k_scale=None, v_scale=None, q_out=None, k_out=None, v_out=None):
    """qk_norm_rope for positions with several axes (cw_qk_norm_rope_axes): positions int32 [axes, T], and
    axis_of (host, rotary_dim / 2 entries) the axis that each rotated pair follows."""
    return _norm_rope(_lens(axis_of), q, k, cos_sin, positions, q_weight, k_weight, eps, interleaved, v, k_pool, v_pool, slots,
                      k_scale, v_scale, q_out, k_out, v_out)


def _norm_rope(axis_of, q, k, cos_sin, positions, q_weight, k_weight, eps, interleaved, v, k_pool, v_pool, slots, k_scale,
               v_scale, q_out, k_out, v_out):
    if not isinstance(q, torch.Tensor) or q.dim() != 3 or not isinstance(k, torch.Tensor) or k.dim() != 3:
        raise ValueError("q and k must be 3-D tensors [T, heads, D]")
    total, hq, d = q.shape
    hkv = k.shape[1]
    if q_out is None or k_out is None or (v is not None and v_out is None):
        new = lambda h: torch.empty(total, h, d, dtype=torch.bfloat16, device=q.device)
        q_out = new(hq) if q_out is None else q_out
        k_out = new(hkv) if k_out is None else k_out
        v_out = new(hkv) if v is not None and v_out is None else v_out
    dev = torch._C._cuda_getDevice()
    axes, pos_shape = 0, (total,)
    if axis_of is not None:
        if not isinstance(positions, torch.Tensor) or positions.dim() != 2:
            raise ValueError("positions must be a 2-D int32 tensor [axes, T]")
        axes = positions.shape[0]
        pos_shape = (axes, total)
    if not _quick_rope(dev, total, hq, hkv, d, q, k, v, cos_sin, positions, (q_weight, k_weight), q_out, k_out, v_out,
                       k_pool, v_pool, slots, k_scale, v_scale, pos_shape):
        _check_rope(total, hq, hkv, d, q, k, v, cos_sin, positions, q_weight, k_weight, q_out, k_out, v_out, k_pool, v_pool,
                    slots, k_scale, v_scale, pos_shape)
    if axis_of is not None and axis_of.shape != (cos_sin.shape[1] // 2,):
        raise ValueError(f"axis_of has shape {axis_of.shape}, expected {(cos_sin.shape[1] // 2,)}")
    vp = vs = vo = kp = vpool = sl = ks = vsc = None
    num_pages, page, dt = 0, 0, L.CW_KV_BF16
    if v is not None:
        vp, vs, vo = v.data_ptr(), v.stride(0) if total > 1 else hkv * d, v_out.data_ptr()
    if k_pool is not None:
        num_pages, _, page, _ = k_pool.shape
        kp, vpool, sl = k_pool.data_ptr(), v_pool.data_ptr(), slots.data_ptr()
        if k_scale is not None:
            dt, ks, vsc = L.CW_KV_FP8_E4M3FN, k_scale.data_ptr(), v_scale.data_ptr()
    head = (q.data_ptr(), q.stride(0) if total > 1 else hq * d, k.data_ptr(), k.stride(0) if total > 1 else hkv * d, vp,
            vs or 0, total, hq, hkv, d, None if q_weight is None else q_weight.data_ptr(),
            None if k_weight is None else k_weight.data_ptr(), eps, cos_sin.data_ptr(), cos_sin.shape[0], cos_sin.shape[1],
            1 if interleaved else 0, positions.data_ptr())
    tail = (q_out.data_ptr(), k_out.data_ptr(), vo, kp, vpool, ks, vsc, sl, num_pages, page, dt,
            torch._C._cuda_getCurrentRawStream(dev))
    if axis_of is None:
        _check(library().cw_qk_norm_rope(*head, *tail))
    else:
        _check(library().cw_qk_norm_rope_axes(*head, axes, _ptr(axis_of), *tail))
    return q_out, k_out, v_out


def _rows(t, name, total, width):
    """Pointer and token stride of a bf16 [T, width] tensor with contiguous rows."""
    _want(t, name, _BF16, (total, width))
    if not t.is_cuda:
        raise ValueError("tensors must be on the GPU")
    if t.stride(1) != 1 and width > 1:
        raise ValueError(f"{name}: a token's elements must be contiguous (strides {t.stride()})")
    return t.data_ptr(), t.stride(0) if total > 1 else width


def residual_norm(x, residual, post_weight=None, gate=None, residual_scale=1.0, pre_weight=None, eps=1e-6, residual_out=None,
                  y_out=None):
    """The norm of a block's output x [T, width] (with post_weight), its gate ([width], or [T, width]) and the scaled
    residual stream (bf16 or fp32), and with pre_weight the norm before the next block, in one pass
    (cw_residual_norm).  Returns (residual_out, y_out); y_out is None without pre_weight."""
    if not isinstance(x, torch.Tensor) or x.dim() != 2:
        raise ValueError("x must be a 2-D tensor [T, width]")
    total, width = x.shape
    xp, xs = _rows(x, "x", total, width)
    _want(residual, "residual", (torch.bfloat16, torch.float32), (total, width))
    if residual_out is None:
        residual_out = torch.empty_like(residual)
    else:
        _want(residual_out, "residual_out", (residual.dtype,), (total, width))
    if pre_weight is None:
        if y_out is not None:
            raise ValueError("y_out without pre_weight")
    elif y_out is None:
        y_out = torch.empty(total, width, dtype=torch.bfloat16, device=x.device)
    else:
        _want(y_out, "y_out", _BF16, (total, width))
    for w, name in ((post_weight, "post_weight"), (pre_weight, "pre_weight")):
        if w is not None:
            _want(w, name, (torch.float32,), (width,))
    gp, gs = None, 0
    if gate is not None:
        if isinstance(gate, torch.Tensor) and gate.dim() == 1:
            _want(gate, "gate", _BF16, (width,))
            gp = _dptr(gate)
        else:
            gp, gs = _rows(gate, "gate", total, width)
    dev = torch._C._cuda_getDevice()
    for t in (x, residual, residual_out, y_out, post_weight, pre_weight, gate):
        if t is not None and t.get_device() != dev:
            _one_device(x, residual, residual_out, y_out, post_weight, pre_weight, gate)
    _check(library().cw_residual_norm(
        xp, xs, _dptr(residual), 1 if residual.dtype is torch.float32 else 0, total, width, _dptr(post_weight), gp, gs,
        float(residual_scale), _dptr(pre_weight), float(eps), _dptr(residual_out), _dptr(y_out),
        torch._C._cuda_getCurrentRawStream(dev)))
    return residual_out, y_out


def diff_workspace_bytes(prefix_lens, suffix_lens, num_kv_pairs, gqa_group, head_dim, page_size,
                         kv_dtype="bf16") -> int:
    lp, ls = _lens_pair(prefix_lens, suffix_lens)
    return int(library().cw_diff_workspace_bytes(_ptr(lp), _ptr(ls), len(lp), num_kv_pairs, gqa_group, head_dim,
                                                 page_size, _dtype_code(kv_dtype)))


def diff_attention(q, k_new, v_new, k_pool, v_pool, block_table, prefix_lens, suffix_lens, gqa_group, softmax_scale,
                   lam, k_scale=None, v_scale=None, norm_weight=None, norm_eps=1e-5, out_scale=1.0, out=None,
                   workspace=None):
    """Differential attention over the paged cache (cw_diff_attention): q [T, 2 Hp, D], k_new and
    v_new [T, 2 pairs, D], pools of 2 pairs heads, lam fp32 [Hp], out [T, Hp, 2 D] with Hp = pairs *
    gqa_group.  The pools are only read."""
    lp, ls = _lens_pair(prefix_lens, suffix_lens)
    total = _total(ls)
    num_pages, heads, page, d = _check_call(q, k_new, v_new, k_pool, v_pool, block_table, len(lp), total, gqa_group,
                                            k_scale, v_scale)
    if heads % 2:
        raise ValueError(f"pools of {heads} heads: differential attention takes pairs of them")
    hp = heads // 2 * int(gqa_group)
    if out is None:
        out = torch.empty(total, hp, 2 * d, dtype=torch.bfloat16, device=q.device)
    _want(lam, "lam", (torch.float32,), (hp,))
    if norm_weight is not None:
        _want(norm_weight, "norm_weight", (torch.float32,), (2 * d,))
    _want(out, "out", _BF16, (total, hp, 2 * d))
    dev = torch._C._cuda_getDevice()
    if not (q.get_device() == dev == lam.get_device() == out.get_device()
            and (norm_weight is None or norm_weight.get_device() == dev)):
        _one_device(q, lam, norm_weight, out)
    if workspace is None:
        workspace = _workspace(diff_workspace_bytes(lp, ls, heads // 2, gqa_group, d, page, _kv_dtype(k_pool)),
                               q.device, None)
    _check(library().cw_diff_attention(
        _dptr(q), _dptr(k_new), _dptr(v_new), _dptr(k_pool), _dptr(v_pool), _dptr(k_scale), _dptr(v_scale),
        _dptr(block_table), block_table.shape[1], num_pages, _ptr(lp), _ptr(ls), len(lp), heads // 2, gqa_group, d,
        page, float(softmax_scale), _kv_dtype(k_pool), _dptr(lam), _dptr(norm_weight), float(norm_eps),
        float(out_scale), _dptr(out), _dptr(workspace), workspace.numel(), _stream()))
    return out


def _window(window) -> int:
    window = int(window)
    if not 0 <= window < 1 << 31:
        raise ValueError(f"window = {window} must be in 0 .. 2^31 - 1")
    return window


def _full_lens(full_lens, num_seqs):
    if full_lens is None:
        return None
    full = _lens(full_lens)
    if full.shape != (num_seqs,):
        raise ValueError(f"full_lens has shape {full.shape}, expected {(num_seqs,)}")
    return full


def shaped_workspace_bytes(prefix_lens, suffix_lens, num_kv_heads, gqa_group, head_dim, page_size, kv_dtype="bf16",
                           window=0, full_lens=None) -> int:
    lp, ls = _lens_pair(prefix_lens, suffix_lens)
    full = _full_lens(full_lens, len(lp))
    return int(library().cw_shaped_workspace_bytes(_ptr(lp), _ptr(ls), len(lp), num_kv_heads, gqa_group, head_dim,
                                                   page_size, _dtype_code(kv_dtype), _window(window), _ptr(full)))


def shaped_attention(q, k_new, v_new, k_pool, v_pool, block_table, prefix_lens, suffix_lens, gqa_group, softmax_scale,
                     score_cap=0.0, slopes=None, window=0, key_begins=None, full_lens=None, k_scale=None, v_scale=None,
                     out=None, lse=None, workspace=None):
    """Attention over the paged cache with capped, biased and masked scores (cw_shaped_attention): score_cap of
    a tanh, slopes fp32 [Hq] of a bias by distance, window in tokens, key_begins int32 [T] (first visible position
    of each new token) and full_lens (host, per sequence: its first tokens all see each other).  The pools are
    only read."""
    lp, ls = _lens_pair(prefix_lens, suffix_lens)
    total = _total(ls)
    num_pages, hkv, page, d = _check_call(q, k_new, v_new, k_pool, v_pool, block_table, len(lp), total, gqa_group,
                                          k_scale, v_scale, out, lse)
    if out is None:
        out = torch.empty_like(q)
    full = _full_lens(full_lens, len(lp))
    if slopes is not None:
        _want(slopes, "slopes", (torch.float32,), (hkv * int(gqa_group),))
    if key_begins is not None:
        _want(key_begins, "key_begins", (torch.int32,), (total,))
    dev = torch._C._cuda_getDevice()
    if not (q.get_device() == dev == out.get_device() and (slopes is None or slopes.get_device() == dev)
            and (key_begins is None or key_begins.get_device() == dev)):
        _one_device(q, out, slopes, key_begins)
    if workspace is None:
        workspace = _workspace(shaped_workspace_bytes(lp, ls, hkv, gqa_group, d, page, _kv_dtype(k_pool), window, full),
                               q.device, None)
    _check(library().cw_shaped_attention(
        _dptr(q), _dptr(k_new), _dptr(v_new), _dptr(k_pool), _dptr(v_pool), _dptr(k_scale), _dptr(v_scale),
        _dptr(block_table), block_table.shape[1], num_pages, _ptr(lp), _ptr(ls), len(lp), hkv, gqa_group, d, page,
        float(softmax_scale), _kv_dtype(k_pool), float(score_cap), _dptr(slopes), _window(window), _dptr(key_begins),
        _ptr(full), _dptr(out), _dptr(lse), _dptr(workspace), workspace.numel(), _stream()))
    return out


# measured ceilings (include/cw_ceiling.h): not part of the attention path

def ceiling_mfma_bf16(workgroups: int, iters: int, sink: torch.Tensor, random: bool = True) -> float:
    """Enqueues the matrix-core loop (random operand bits, or the low-entropy
    patterns with `random=False`); returns the FLOPs it performs."""
    kind = L.CW_CEILING_RANDOM if random else L.CW_CEILING_LOW_ENTROPY
    _check(library().cw_ceiling_mfma_bf16(int(workgroups), int(iters), kind, _dptr(sink), _stream()))
    return float(workgroups) * 8 * iters * 131072


def ceiling_stream_read(src: torch.Tensor, sink: torch.Tensor) -> int:
    """Enqueues a streaming read of `src`; returns the bytes it moves."""
    n = src.numel() * src.element_size()
    _check(library().cw_ceiling_stream_read(_dptr(src), n, _dptr(sink), _stream()))
    return n


def ceiling_stream_copy(src: torch.Tensor, dst: torch.Tensor) -> int:
    """Enqueues a streaming copy of `src` into `dst`; returns the bytes it moves."""
    n = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() < n:
        raise ValueError("dst is smaller than src")
    _check(library().cw_ceiling_stream_copy(_dptr(src), _dptr(dst), n, _stream()))
    return 2 * n

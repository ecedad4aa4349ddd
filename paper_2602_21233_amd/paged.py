"""Binding of the paged-KV-cache calls of include/sparse_prefill.h: block tables and slot maps of a serving step, the new
tokens' keys and values into their pages, attention over the pages.  Argument marshalling only."""
from __future__ import annotations

import ctypes
import struct

import torch

from .binding import SpaError, SpaPagedParams, _check, _dev_bf16, _stream, load_library

# 9 int32, a float, 2 int32, a float, table_stride and six stride pairs: see SpaPagedParams
_PARAMS = struct.Struct("@9if2if13q")
assert _PARAMS.size == ctypes.sizeof(SpaPagedParams)
_NO_STRIDE = (0, 0)


def make_paged_params(*, batch=1, n_q_heads=1, n_kv_heads=1, head_dim=64, page_size, n_pages, max_pages=1, n_tokens, max_new_tokens=0,
                      softmax_scale=None, n_sink_tokens=0, window_tokens=0, softcap=0.0, table_stride=1, q=_NO_STRIDE, k=_NO_STRIDE,
                      v=_NO_STRIDE, out=_NO_STRIDE, k_pages=_NO_STRIDE, vt_pages=_NO_STRIDE) -> SpaPagedParams:
    """q, k, v, out: (token, head) strides; k_pages, vt_pages: (page, head) strides, all in elements."""
    scale = 0.0 if softmax_scale is None else softmax_scale
    try:
        return SpaPagedParams.from_buffer_copy(_PARAMS.pack(
            batch, n_q_heads, n_kv_heads, head_dim, page_size, n_pages, max_pages, n_tokens, max_new_tokens, scale, n_sink_tokens,
            window_tokens, softcap, table_stride, *q, *k, *v, *out, *k_pages, *vt_pages))
    except (struct.error, OverflowError):        # a value that does not fit its field
        raise SpaError(-2, load_library().spa_strerror(-2)) from None


def paged_workspace_bytes(p: SpaPagedParams) -> int:
    n = ctypes.c_size_t()
    _check(load_library().spa_paged_workspace_bytes(ctypes.byref(p), ctypes.byref(n)))
    return n.value


def _ints(name, t, device, *shape):
    if t.dtype != torch.int32 or t.device != device or not t.is_contiguous() or tuple(t.shape) != shape:
        raise TypeError(f"{name} must be a contiguous int32 tensor of shape {list(shape)} on {device}")
    return t.data_ptr()


def _table(t, device, batch):
    if t.dtype != torch.int32 or t.device != device or t.dim() != 2 or t.shape[0] != batch or (t.shape[1] > 1 and t.stride(1) != 1):
        raise TypeError(f"block_table must be an int32 tensor [{batch}, max_pages] on {device} with contiguous rows")
    return t.data_ptr()


def _rows(name, t, device, *shape):
    if t.device != device or tuple(t.shape) != shape or t.stride(2) != 1:
        raise TypeError(f"{name} must be a tensor of shape {list(shape)} on {device} with a contiguous last axis")
    return _two_strides(t.stride(), shape)


def _two_strides(st, shape):
    """Strides of the two outer axes; an axis of one entry may have any, so it gets that of a dense tensor."""
    inner = st[1] if shape[1] > 1 else shape[2] * (shape[3] if len(shape) > 3 else 1)
    return st[0] if shape[0] > 1 else shape[1] * inner, inner


def _cache(k_pages, vt_pages):
    """(n_pages, n_kv_heads, page_size, head_dim, K strides, V strides)"""
    n, h, p, d = k_pages.shape
    ks, vs = k_pages.stride(), vt_pages.stride()
    if tuple(vt_pages.shape) != (n, h, d, p) or k_pages.device != vt_pages.device:
        raise TypeError("vt_pages must be [n_pages, n_kv_heads, head_dim, page_size] beside k_pages [n_pages, n_kv_heads, page_size, head_dim]")
    if ks[3] != 1 or ks[2] != d or vs[3] != 1 or vs[2] != p:
        raise TypeError("the two inner axes of k_pages and vt_pages must be contiguous")
    return n, h, p, d, _two_strides(ks, (n, h, p, d)), _two_strides(vs, (n, h, d, p))


class _on:
    """Calls go to the tensors' device, whichever is current."""
    __slots__ = ("index", "before")

    def __init__(self, device):
        self.index = device.index

    def __enter__(self):
        self.before = torch.cuda.current_device()
        if self.before != self.index:
            torch.cuda.set_device(self.index)

    def __exit__(self, *exc):
        if self.before != self.index:
            torch.cuda.set_device(self.before)


def paged_plan(block_table, ctx_lens, new_lens, free_pages, free_range, n_tokens, page_size, n_pages):
    """sparse_prefill_paged_plan: block_table (int32 [B, max_pages]) gets the pages that the step takes from
    free_pages[free_range[0]:free_range[1]].  Returns (q_starts [B+1], kv_lens [B], slots [n_tokens], positions
    [n_tokens], taken [2]), int32 tensors that lie in one allocation."""
    dev, B = ctx_lens.device, ctx_lens.shape[0]
    if dev.type != "cuda":
        raise TypeError("expected tensors on the GPU")
    ptrs = (_ints("ctx_lens", ctx_lens, dev, B), _ints("new_lens", new_lens, dev, B), _ints("free_pages", free_pages, dev, free_pages.numel()))
    ptrs += (free_pages.numel(), _ints("free_range", free_range, dev, 2), _table(block_table, dev, B))
    p = make_paged_params(batch=B, page_size=page_size, n_pages=n_pages, max_pages=block_table.shape[1], n_tokens=n_tokens,
                          table_stride=block_table.stride(0) if B > 1 else block_table.shape[1])
    got = torch.empty(2 * B + 1 + 2 * n_tokens + 2, dtype=torch.int32, device=dev).split((B + 1, B, n_tokens, n_tokens, 2))
    with _on(dev):
        _check(load_library().sparse_prefill_paged_plan(ctypes.byref(p), *ptrs, *[t.data_ptr() for t in got], _stream(ctx_lens)))
    return got


def paged_append(k, v, slots, k_pages, vt_pages):
    """sparse_prefill_paged_append: k, v [n_tokens, n_kv_heads, head_dim] to the places slots (int32 [n_tokens]) of the cache."""
    _dev_bf16(k, v, k_pages, vt_pages)
    n, h, page, d, kps, vps = _cache(k_pages, vt_pages)
    dev, T = k_pages.device, slots.shape[0]
    p = make_paged_params(n_q_heads=h, n_kv_heads=h, head_dim=d, page_size=page, n_pages=n, n_tokens=T, k=_rows("k", k, dev, T, h, d),
                          v=_rows("v", v, dev, T, h, d), k_pages=kps, vt_pages=vps)
    with _on(dev):
        _check(load_library().sparse_prefill_paged_append(ctypes.byref(p), k.data_ptr(), v.data_ptr(), _ints("slots", slots, dev, T),
                                                          k_pages.data_ptr(), vt_pages.data_ptr(), _stream(k_pages)))


def paged_attn(q, k_pages, vt_pages, block_table, q_starts, kv_lens, max_new_tokens=0, softmax_scale=None, n_sink_tokens=0,
               window_tokens=0, softcap=0.0, slopes=None, return_lse=False, out=None, workspace=None):
    """sparse_prefill_paged_attn: q [n_tokens, n_q_heads, head_dim] -> out of the same shape (and lse [n_tokens, n_q_heads] fp32).
    max_new_tokens: the most new tokens of a request, where the host knows it; slopes: fp32 [n_q_heads], bias by distance.
    Rows of padding are left as they are in `out` (as allocated where none is given)."""
    _dev_bf16(q, k_pages, vt_pages)
    n, h, page, d, kps, vps = _cache(k_pages, vt_pages)
    dev, B = k_pages.device, kv_lens.shape[0]
    T, Hq, _ = q.shape
    if out is None:
        out = torch.empty((T, Hq, d), dtype=torch.bfloat16, device=dev)
    else:
        _dev_bf16(out)
    table = _table(block_table, dev, B)
    p = make_paged_params(batch=B, n_q_heads=Hq, n_kv_heads=h, head_dim=d, page_size=page, n_pages=n, max_pages=block_table.shape[1], n_tokens=T,
                          max_new_tokens=max_new_tokens, softmax_scale=softmax_scale, n_sink_tokens=n_sink_tokens, window_tokens=window_tokens,
                          softcap=softcap, table_stride=block_table.stride(0) if B > 1 else block_table.shape[1],
                          q=_rows("q", q, dev, T, Hq, d), out=_rows("out", out, dev, T, Hq, d), k_pages=kps, vt_pages=vps)
    if slopes is not None and (slopes.dtype != torch.float32 or slopes.device != dev or not slopes.is_contiguous() or tuple(slopes.shape) != (Hq,)):
        raise TypeError(f"slopes must be a contiguous fp32 tensor [{Hq}] on {dev}")
    lse = torch.empty((T, Hq), dtype=torch.float32, device=dev) if return_lse else None
    if workspace is None:
        workspace = torch.empty(paged_workspace_bytes(p), dtype=torch.uint8, device=dev)
    elif workspace.dtype != torch.uint8 or workspace.device != dev or not workspace.is_contiguous():
        raise TypeError(f"workspace must be a contiguous uint8 tensor on {dev}")
    with _on(dev):
        _check(load_library().sparse_prefill_paged_attn(
            ctypes.byref(p), q.data_ptr(), k_pages.data_ptr(), vt_pages.data_ptr(), table, _ints("q_starts", q_starts, dev, B + 1),
            _ints("kv_lens", kv_lens, dev, B), None if slopes is None else slopes.data_ptr(), out.data_ptr(),
            None if lse is None else lse.data_ptr(), workspace.data_ptr(), workspace.numel(), _stream(q)))
    return (out, lse) if return_lse else out

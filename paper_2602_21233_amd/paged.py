"""Binding of the paged-KV-cache calls of include/sparse_prefill.h: block tables and slot maps of a serving step, the new
tokens' keys and values into their pages, attention over the pages.  Argument marshalling only; a step makes these calls for
every layer and is short, so they are written for few Python operations."""
from __future__ import annotations

import ctypes
import functools
import struct

import torch

from . import binding
from .binding import SpaError, SpaPagedParams, _check, _raw_stream, load_library

# 9 int32, a float, 2 int32, a float, table_stride and six stride pairs: see SpaPagedParams
_PARAMS = struct.Struct("@9if2if13q")
assert _PARAMS.size == ctypes.sizeof(SpaPagedParams)
_pack = _PARAMS.pack
_I32, _BF16 = torch.int32, torch.bfloat16


def _unfit():
    """For a value that does not fit its field of the parameters."""
    return SpaError(-2, load_library().spa_strerror(-2).decode())


def make_paged_params(*, batch=1, n_q_heads=1, n_kv_heads=1, head_dim=64, page_size, n_pages, max_pages=1, n_tokens, max_new_tokens=0,
                      softmax_scale=None, n_sink_tokens=0, window_tokens=0, softcap=0.0, table_stride=1, q=(0, 0), k=(0, 0), v=(0, 0), out=(0, 0),
                      k_pages=(0, 0), vt_pages=(0, 0)) -> SpaPagedParams:
    """q, k, v, out: (token, head) strides; k_pages, vt_pages: (page, head) strides, all in elements."""
    try:
        return SpaPagedParams.from_buffer_copy(_pack(
            batch, n_q_heads, n_kv_heads, head_dim, page_size, n_pages, max_pages, n_tokens, max_new_tokens, softmax_scale or 0.0, n_sink_tokens,
            window_tokens, softcap, table_stride, *q, *k, *v, *out, *k_pages, *vt_pages))
    except (struct.error, OverflowError):
        raise _unfit() from None


def paged_workspace_bytes(p: SpaPagedParams) -> int:
    """sparse_prefill_paged_attn's scratch for these parameters."""
    return _workspace_bytes(bytes(p))


@functools.lru_cache(maxsize=256)                # by the sizes in the packed structure
def _workspace_bytes(packed: bytes) -> int:
    n = ctypes.c_size_t()
    _check(load_library().spa_paged_workspace_bytes(packed, ctypes.byref(n)))
    return n.value


def _bad_ints(name, n, device):
    return TypeError(f"{name} must be a contiguous int32 tensor [{n}] on {device}")


def _table(t, device, batch):
    """(address, columns, row stride)"""
    if t.dtype is not _I32 or t.device != device or t.dim() != 2:
        raise TypeError(f"block_table must be an int32 tensor [{batch}, max_pages] on {device}")
    rows, columns = t.shape
    stride, inner = t.stride()
    if rows != batch or (inner != 1 and columns > 1):
        raise TypeError(f"block_table must be an int32 tensor [{batch}, max_pages] with contiguous rows")
    return t.data_ptr(), columns, stride if rows > 1 else columns


def _rows(name, t, device, n, heads, dim):
    """(token, head) strides; an axis of one entry may have any, so it gets that of a dense tensor."""
    if t.dtype is not _BF16 or t.device != device or t.shape != (n, heads, dim):
        raise TypeError(f"{name} must be a bf16 tensor [{n}, {heads}, {dim}] on {device}")
    token, head, inner = t.stride()
    if inner != 1:
        raise TypeError(f"the last axis of {name} must be contiguous")
    if heads == 1:
        head = dim
    return (token if n > 1 else heads * head), head


def _cache(k_pages, vt_pages):
    """(n_pages, n_kv_heads, page_size, head_dim, K's page and head strides, V's, device)"""
    if k_pages.dim() != 4:
        raise TypeError("k_pages must be [n_pages, n_kv_heads, page_size, head_dim]")
    n, h, p, d = k_pages.shape
    device = k_pages.device
    if k_pages.dtype is not _BF16 or vt_pages.dtype is not _BF16 or not k_pages.is_cuda or vt_pages.device != device:
        raise TypeError("k_pages and vt_pages must be bf16 tensors on one GPU")
    k0, k1, k2, k3 = k_pages.stride()
    v0, v1, v2, v3 = vt_pages.stride()
    if vt_pages.shape != (n, h, d, p) or k3 != 1 or k2 != d or v3 != 1 or v2 != p:
        raise TypeError("k_pages must be [n_pages, n_kv_heads, page_size, head_dim] and vt_pages [n_pages, n_kv_heads, head_dim, page_size], the "
                        "two inner axes contiguous")
    if h == 1:
        k1 = v1 = p * d
    if n == 1:
        k0, v0 = h * k1, h * v1
    return n, h, p, d, k0, k1, v0, v1, device


def _launch(name, device, *args):
    """The library's call `name` with args and the current stream of the tensors' device, whichever device is current."""
    index = device.index
    if torch._C._cuda_getDevice() != index:
        with torch.cuda.device(device):
            return _launch(name, device, *args)
    stream = _raw_stream(index) if _raw_stream is not None else torch.cuda.current_stream(device).cuda_stream
    rc = getattr(binding._lib or load_library(), name)(*args, stream)
    if rc != 0:
        _check(rc)


def paged_plan(block_table, ctx_lens, new_lens, free_pages, free_range, n_tokens, page_size, n_pages):
    """sparse_prefill_paged_plan: block_table (int32 [B, max_pages]) gets the pages that the step takes from
    free_pages[free_range[0]:free_range[1]].  Returns (q_starts [B+1], kv_lens [B], slots [n_tokens], positions
    [n_tokens], taken [2]), int32 tensors that lie in one allocation."""
    dev = ctx_lens.device
    B, n_free = ctx_lens.shape[0], free_pages.shape[0]
    if not ctx_lens.is_cuda:
        raise TypeError("expected tensors on the GPU")
    for name, t, n in (("ctx_lens", ctx_lens, B), ("new_lens", new_lens, B), ("free_pages", free_pages, n_free), ("free_range", free_range, 2)):
        if t.dtype is not _I32 or t.device != dev or t.shape != (n,) or not t.is_contiguous():
            raise _bad_ints(name, n, dev)
    table, columns, stride = _table(block_table, dev, B)
    try:
        p = _pack(B, 1, 1, 64, page_size, n_pages, columns, n_tokens, 0, 0.0, 0, 0, 0.0, stride, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0)
    except (struct.error, OverflowError):
        raise _unfit() from None
    all_of = torch.empty(2 * B + 3 + 2 * n_tokens if n_tokens > 0 else 2 * B + 3, dtype=_I32, device=dev)
    at = all_of.data_ptr()
    kv, slots = at + 4 * (B + 1), at + 4 * (2 * B + 1)
    positions = slots + 4 * n_tokens
    _launch("sparse_prefill_paged_plan", dev, p, ctx_lens.data_ptr(), new_lens.data_ptr(), free_pages.data_ptr(), n_free, free_range.data_ptr(),
            table, at, kv, slots, positions, positions + 4 * n_tokens)
    return torch.split_with_sizes(all_of, (B + 1, B, n_tokens, n_tokens, 2))


def paged_append(k, v, slots, k_pages, vt_pages):
    """sparse_prefill_paged_append: k, v [n_tokens, n_kv_heads, head_dim] to the places slots (int32 [n_tokens], each
    once, or none: -1) of the cache."""
    n, h, page, d, k0, k1, v0, v1, dev = _cache(k_pages, vt_pages)
    T = slots.shape[0]
    if slots.dtype is not _I32 or slots.device != dev or slots.dim() != 1 or not slots.is_contiguous():
        raise _bad_ints("slots", T, dev)
    rows = *_rows("k", k, dev, T, h, d), *_rows("v", v, dev, T, h, d)
    try:
        p = _pack(1, h, h, d, page, n, 1, T, 0, 0.0, 0, 0, 0.0, 1, 0, 0, *rows, 0, 0, k0, k1, v0, v1)
    except (struct.error, OverflowError):
        raise _unfit() from None
    _launch("sparse_prefill_paged_append", dev, p, k.data_ptr(), v.data_ptr(), slots.data_ptr(), k_pages.data_ptr(), vt_pages.data_ptr())


def paged_attn(q, k_pages, vt_pages, block_table, q_starts, kv_lens, max_new_tokens=0, softmax_scale=None, n_sink_tokens=0,
               window_tokens=0, softcap=0.0, slopes=None, return_lse=False, out=None, workspace=None):
    """sparse_prefill_paged_attn: q [n_tokens, n_q_heads, head_dim] -> out of the same shape (and lse [n_tokens, n_q_heads] fp32).
    max_new_tokens: the most new tokens of a request, where the host knows it (decode steps are up to an eighth faster with it); slopes: fp32 [n_q_heads], bias by distance.
    Rows of padding are left as they are in `out` (as allocated where none is given)."""
    n, h, page, d, k0, k1, v0, v1, dev = _cache(k_pages, vt_pages)
    if q.dim() != 3 or kv_lens.dim() != 1:
        raise TypeError("q must be [n_tokens, n_q_heads, head_dim] and kv_lens [batch]")
    B = kv_lens.shape[0]
    T, Hq, _ = q.shape
    for name, t, many in (("q_starts", q_starts, B + 1), ("kv_lens", kv_lens, B)):
        if t.dtype is not _I32 or t.device != dev or t.shape != (many,) or not t.is_contiguous():
            raise _bad_ints(name, many, dev)
    q_token, q_head = _rows("q", q, dev, T, Hq, d)
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        o_token, o_head = Hq * d, d
    else:
        o_token, o_head = _rows("out", out, dev, T, Hq, d)
    table, columns, stride = _table(block_table, dev, B)
    if slopes is not None and (slopes.dtype is not torch.float32 or slopes.device != dev or slopes.shape != (Hq,) or not slopes.is_contiguous()):
        raise TypeError(f"slopes must be a contiguous fp32 tensor [{Hq}] on {dev}")
    try:
        p = _pack(B, Hq, h, d, page, n, columns, T, max_new_tokens, softmax_scale or 0.0, n_sink_tokens, window_tokens, softcap, stride,
                  q_token, q_head, 0, 0, 0, 0, o_token, o_head, k0, k1, v0, v1)
    except (struct.error, OverflowError):
        raise _unfit() from None
    lse = torch.empty((T, Hq), dtype=torch.float32, device=dev) if return_lse else None
    if workspace is None:
        ws_bytes = _workspace_bytes(p)
        if ws_bytes:
            workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
    elif workspace.dtype is not torch.uint8 or workspace.device != dev or not workspace.is_contiguous():
        raise TypeError(f"workspace must be a contiguous uint8 tensor on {dev}")
    else:
        ws_bytes = workspace.numel()
    _launch("sparse_prefill_paged_attn", dev, p, q.data_ptr(), k_pages.data_ptr(), vt_pages.data_ptr(), table, q_starts.data_ptr(),
            kv_lens.data_ptr(), None if slopes is None else slopes.data_ptr(), out.data_ptr(), None if lse is None else lse.data_ptr(),
            None if workspace is None else workspace.data_ptr(), ws_bytes)
    return (out, lse) if return_lse else out

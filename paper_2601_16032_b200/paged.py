"""Wrappers for torch CUDA tensors of the entry points around the paged key/value cache.

Like `forward` they only check and marshal: shapes, strides, pointers and the current stream of the tensors' device go
to the C ABI, where the remaining checks are made.  Outputs that are not given are allocated with torch.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

from . import binding as _b
from .binding import AttnError, KVCache, PagePool, RopeOpts


class PagePlan(NamedTuple):
    """What `page_plan` returns, all on the device: see attn_page_plan for each."""
    seq_len: object
    q_start: object
    slot: object
    position: object
    request: object
    free_count: object
    info: object


def _need(condition: bool, message: str) -> None:
    if not condition:
        raise AttnError(-1, message)


def _run(device, call, *args) -> None:
    """Calls `call(*args, stream)` with `device` current and its current stream."""
    import torch
    index = device.index
    if index == torch.cuda.current_device():
        call(*args, torch.cuda.current_stream().cuda_stream)
    else:
        with torch.cuda.device(index):
            call(*args, torch.cuda.current_stream().cuda_stream)


def _kind(t) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return _b.BF16
    if t.dtype == torch.float16:
        return _b.F16
    raise AttnError(-1, "tensors must be float16 or bfloat16")


def _rows(name: str, t, like) -> tuple:
    """The outer and inner stride of a [outer, inner, d] tensor for the C ABI (both 0: contiguous)."""
    _need(t.dim() == 3 and t.device == like.device and t.dtype == like.dtype, f"{name} must be a tensor of three dimensions, of q's type and on its device")
    n, h, d = t.shape
    a, b, c = t.stride()
    _need(c == 1 or d <= 1, f"{name}: the elements of a row must be contiguous")
    if n <= 1:
        a = 0 if h > 1 else h * d
    if h <= 1:
        b = 0
    _need(a != 0 or b != 0 or n * h <= 1, f"{name} must not be expanded over both of its outer dimensions")
    return a, b


def _ints(name: str, t, shape: tuple, device, dtype) -> int:
    """The address of a contiguous tensor of this shape and type on this device."""
    _need(t.dtype == dtype and t.device == device and t.is_contiguous() and tuple(t.shape) == shape,
          f"{name} must be a contiguous {dtype} tensor of shape {shape} on the device of the others")
    return t.data_ptr()


def _cache(k_cache, v_cache, layout: int, kv_heads: int, d: int, like) -> KVCache:
    _need(k_cache.dim() == 4 and k_cache.shape == v_cache.shape and k_cache.stride() == v_cache.stride() and k_cache.dtype == v_cache.dtype == like.dtype
          and k_cache.device == v_cache.device == like.device, "k_cache and v_cache must be alike: four dimensions, q's type and device, the same strides")
    _need(layout in (_b.LAYOUT_BHND, _b.LAYOUT_BNHD), f"unknown layout {layout}")
    shape, stride = k_cache.shape, [0 if n <= 1 else s for n, s in zip(k_cache.shape, k_cache.stride())]
    token, head = (1, 2) if layout == _b.LAYOUT_BNHD else (2, 1)
    _need(k_cache.stride(3) == 1 and shape[3] == d and shape[head] == kv_heads, "the cache must hold rows of d contiguous elements for k's heads")
    return KVCache(k_cache.data_ptr(), v_cache.data_ptr(), shape[0], stride[0], stride[token], stride[head], shape[token], kv_heads, d, _kind(like), layout)


def page_plan(cached, added, page_size: int, block_table, free_pages, free_count, token_cap: int, *, seq_len=None, free_count_out=None) -> PagePlan:
    """Block tables, slots and positions of a serving step (attn_page_plan).

    cached, added: [B] int32.  block_table [B, width] int32 and free_pages [capacity] int32 are updated in place;
    free_count [1] int32 is read, its new value goes to free_count_out (a new tensor if not given; may be free_count).
    seq_len: the new lengths (a new tensor if not given; may be cached).
    """
    import torch
    device, int32 = cached.device, torch.int32
    _need(cached.is_cuda, "the tensors must be CUDA tensors")
    B = cached.numel()
    _need(block_table.dim() == 2 and block_table.dtype == int32 and block_table.device == device and block_table.shape[0] == B and block_table.shape[1] > 0
          and block_table.stride(1) == 1, "block_table must be an int32 tensor [B, width] on the device of the others with contiguous rows")
    _need(token_cap >= 0, "token_cap must not be negative")
    seq_len = torch.empty_like(cached) if seq_len is None else seq_len
    free_count_out = torch.empty_like(free_count) if free_count_out is None else free_count_out
    whole = torch.empty(B + 5 + 2 * token_cap, dtype=int32, device=device)      # one allocation for the small ones
    q_start, info, position, request = whole.split((B + 1, 4, token_cap, token_cap))
    slot = torch.empty(token_cap, dtype=torch.int64, device=device)
    width = block_table.shape[1]
    pool = PagePool(block_table.data_ptr(), block_table.stride(0) if B > 1 else width, _ints("free_pages", free_pages, (free_pages.numel(),), device, int32),
                    _ints("free_count", free_count, (1,), device, int32), _ints("free_count_out", free_count_out, (1,), device, int32), width,
                    free_pages.numel(), page_size)
    _run(device, _b.attn_page_plan, pool, _ints("cached", cached, (B,), device, int32), _ints("added", added, (B,), device, int32), B,
         _ints("seq_len", seq_len, (B,), device, int32), q_start.data_ptr(), slot.data_ptr(), position.data_ptr(), request.data_ptr(), token_cap,
         info.data_ptr())
    return PagePlan(seq_len, q_start, slot, position, request, free_count_out, info)


def _rotation(position, inv_freq, T: int, device) -> tuple:
    import torch
    if inv_freq is None:
        return 0, 0, 0
    _need(position is not None, "a rotation needs position")
    return (_ints("position", position, (T,), device, torch.int32), _ints("inv_freq", inv_freq, (inv_freq.numel(),), device, torch.float64), 2 * inv_freq.numel())


def _weights(q_weight, k_weight, d: int, like) -> tuple:
    import torch
    given = [w for w in (q_weight, k_weight) if w is not None]
    f32 = any(w.dtype == torch.float32 for w in given)
    kind = torch.float32 if f32 else like.dtype
    return tuple(0 if w is None else _ints("weight", w, (d,), like.device, kind) for w in (q_weight, k_weight)) + (int(f32),)


def qk_norm_rope(q, k, v=None, *, q_weight=None, k_weight=None, eps: float = 1e-6, position=None, inv_freq=None, interleaved: bool = False,
                 k_cache=None, v_cache=None, cache_layout: int = _b.LAYOUT_BNHD, slot=None, q_out=None, k_out=None):
    """RMS norm of every head of q and k, the position rotation and the append to the paged cache (attn_qk_norm_rope).

    q [T, H, d], k and v [T, kv_heads, d], any token and head strides; weights [d] (q's type or float32; None: no norm); position
    [T] int32; inv_freq [rot_dim / 2] float64 (None: no rotation); slot [T] int64 with k_cache, v_cache ([page, token, head, d],
    or [page, head, token, d] with LAYOUT_BHND).  Returns (q_out, k_out); k_out is None if it is not given and there is a cache.
    """
    import torch
    _need(q.is_cuda and q.dim() == 3, "q must be a CUDA tensor [T, H, d]")
    T, H, d = q.shape
    kv_heads = k.shape[1] if k.dim() == 3 else 0
    _need(k.dim() == 3 and k.shape == (T, kv_heads, d) and (v is None or v.shape == k.shape), "k and v must be [T, kv_heads, d]")
    cached = k_cache is not None
    _need(cached == (v_cache is not None) == (slot is not None) == (v is not None), "k_cache, v_cache, slot and v go together")
    q_out = torch.empty((T, H, d), dtype=q.dtype, device=q.device) if q_out is None else q_out
    if k_out is None and not cached:
        k_out = torch.empty((T, kv_heads, d), dtype=q.dtype, device=q.device)
    _need(q_out.shape == q.shape and (k_out is None or k_out.shape == k.shape), "q_out and k_out must have the shapes of q and k")
    where, freq, rot = _rotation(position, inv_freq, T, q.device)
    wq, wk, f32 = _weights(q_weight, k_weight, d, q)
    cache = _cache(k_cache, v_cache, cache_layout, kv_heads, d, q) if cached else None
    opts = RopeOpts(*_rows("q", q, q), *_rows("k", k, q), *(_rows("v", v, q) if cached else (0, 0)), *_rows("q_out", q_out, q),
                    *(_rows("k_out", k_out, q) if k_out is not None else (0, 0)), 0, 0, 0, 0,
                    ctypes.pointer(cache) if cached else None, _ints("slot", slot, (T,), q.device, torch.int64) if cached else None, f32)
    if T > 0:
        _run(q.device, lambda stream: _b.attn_qk_norm_rope(
            q.data_ptr(), k.data_ptr(), v.data_ptr() if cached else 0, q_out.data_ptr(), k_out.data_ptr() if k_out is not None else 0, T, H, kv_heads, d,
            _kind(q), wq, wk, eps, where, freq, rot, int(interleaved), stream, opts))
    return q_out, k_out


def qk_norm_rope_backward(dq_out, dk_out, q, k, *, q_weight=None, k_weight=None, eps: float = 1e-6, position=None, inv_freq=None,
                          interleaved: bool = False, dq=None, dk=None, workspace=None):
    """Gradients of qk_norm_rope's norm and rotation (attn_qk_norm_rope_bwd): (dq, dk, dq_weight, dk_weight).

    dq_out, dk_out: gradients of q_out and k_out; q, k and the rest as given to qk_norm_rope.  dq_weight, dk_weight: float32 (None without
    the weight).  workspace: a tensor of at least attn_rope_bwd_workspace_bytes(d) bytes (allocated if not given).
    """
    import torch
    _need(q.is_cuda and q.dim() == 3 and k.dim() == 3, "q must be a CUDA tensor [T, H, d], k [T, kv_heads, d]")
    T, H, d = q.shape
    kv_heads = k.shape[1]
    dq = torch.empty((T, H, d), dtype=q.dtype, device=q.device) if dq is None else dq
    dk = torch.empty((T, kv_heads, d), dtype=q.dtype, device=q.device) if dk is None else dk
    _need(k.shape == (T, kv_heads, d) and dq_out.shape == dq.shape == q.shape and dk_out.shape == dk.shape == k.shape, "gradients must have the shapes of q and k")
    if workspace is None:
        workspace = torch.empty(_b.attn_rope_bwd_workspace_bytes(d), dtype=torch.uint8, device=q.device)
    _need(workspace.device == q.device and workspace.is_contiguous(), "workspace must be a contiguous tensor on q's device")
    where, freq, rot = _rotation(position, inv_freq, T, q.device)
    wq, wk, f32 = _weights(q_weight, k_weight, d, q)
    both = torch.empty((2, d), dtype=torch.float32, device=q.device)
    dq_weight, dk_weight = (both[0] if wq else None), (both[1] if wk else None)
    opts = RopeOpts(*_rows("q", q, q), *_rows("k", k, q), 0, 0, *_rows("dq_out", dq_out, q), *_rows("dk_out", dk_out, q), *_rows("dq", dq, q),
                    *_rows("dk", dk, q), None, None, f32)
    if T == 0:
        both.zero_()
    else:
        _run(q.device, lambda stream: _b.attn_qk_norm_rope_bwd(
            dq_out.data_ptr(), dk_out.data_ptr(), q.data_ptr(), k.data_ptr(), dq.data_ptr(), dk.data_ptr(), dq_weight.data_ptr() if wq else 0,
            dk_weight.data_ptr() if wk else 0, T, H, kv_heads, d, _kind(q), wq, wk, eps, where, freq, rot, int(interleaved), workspace.data_ptr(),
            workspace.numel() * workspace.element_size(), stream, opts))
    return dq, dk, dq_weight, dk_weight

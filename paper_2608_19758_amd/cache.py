"""Paged KV cache: append, attention, weights and eviction (argument marshalling
over the ``fp2_cache_*`` entry points of ``include/fp2.h``, which states their
semantics and layouts).

A cache is a ``KVCache``: pools of token slots in bf16, in e4m3 codes with one
fp32 scale per head (what ``prefill`` reads), or in e4m3 codes with one
power-of-two scale for each block of ``scale_tokens`` tokens and head.
``make_cache_params`` describes a call, ``alloc_cache`` makes an empty cache
for it.
"""
from __future__ import annotations

import contextlib
import ctypes
import dataclasses
from typing import Optional

import torch

from . import (_INT32, _F32, BF16, FP8_E4M3, HEAD_DIM, _check, _host_ptr, _need, _ptr, lib)


class CacheParams(ctypes.Structure):
    """Mirror of fp2_cache_params_t."""
    _fields_ = [(n, ctypes.c_int32) for n in (
        "batch", "num_q_heads", "num_kv_heads", "head_dim", "page_size", "max_pages_per_seq",
        "max_seq_len", "max_kv_len", "dtype", "scale_tokens", "sink_tokens", "window_tokens",
        "kv_splits")] + [("softmax_scale", ctypes.c_float)]


class _CachePointers(ctypes.Structure):
    """Mirror of fp2_kv_cache_t."""
    _fields_ = [(n, ctypes.c_void_p) for n in (
        "k", "v", "k_head_scale", "v_head_scale", "k_block_scale", "v_block_scale")]


@dataclasses.dataclass
class KVCache:
    """One layer's cache. k and v: [slots, num_kv_heads, 128] in bf16 or one-byte codes.
    Codes: k_scale and v_scale fp32 [num_kv_heads], or, with scale_tokens > 0, uint8
    [slots / scale_tokens, num_kv_heads] of the powers 2^(byte - 127)."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: Optional[torch.Tensor] = None
    v_scale: Optional[torch.Tensor] = None


def make_cache_params(*, batch, num_q_heads, num_kv_heads, max_seq_len, max_kv_len, page_size,
                      max_pages_per_seq=0, dtype="bf16", scale_tokens=0, sink_tokens=0,
                      window_tokens=0, softmax_scale=0.0, kv_splits=0,
                      head_dim=HEAD_DIM) -> CacheParams:
    """fp2_cache_params_t. max_seq_len bounds the new tokens of a sequence in the call,
    max_kv_len its tokens in the cache; max_pages_per_seq 0: what max_kv_len needs;
    dtype ("bf16" or "fp8") and scale_tokens (0: a scale per head) are the cache's."""
    dt = {"bf16": BF16, "fp8": FP8_E4M3}.get(dtype, dtype)
    pages = max_pages_per_seq or (max_kv_len + page_size - 1) // max(1, page_size)
    return CacheParams(batch=batch, num_q_heads=num_q_heads, num_kv_heads=num_kv_heads,
                       head_dim=head_dim, page_size=page_size, max_pages_per_seq=pages,
                       max_seq_len=max_seq_len, max_kv_len=max_kv_len, dtype=dt,
                       scale_tokens=scale_tokens, sink_tokens=sink_tokens,
                       window_tokens=window_tokens, softmax_scale=softmax_scale,
                       kv_splits=kv_splits)


def cache_workspace_bytes(p: CacheParams) -> int:
    return int(lib().fp2_cache_workspace_bytes(ctypes.byref(p)))


def alloc_cache_workspace(p: CacheParams, device="cuda") -> torch.Tensor:
    return torch.empty(max(1, cache_workspace_bytes(p)), dtype=torch.uint8, device=device)


def alloc_cache(p: CacheParams, num_pages: int, device="cuda", k_scale=None, v_scale=None) -> KVCache:
    """An empty cache of num_pages pages. Codes with a scale per head need the scales
    (fp32 [num_kv_heads]) from the caller; block scales start at 1."""
    shape = (num_pages * p.page_size, p.num_kv_heads, p.head_dim)
    dt = torch.bfloat16 if p.dtype == BF16 else torch.uint8
    if p.dtype == FP8_E4M3 and p.scale_tokens == 0:
        if k_scale is None or v_scale is None:
            raise ValueError("a cache with a scale per head needs k_scale and v_scale")
    elif k_scale is not None or v_scale is not None:
        raise ValueError("k_scale and v_scale are for caches with a scale per head")
    elif p.scale_tokens:
        rows = (shape[0] // p.scale_tokens, p.num_kv_heads)
        k_scale, v_scale = (torch.full(rows, 127, dtype=torch.uint8, device=device) for _ in "kv")
    return KVCache(torch.zeros(shape, dtype=dt, device=device),
                   torch.zeros(shape, dtype=dt, device=device), k_scale, v_scale)


_ROWS = {BF16: (torch.bfloat16,), FP8_E4M3: (torch.uint8, torch.float8_e4m3fn)}
_BF16 = (torch.bfloat16,)


def _check_cache(p: CacheParams, c: KVCache, need_v=True):
    row = p.num_kv_heads * p.head_dim
    slots = c.k.numel() // max(1, row)
    for name, t, s in (("k", c.k, c.k_scale), ("v", c.v, c.v_scale)):
        if t is None and not need_v and name == "v":
            continue
        _need(t, "cache." + name, dtypes=_ROWS.get(p.dtype), divisible=max(1, row * p.page_size))
        if t.numel() != c.k.numel():
            raise ValueError("cache.k and cache.v differ in size")
        if p.dtype != FP8_E4M3:
            continue
        if s is None:
            raise ValueError("cache.%s_scale is missing" % name)
        if p.scale_tokens > 0:
            _need(s, "cache.%s_scale" % name, dtypes=(torch.uint8,),
                  min_numel=slots // p.scale_tokens * p.num_kv_heads)
        else:
            _need(s, "cache.%s_scale" % name, dtypes=_F32, min_numel=p.num_kv_heads)


def _check_table(p: CacheParams, name, t, width):
    _need(t, name, dtypes=_INT32)
    if t.dim() != 2 or t.shape[1] != width or t.shape[0] < p.batch:
        raise ValueError("%s must be int32 [>= batch, %d], got %s" % (name, width, tuple(t.shape)))


def _pointers(p: CacheParams, c: KVCache):
    block = p.scale_tokens > 0
    ks, vs = _ptr(c.k_scale), _ptr(c.v_scale)
    return _CachePointers(_ptr(c.k), _ptr(c.v), None if block else ks, None if block else vs,
                          ks if block else None, vs if block else None)


def _same_device(named):
    """Every tensor is a CUDA tensor, all on one device, which is returned."""
    dev = None
    for name, t in named:
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError("%s must be a CUDA tensor" % name)
        dev = t.device if dev is None else dev
        if t.device != dev:
            raise ValueError("%s is on %s, other arguments on %s" % (name, t.device, dev))
    return dev


def _on(dev, stream):
    """The device made current for the call, and the stream to use (dev's current one if None)."""
    if stream is None:
        stream = torch.cuda.current_stream(dev)
    elif stream.device != dev:
        raise ValueError("stream is on %s, the tensors on %s" % (stream.device, dev))
    same = torch.cuda.current_device() == dev.index
    return (contextlib.nullcontext() if same else torch.cuda.device(dev)), ctypes.c_void_p(stream.cuda_stream)


def _lengths(p, cu_seqlens, cu_seqlens_k, host, host_k):
    for name, t in (("cu_seqlens", cu_seqlens), ("cu_seqlens_k", cu_seqlens_k)):
        _need(t, name, dtypes=_INT32, min_numel=p.batch + 1)
    for name, t in (("cu_seqlens_host", host), ("cu_seqlens_k_host", host_k)):
        if t is None:
            continue
        size = t.numel() if isinstance(t, torch.Tensor) else t.size
        if str(t.dtype).replace("torch.", "") != "int32" or size < p.batch + 1 \
                or (isinstance(t, torch.Tensor) and t.is_cuda):
            raise ValueError("%s must be a host int32 array of batch + 1 entries" % name)


def _queries(p, q, name="q"):
    _need(q, name, dtypes=_BF16, divisible=p.num_q_heads * p.head_dim)
    return q.numel() // (p.num_q_heads * p.head_dim)


def cache_append(p: CacheParams, k_new, v_new, cache: KVCache, cu_seqlens, cu_seqlens_k, block_table,
                 *, cu_seqlens_host=None, cu_seqlens_k_host=None, stream=None) -> None:
    """fp2_cache_append: k_new and v_new bf16 [new tokens, num_kv_heads, 128] into the
    cache's pages, in its type."""
    _check_cache(p, cache)
    for name, t in (("k_new", k_new), ("v_new", v_new)):
        _need(t, name, dtypes=_BF16, divisible=p.num_kv_heads * p.head_dim)
    if k_new.numel() != v_new.numel():
        raise ValueError("k_new and v_new differ in size")
    _lengths(p, cu_seqlens, cu_seqlens_k, cu_seqlens_host, cu_seqlens_k_host)
    _check_table(p, "block_table", block_table, p.max_pages_per_seq)
    dev = _same_device((("cache.k", cache.k), ("cache.v", cache.v), ("cache.k_scale", cache.k_scale),
                        ("cache.v_scale", cache.v_scale), ("k_new", k_new), ("v_new", v_new),
                        ("cu_seqlens", cu_seqlens), ("cu_seqlens_k", cu_seqlens_k),
                        ("block_table", block_table)))
    c = _pointers(p, cache)
    guard, s = _on(dev, stream)
    with guard:
        _check("fp2_cache_append", lib().fp2_cache_append(
            ctypes.byref(p), _ptr(k_new), _ptr(v_new), _ptr(cu_seqlens), _host_ptr(cu_seqlens_host),
            _ptr(cu_seqlens_k), _host_ptr(cu_seqlens_k_host), ctypes.byref(c), _ptr(block_table), s))


def cache_attend(p: CacheParams, q, cache: KVCache, cu_seqlens, cu_seqlens_k, block_table, *, out=None,
                 lse=None, want_lse=False, workspace=None, cu_seqlens_host=None,
                 cu_seqlens_k_host=None, stream=None):
    """fp2_cache_attend: returns (out bf16 like q, lse fp32 [tokens, num_q_heads] or None)."""
    rows = _queries(p, q)
    _check_cache(p, cache)
    _lengths(p, cu_seqlens, cu_seqlens_k, cu_seqlens_host, cu_seqlens_k_host)
    _check_table(p, "block_table", block_table, p.max_pages_per_seq)
    if out is None:
        out = torch.empty_like(q)
    if lse is None and want_lse:
        lse = torch.empty((rows, p.num_q_heads), dtype=torch.float32, device=q.device)
    _need(out, "out", dtypes=_BF16, min_numel=q.numel())
    _need(lse, "lse", dtypes=_F32, min_numel=rows * p.num_q_heads)
    if workspace is None:
        workspace = alloc_cache_workspace(p, q.device)
    _need(workspace, "workspace", esz=1)
    dev = _same_device((("q", q), ("cache.k", cache.k), ("cache.v", cache.v),
                        ("cache.k_scale", cache.k_scale), ("cache.v_scale", cache.v_scale),
                        ("cu_seqlens", cu_seqlens), ("cu_seqlens_k", cu_seqlens_k),
                        ("block_table", block_table), ("out", out), ("lse", lse),
                        ("workspace", workspace)))
    c = _pointers(p, cache)
    guard, s = _on(dev, stream)
    with guard:
        _check("fp2_cache_attend", lib().fp2_cache_attend(
            ctypes.byref(p), _ptr(q), _ptr(cu_seqlens), _host_ptr(cu_seqlens_host),
            _ptr(cu_seqlens_k), _host_ptr(cu_seqlens_k_host), ctypes.byref(c), _ptr(block_table),
            _ptr(out), _ptr(lse), _ptr(workspace), workspace.numel(), s))
    return out, lse


def _weight_rows(p: CacheParams, name, w):
    _need(w, name, dtypes=_F32)
    if w.dim() != 3 or w.shape[0] < p.batch or w.shape[1] != p.num_kv_heads or w.shape[2] < p.max_kv_len:
        raise ValueError("%s must be fp32 [>= batch, num_kv_heads, >= max_kv_len], got %s"
                         % (name, tuple(w.shape)))


def cache_weights(p: CacheParams, q, lse, cache: KVCache, cu_seqlens, cu_seqlens_k, block_table, *,
                  weights=None, weights_in=None, workspace=None, cu_seqlens_host=None,
                  cu_seqlens_k_host=None, stream=None):
    """fp2_cache_weights: weights = weights_in (zeros if None) plus what each cached token
    received of these queries, fp32 [batch, num_kv_heads, max_kv_len or more]. To add in
    place give the same tensor as both. A result that is allocated here starts as a copy of
    weights_in (zeros without one), so entries past a sequence are defined."""
    rows = _queries(p, q)
    _check_cache(p, cache, need_v=False)
    _lengths(p, cu_seqlens, cu_seqlens_k, cu_seqlens_host, cu_seqlens_k_host)
    _check_table(p, "block_table", block_table, p.max_pages_per_seq)
    _need(lse, "lse", dtypes=_F32, min_numel=rows * p.num_q_heads)
    if weights_in is not None:
        _weight_rows(p, "weights_in", weights_in)
    if weights is None:
        weights = (torch.zeros((p.batch, p.num_kv_heads, p.max_kv_len), dtype=torch.float32, device=q.device)
                   if weights_in is None else weights_in.clone())
    _weight_rows(p, "weights", weights)
    if weights_in is not None and weights_in.shape[2] != weights.shape[2]:
        raise ValueError("weights and weights_in differ in their last size")
    if workspace is None:
        workspace = alloc_cache_workspace(p, q.device)
    _need(workspace, "workspace", esz=1)
    dev = _same_device((("q", q), ("lse", lse), ("cache.k", cache.k), ("cache.k_scale", cache.k_scale),
                        ("cu_seqlens", cu_seqlens), ("cu_seqlens_k", cu_seqlens_k),
                        ("block_table", block_table), ("weights", weights), ("weights_in", weights_in),
                        ("workspace", workspace)))
    c = _pointers(p, cache)
    guard, s = _on(dev, stream)
    with guard:
        _check("fp2_cache_weights", lib().fp2_cache_weights(
            ctypes.byref(p), _ptr(q), _ptr(lse), _ptr(cu_seqlens), _host_ptr(cu_seqlens_host),
            _ptr(cu_seqlens_k), _host_ptr(cu_seqlens_k_host), ctypes.byref(c), _ptr(block_table),
            _ptr(weights_in), _ptr(weights), weights.shape[2], _ptr(workspace), workspace.numel(), s))
    return weights


def cache_evict(p: CacheParams, cache: KVCache, weights, cu_seqlens_k, block_table, target_table, *,
                budget: int, recent_tokens: int = 0, kept=None, cu_seqlens_k_out=None,
                weights_out=None, cu_seqlens_k_host=None, stream=None):
    """fp2_cache_evict: the `budget` tokens of each sequence and KV head that stay go to the
    pages of target_table (int32 [batch, pages], other pages than block_table's). Returns
    (kept int32 [batch, num_kv_heads, budget], the new cu_seqlens_k, the weights that stay)."""
    _check_cache(p, cache)
    _need(cu_seqlens_k, "cu_seqlens_k", dtypes=_INT32, min_numel=p.batch + 1)
    _lengths(p, None, None, None, cu_seqlens_k_host)
    _check_table(p, "block_table", block_table, p.max_pages_per_seq)
    if not (isinstance(target_table, torch.Tensor) and target_table.dim() == 2):
        raise ValueError("target_table must be int32 [>= batch, pages]")
    _check_table(p, "target_table", target_table, target_table.shape[1])
    _weight_rows(p, "weights", weights)
    dev = cache.k.device
    if kept is None:
        kept = torch.empty((p.batch, p.num_kv_heads, max(1, budget)), dtype=torch.int32, device=dev)
    if cu_seqlens_k_out is None:
        cu_seqlens_k_out = torch.empty(p.batch + 1, dtype=torch.int32, device=dev)
    if weights_out is None:
        weights_out = torch.empty_like(weights)
    _need(kept, "kept", dtypes=_INT32, min_numel=p.batch * p.num_kv_heads * budget)
    _need(cu_seqlens_k_out, "cu_seqlens_k_out", dtypes=_INT32, min_numel=p.batch + 1)
    _weight_rows(p, "weights_out", weights_out)
    if weights_out.shape[2] != weights.shape[2]:
        raise ValueError("weights and weights_out differ in their last size")
    dev = _same_device((("cache.k", cache.k), ("cache.v", cache.v), ("cache.k_scale", cache.k_scale),
                        ("cache.v_scale", cache.v_scale), ("weights", weights),
                        ("cu_seqlens_k", cu_seqlens_k), ("block_table", block_table),
                        ("target_table", target_table), ("kept", kept),
                        ("cu_seqlens_k_out", cu_seqlens_k_out), ("weights_out", weights_out)))
    c = _pointers(p, cache)
    guard, s = _on(dev, stream)
    with guard:
        _check("fp2_cache_evict", lib().fp2_cache_evict(
            ctypes.byref(p), ctypes.byref(c), _ptr(cu_seqlens_k), _host_ptr(cu_seqlens_k_host),
            _ptr(block_table), _ptr(target_table), target_table.shape[1], int(budget),
            int(recent_tokens), _ptr(weights), _ptr(weights_out), weights.shape[2], _ptr(kept),
            _ptr(cu_seqlens_k_out), s))
    return kept, cu_seqlens_k_out, weights_out

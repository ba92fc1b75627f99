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

import numpy as np
import torch

from . import _F32, _INT32, BF16, FP8_E4M3, HEAD_DIM, _check, lib


CACHE_WORKSPACE_MAX = 140 << 20     # FP2_CACHE_WORKSPACE_MAX


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


_BYTES = (torch.uint8, torch.int8)
_CODES = (torch.uint8, torch.float8_e4m3fn)
_ONE_BF16, _ONE_U8, _ONE_F32, _ONE_I32 = ((t,) for t in (torch.bfloat16, torch.uint8, *_F32, *_INT32))
_NUMPY_I32 = np.dtype(np.int32)


class _Args:
    """Checks tensors one by one and gives their addresses: CUDA tensors on one device, dense, of the
    right type and of at least `least` elements. The C ABI sees only pointers, and refuses a null one where
    a call needs it, so `optional` says which this class lets through. (Half of a small call's
    time is spent here, so each property of a tensor is asked for once.)"""
    __slots__ = ("dev", "odd")

    def __init__(self):
        self.dev = None     # index of the first tensor's device
        self.odd = None     # first tensor that is not on a CUDA device, or on another one; refused at the end

    def __call__(self, name, t, dtypes, least=0, multiple=1, optional=False):
        if t is None and optional:
            return None
        if not isinstance(t, torch.Tensor):
            raise ValueError("%s must be a torch tensor" % name)
        if t.dtype not in dtypes:
            raise ValueError("%s must have dtype in %s, got %s" % (name, dtypes, t.dtype))
        if not t.is_contiguous():
            raise ValueError("%s must be contiguous" % name)
        if least or multiple > 1:
            n = t.numel()
            if n < least or n % multiple:
                raise ValueError("%s holds %d elements, needs at least %d and a multiple of %d"
                                 % (name, n, least, multiple))
        dev = t.get_device()
        if dev != self.dev or dev < 0:
            if self.dev is None:
                self.dev = dev
            if (dev != self.dev or dev < 0) and self.odd is None:
                self.odd = (name, t.device)
        return t.data_ptr()

    def table(self, batch, name, t, width):
        shape = t.shape if isinstance(t, torch.Tensor) else ()
        if len(shape) != 2 or shape[1] != width or shape[0] < batch:
            raise ValueError("%s must be int32 [>= batch, %d], got %s" % (name, width, tuple(shape)))
        return self(name, t, _ONE_I32)

    def weights(self, p, name, w, optional=False):
        if w is None and optional:
            return None
        shape = w.shape if isinstance(w, torch.Tensor) else ()
        if len(shape) != 3 or shape[0] < p.batch or shape[1] != p.num_kv_heads or shape[2] < p.max_kv_len:
            raise ValueError("%s must be fp32 [>= batch, num_kv_heads, >= max_kv_len], got %s"
                             % (name, tuple(shape)))
        return self(name, w, _ONE_F32)

    def cache(self, p, c, need_v=True):
        """fp2_kv_cache_t of the cache."""
        if c is None:
            raise ValueError("cache must be a KVCache")
        heads, scale_tokens, dtype = p.num_kv_heads, p.scale_tokens, p.dtype
        row = max(1, heads * p.head_dim * max(1, p.page_size))
        rows = _ONE_BF16 if dtype == BF16 else _CODES if dtype == FP8_E4M3 else ()
        k = self("cache.k", c.k, rows, 0, row)
        v = self("cache.v", c.v, rows, optional=True)
        size = c.k.numel()
        if v is not None and c.v.numel() != size:
            raise ValueError("cache.k and cache.v differ in size")
        if dtype != FP8_E4M3:
            return _CachePointers(k, v, None, None, None, None)
        if c.k_scale is None or (need_v and c.v_scale is None):
            raise ValueError("cache.k_scale or cache.v_scale is missing")
        if scale_tokens > 0:
            least = size // (scale_tokens * p.head_dim)
            ks, vs = (self("cache.k_scale", c.k_scale, _ONE_U8, least),
                      self("cache.v_scale", c.v_scale, _ONE_U8, least, optional=not need_v))
            return _CachePointers(k, v, None, None, ks, vs)
        ks, vs = (self("cache.k_scale", c.k_scale, _ONE_F32, heads),
                  self("cache.v_scale", c.v_scale, _ONE_F32, heads, optional=not need_v))
        return _CachePointers(k, v, ks, vs, None, None)

    @staticmethod
    def host(name, t, batch, rows=None):
        """Address of a host array of lengths; `rows`: new tokens that the call's tensors hold."""
        if t is None:
            return None
        if isinstance(t, torch.Tensor):
            ok = t.dtype == torch.int32 and not t.is_cuda and t.is_contiguous()
            size, at = t.numel(), t.data_ptr()
        else:
            ok = isinstance(t, np.ndarray) and t.dtype == _NUMPY_I32 and t.flags.c_contiguous
            size, at = t.size if ok else 0, None
        if not ok:
            raise ValueError("%s must be a dense host int32 array" % name)
        if size < batch + 1:
            raise ValueError("%s must have batch + 1 entries" % name)
        if rows is not None and t[batch] > rows:
            raise ValueError("%d new tokens, tensors hold %d" % (int(t[batch]), rows))
        if at is None:   # (.ctypes.data takes five times as long, and serves arrays that are read-only)
            at = ctypes.byref(ctypes.c_int32.from_buffer(t)) if t.flags.writeable else t.ctypes.data
        return at

    def lengths(self, batch, cu, cuk, host, host_k, rows=None):
        return (self("cu_seqlens", cu, _ONE_I32, batch + 1, optional=True), self.host("cu_seqlens_host", host, batch, rows),
                self("cu_seqlens_k", cuk, _ONE_I32, batch + 1, optional=True), self.host("cu_seqlens_k_host", host_k, batch))

    def call(self, name, stream, *args):
        """The entry point on `stream` (the current one of the tensors' device if None), with that
        device made current."""
        if self.odd is not None:
            raise ValueError("%s must be a CUDA tensor on the device of the others (%s), got one on %s"
                             % (self.odd[0], self.dev, self.odd[1]))
        if stream is None:
            handle = torch._C._cuda_getCurrentRawStream(self.dev)
        elif stream.device.index != self.dev:
            raise ValueError("stream is on %s, the tensors on cuda:%d" % (stream.device, self.dev))
        else:
            handle = stream.cuda_stream
        if torch.cuda.current_device() == self.dev:
            st = getattr(lib(), name)(*args, handle)
        else:
            with torch.cuda.device(self.dev):
                st = getattr(lib(), name)(*args, handle)
        if st:
            _check(name, st)


def on_stream(stream):
    """What is allocated for a call belongs to the stream that it runs on: the allocator may give the
    memory to later work there, and to no other stream's."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def cache_append(p: CacheParams, k_new, v_new, cache: KVCache, cu_seqlens, cu_seqlens_k, block_table,
                 *, cu_seqlens_host=None, cu_seqlens_k_host=None, stream=None) -> None:
    """fp2_cache_append: k_new and v_new bf16 [new tokens, num_kv_heads, 128] into the
    cache's pages, in its type."""
    a, batch = _Args(), p.batch
    c = a.cache(p, cache)
    row = p.num_kv_heads * p.head_dim
    k, v = a("k_new", k_new, _ONE_BF16), a("v_new", v_new, _ONE_BF16)
    size = k_new.numel()
    if size != v_new.numel() or size % row:
        raise ValueError("k_new and v_new must be of one size and hold rows of %d" % row)
    lens = a.lengths(batch, cu_seqlens, cu_seqlens_k, cu_seqlens_host, cu_seqlens_k_host, size // row)
    table = a.table(batch, "block_table", block_table, p.max_pages_per_seq)
    a.call("fp2_cache_append", stream, ctypes.byref(p), k, v, *lens, ctypes.byref(c), table)


def cache_attend(p: CacheParams, q, cache: KVCache, cu_seqlens, cu_seqlens_k, block_table, *, out=None,
                 lse=None, want_lse=False, workspace=None, cu_seqlens_host=None,
                 cu_seqlens_k_host=None, stream=None):
    """fp2_cache_attend: returns (out bf16 like q, lse fp32 [tokens, num_q_heads] or None)."""
    a, batch, heads = _Args(), p.batch, p.num_q_heads
    row = heads * p.head_dim
    qp = a("q", q, _ONE_BF16, 0, row)
    size = q.numel()
    rows = size // row
    c = a.cache(p, cache)
    lens = a.lengths(batch, cu_seqlens, cu_seqlens_k, cu_seqlens_host, cu_seqlens_k_host, rows)
    table = a.table(batch, "block_table", block_table, p.max_pages_per_seq)
    with on_stream(stream):
        if out is None:
            out = torch.empty_like(q)
        if lse is None and want_lse:
            lse = torch.empty((rows, heads), dtype=torch.float32, device=q.device)
        if workspace is None:
            workspace = alloc_cache_workspace(p, q.device)
    op, lp = a("out", out, _ONE_BF16, size), a("lse", lse, _ONE_F32, rows * heads, optional=True)
    if op < qp + 2 * size and qp < op + 2 * size:
        raise ValueError("out must not overlap q")
    if lp is not None:
        end = lp + 4 * rows * heads
        if (lp < qp + 2 * size and qp < end) or (lp < op + 2 * size and op < end):
            raise ValueError("lse must not overlap q or out")
    ws = a("workspace", workspace, _BYTES)
    a.call("fp2_cache_attend", stream, ctypes.byref(p), qp, *lens, ctypes.byref(c), table, op, lp, ws,
           workspace.numel())
    return out, lse


def cache_weights(p: CacheParams, q, lse, cache: KVCache, cu_seqlens, cu_seqlens_k, block_table, *,
                  weights=None, weights_in=None, workspace=None, cu_seqlens_host=None,
                  cu_seqlens_k_host=None, stream=None):
    """fp2_cache_weights: weights = weights_in (zeros if None) plus what each cached token
    received of these queries, fp32 [batch, num_kv_heads, max_kv_len or more]. To add in
    place give the same tensor as both."""
    a, batch = _Args(), p.batch
    row = p.num_q_heads * p.head_dim
    qp = a("q", q, _ONE_BF16, 0, row)
    size = q.numel()
    lp = a("lse", lse, _ONE_F32, size // p.head_dim, optional=True)
    c = a.cache(p, cache, need_v=False)
    lens = a.lengths(batch, cu_seqlens, cu_seqlens_k, cu_seqlens_host, cu_seqlens_k_host, size // row)
    table = a.table(batch, "block_table", block_table, p.max_pages_per_seq)
    wi = a.weights(p, "weights_in", weights_in, optional=True)
    with on_stream(stream):
        if weights is None:
            shape = (p.batch, p.num_kv_heads, p.max_kv_len if weights_in is None else weights_in.shape[2])
            weights = torch.empty(shape, dtype=torch.float32, device=q.device)
        if workspace is None:
            workspace = alloc_cache_workspace(p, q.device)
    w = a.weights(p, "weights", weights)
    if weights_in is not None and weights_in.shape[2] != weights.shape[2]:
        raise ValueError("weights and weights_in differ in their last size")
    ws = a("workspace", workspace, _BYTES)
    a.call("fp2_cache_weights", stream, ctypes.byref(p), qp, lp, *lens, ctypes.byref(c), table, wi, w,
           weights.shape[2], ws, workspace.numel())
    if (p.batch == 0 or p.max_kv_len == 0) and weights is not weights_in:     # a call without tokens
        with on_stream(stream):
            if weights_in is None:
                weights[:batch].zero_()
            else:
                weights[:batch].copy_(weights_in[:batch])
    return weights


def cache_evict(p: CacheParams, cache: KVCache, weights, cu_seqlens_k, block_table, target_table, *,
                budget: int, recent_tokens: int = 0, kept=None, cu_seqlens_k_out=None,
                weights_out=None, cu_seqlens_k_host=None, stream=None):
    """fp2_cache_evict: the `budget` tokens of each sequence and KV head that stay go to the
    pages of target_table (int32 [batch, pages], other pages than block_table's). Returns
    (kept int32 [batch, num_kv_heads, budget], the new cu_seqlens_k, the weights that stay)."""
    a, batch = _Args(), p.batch
    c = a.cache(p, cache)
    _, _, cuk, cuk_host = a.lengths(batch, None, cu_seqlens_k, None, cu_seqlens_k_host)
    table = a.table(batch, "block_table", block_table, p.max_pages_per_seq)
    pages = target_table.shape[-1] if isinstance(target_table, torch.Tensor) and target_table.dim() else -1
    target = a.table(batch, "target_table", target_table, pages)
    w = a.weights(p, "weights", weights)
    heads, stride = p.num_kv_heads, weights.shape[2]
    with on_stream(stream):
        if kept is None:
            kept = cache.k.new_empty((batch, heads, max(1, budget)), dtype=torch.int32)
        if cu_seqlens_k_out is None:
            cu_seqlens_k_out = cache.k.new_empty(batch + 1, dtype=torch.int32)
        if weights_out is None:
            weights_out = weights.new_empty((batch, heads, stride))
    wo = a.weights(p, "weights_out", weights_out)
    if weights_out.shape[2] != stride:
        raise ValueError("weights and weights_out differ in their last size")
    kp = a("kept", kept, _ONE_I32, batch * heads * budget)
    if kept.dim() == 3 and tuple(kept.shape[1:]) != (heads, max(1, budget)):     # rows lie `budget` apart
        raise ValueError("kept must be int32 [>= batch, %d, %d], got %s" % (heads, budget, tuple(kept.shape)))
    co = a("cu_seqlens_k_out", cu_seqlens_k_out, _ONE_I32, batch + 1)
    a.call("fp2_cache_evict", stream, ctypes.byref(p), ctypes.byref(c), cuk, cuk_host, table, target, pages,
           int(budget), int(recent_tokens), w, wo, stride, kp, co)
    if p.batch == 0 or p.max_kv_len == 0:                                      # a call without tokens
        with on_stream(stream):
            kept.view(-1)[:batch * heads * budget].fill_(-1)
            cu_seqlens_k_out.view(-1)[:batch + 1].zero_()
            weights_out[:batch].zero_()
    return kept, cu_seqlens_k_out, weights_out

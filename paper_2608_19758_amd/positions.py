"""Positions of queries and keys: rotary turns, appending with them, and cached tokens
read back or moved to other positions (argument marshalling over ``fp2_rotary``,
``fp2_cache_append_rotary``, ``fp2_cache_read`` and ``fp2_cache_move`` of
``include/fp2.h``, which states their semantics and layouts).

``make_rotary`` builds, once for a model, what the calls take: the frequencies,
scaled for long contexts where wanted, as fractions of a turn in 64-bit fixed
point on the device.
"""
from __future__ import annotations

import ctypes
import dataclasses
import math

import numpy as np
import torch

from . import _F32, BF16, FP8_E4M3, HEAD_DIM
from .cache import _CODES, _ONE_BF16, _ONE_I32, CacheParams, KVCache, _Args, on_stream

_ONE_I64 = (torch.int64,)


class _RotaryArgs(ctypes.Structure):
    """Mirror of fp2_rotary_t."""
    _fields_ = [("turns", ctypes.c_void_p), ("dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class _RotaryRows(ctypes.Structure):
    """Mirror of fp2_rotary_rows_t."""
    _fields_ = [("x", ctypes.c_void_p), ("x_stride", ctypes.c_int64), ("out", ctypes.c_void_p),
                ("out_stride", ctypes.c_int64), ("heads", ctypes.c_int32), ("out_dtype", ctypes.c_int32),
                ("out_scale", ctypes.c_void_p)]


@dataclasses.dataclass(frozen=True, eq=False)
class Rotary:
    """fp2_rotary_t: turns int64 [dim / 2] on the device (the bits of f / (2 pi) * 2^64), pairs (2i, 2i + 1)
    if interleaved, else (i, i + dim / 2); scale multiplies both parts. Its tensor is checked here, once."""
    turns: torch.Tensor
    dim: int
    interleaved: bool = False
    scale: float = 1.0

    def __post_init__(self):
        if not isinstance(self.dim, int) or not 2 <= self.dim <= HEAD_DIM or self.dim % 2:
            raise ValueError("dim must be even and in [2, %d], got %r" % (HEAD_DIM, self.dim))
        a = _Args()
        at = a("turns", self.turns, _ONE_I64, self.dim // 2)
        object.__setattr__(self, "_args", _RotaryArgs(at, self.dim, bool(self.interleaved), self.scale))
        object.__setattr__(self, "_dev", self.turns.get_device())

    def __reduce__(self):     # a copy has a tensor of its own, and its address
        return Rotary, (self.turns, self.dim, self.interleaved, self.scale)


def rotary_frequencies(dim: int, base: float = 10000.0, *, scaling: str = "none", factor: float = 1.0,
                       original_len: int = 0, low: float = 1.0, high=None):
    """(radians a position of each of the dim / 2 pairs in 64 bits, the factor of both parts).
    base^(-2i/dim), and for contexts `factor` times as long as the `original_len` that a model
    was trained on:

    "linear"  all divided by factor;
    "base"    base times factor^(dim / (dim - 2)): the slowest pair as with "linear", the fastest as it is;
    "bands"   pairs of at most `low` turns in original_len divided by factor, of at least `high` (4) as they
              are, between them in proportion to the turns;
    "ramp"    the same between `low` and `high` (32) turns in proportion to the index of the pair, of which the
              bounds are rounded outwards; both parts times 1 + ln(factor) / 10."""
    if isinstance(dim, bool) or not isinstance(dim, int) or not 2 <= dim <= HEAD_DIM or dim % 2:
        raise ValueError("dim must be even and in [2, %d], got %r" % (HEAD_DIM, dim))
    if not (math.isfinite(base) and base > 1.0):
        raise ValueError("base must be finite and above 1, got %r" % (base,))
    if not (math.isfinite(factor) and factor >= 1.0):
        raise ValueError("factor must be finite and at least 1, got %r" % (factor,))
    if scaling not in ("none", "linear", "base", "bands", "ramp"):
        raise ValueError("scaling %r is none of none, linear, base, bands, ramp" % (scaling,))
    if scaling == "none" and factor != 1.0:
        raise ValueError("a factor of %r without scaling" % (factor,))
    if scaling == "base":
        if dim == 2:
            raise ValueError("scaling by the base needs more than one pair")
        base = base * factor ** (dim / (dim - 2))
    i = np.arange(dim // 2, dtype=np.float64)
    f = base ** (-2.0 * i / dim)
    if scaling == "linear":
        return f / factor, 1.0
    if scaling in ("none", "base"):
        return f, 1.0
    high = (4.0 if scaling == "bands" else 32.0) if high is None else high
    if original_len < 1:
        raise ValueError("scaling %r needs original_len" % scaling)
    if not 0.0 < low < high:
        raise ValueError("low and high must be positive and in order, got %r and %r" % (low, high))
    if scaling == "bands":
        keep = np.clip((original_len * f / (2.0 * math.pi) - low) / (high - low), 0.0, 1.0)
        return f * keep + f / factor * (1.0 - keep), 1.0

    def index(turns):     # of the pair that makes so many turns
        return dim * math.log(original_len / (2.0 * math.pi * turns)) / (2.0 * math.log(base))

    first, last = max(math.floor(index(high)), 0), min(math.ceil(index(low)), dim - 1)
    slow = np.clip((i - first) / max(last - first, 0.001), 0.0, 1.0)
    return f * (1.0 - slow) + f / factor * slow, 1.0 + 0.1 * math.log(factor)


def make_rotary(dim: int = HEAD_DIM, *, base: float = 10000.0, interleaved: bool = False, scaling: str = "none",
                factor: float = 1.0, original_len: int = 0, low: float = 1.0, high=None, scale=None,
                frequencies=None, device="cuda") -> Rotary:
    """A model's rotary positions. The frequencies are those of rotary_frequencies, or `frequencies` (radians
    a position, dim / 2 of them); `scale` replaces the factor of both parts that goes with them."""
    f, amplitude = rotary_frequencies(dim, base, scaling=scaling, factor=factor, original_len=original_len,
                                      low=low, high=high)
    if frequencies is not None:
        if scaling != "none":
            raise ValueError("frequencies are given as they are used: without scaling")
        if isinstance(frequencies, torch.Tensor):
            frequencies = frequencies.detach().double().cpu().numpy()
        f = np.asarray(frequencies, np.float64)
        if f.shape != (dim // 2,) or not np.isfinite(f).all():
            raise ValueError("frequencies must be %d finite numbers" % (dim // 2))
    amplitude = float(amplitude if scale is None else scale)
    if not (math.isfinite(amplitude) and amplitude > 0.0):
        raise ValueError("scale must be positive and finite, got %r" % (scale,))
    turns = [round(math.fmod(x / (2.0 * math.pi), 1.0) * 2.0 ** 64) % 2 ** 64 for x in f.tolist()]
    signed = np.array(turns, np.uint64).view(np.int64)
    return Rotary(torch.from_numpy(signed).to(device), dim, bool(interleaved), amplitude)


def _rotary_args(a: _Args, r: Rotary):
    """fp2_rotary_t of r, by reference."""
    if not isinstance(r, Rotary):
        raise ValueError("rotary must be a Rotary (make_rotary)")
    if r._dev != a.dev or r._dev < 0:
        a.place("rotary.turns", r.turns, r._dev)
    return ctypes.byref(r._args)


_CODE_BYTES = torch.uint8


def _turned_rows(a: _Args, name, x, heads, out, scale, stream):
    """fp2_rotary_rows_t of x, its output (made on `stream` where none is given) and its tokens."""
    at, stride, tokens, wide = a.rows(name, x, heads)
    if out is None:
        if stream is None and scale is None:     # (rows that are dense are contiguous; empty_like is the fastest)
            out = torch.empty_like(x)
        else:
            with on_stream(stream):
                out = torch.empty(x.shape, dtype=x.dtype if scale is None else _CODE_BYTES, device=x.device)
        to, to_stride = out.data_ptr(), wide * HEAD_DIM
    else:
        to, to_stride, there, _ = a.rows(name + "'s output", out, wide, _ONE_BF16 if scale is None else _CODES)
        if there < tokens:
            raise ValueError("%s has %d tokens, its output %d" % (name, tokens, there))
        if tokens <= 1:     # strides of a single row do not count: its output's may be any, in place the same
            to_stride = stride
    if scale is None:
        return _RotaryRows(at, stride, to, to_stride, wide, BF16, None), out, tokens
    return _RotaryRows(at, stride, to, to_stride, wide, FP8_E4M3, a(name + "_scale", scale, _F32, wide)), out, tokens


def _meet(a, b, tokens):
    """Whether rows (address, stride and width in bytes) that are written meet others: those of one stride may
    lie between each other's (parts of one matrix)."""
    (x, xs, xw), (y, ys, yw) = a, b
    if tokens == 0 or x >= y + (tokens - 1) * ys + yw or y >= x + (tokens - 1) * xs + xw:
        return False
    off = (y - x) % xs if xs == ys and xs > 0 else 0
    return off < xw or off + yw > xs


def _share(x, n, y, m):
    """Whether n bytes at x share memory with m bytes at y."""
    return x < y + m and y < x + n


def rotary(r: Rotary, q, positions, k=None, *, out=None, k_out=None, q_scale=None, inverse: bool = False, stream=None):
    """fp2_rotary: q (and k) bf16 [tokens, heads, 128] turned by positions int32 [tokens]. Rows may be parts of a
    wider matrix; out and k_out may be q and k themselves. With q_scale (fp32 [heads]) the queries come as e4m3
    codes of q / q_scale. inverse takes a turn back. Returns out, or (out, k_out) if k is given."""
    a = _Args()
    rows, out, tokens = _turned_rows(a, "q", q, None, out, q_scale, stream)
    krows = None
    if k is not None:
        krows, k_out, there = _turned_rows(a, "k", k, None, k_out, None, stream)
        if there != tokens:
            raise ValueError("q has %d tokens, k %d" % (tokens, there))
        krows = ctypes.byref(krows)
    pos = a("positions", positions, _ONE_I32, tokens)
    a.call("fp2_rotary", stream, _rotary_args(a, r), tokens, pos, 1 if inverse else 0, ctypes.byref(rows), krows)
    return out if k is None else (out, k_out)


def cache_append_rotary(p: CacheParams, r: Rotary, q, k_new, v_new, cache: KVCache, cu_seqlens, cu_seqlens_k,
                        block_table, *, positions=None, out=None, q_scale=None, cu_seqlens_host=None,
                        cu_seqlens_k_host=None, stream=None):
    """fp2_cache_append_rotary: k_new and v_new bf16 [new tokens, num_kv_heads, 128] into the cache's pages, the
    keys turned by positions (int32 [new tokens]; None: their indexes in the sequence), and q [new tokens,
    num_q_heads, 128] (None: no queries) turned as rotary does it. Returns the queries."""
    a, batch, met = _Args(), p.batch, None
    c = a.cache(p, cache)
    k, ks, tokens, _ = a.rows("k_new", k_new, p.num_kv_heads)
    v, vs, there, _ = a.rows("v_new", v_new, p.num_kv_heads)
    rows = None
    if q is not None:
        given = out is not None
        rows, out, asked = _turned_rows(a, "q", q, p.num_q_heads, out, q_scale, stream)
        if given and cu_seqlens_host is None and asked == tokens == there:   # (with it the call itself looks)
            e, wide = 2 if q_scale is None else 1, p.num_q_heads * HEAD_DIM
            o, x = (rows.out, e * rows.out_stride, e * wide), (rows.x, 2 * rows.x_stride, 2 * wide)
            width = 2 * p.num_kv_heads * HEAD_DIM
            if (o != x and _meet(o, x, tokens)) or _meet(o, (k, 2 * ks, width), tokens) or \
                    _meet(o, (v, 2 * vs, width), tokens):
                raise ValueError("q's output must not overlap k_new, v_new or other rows of q")
            met = o
        rows = ctypes.byref(rows)
        there = there if asked == tokens else asked
    if there != tokens:
        raise ValueError("q, k_new and v_new differ in their tokens")
    lens = a.lengths(batch, cu_seqlens, cu_seqlens_k, cu_seqlens_host, cu_seqlens_k_host, tokens)
    pos = a("positions", positions, _ONE_I32, tokens, optional=True)
    if met and pos is not None and _meet(met, (pos, 4, 4), tokens):
        raise ValueError("q's output must not overlap positions")
    table = a.table(batch, "block_table", block_table, p.max_pages_per_seq)
    args = _rotary_args(a, r)
    if tokens:
        a.call("fp2_cache_append_rotary", stream, ctypes.byref(p), args, rows, k, ks, v, vs, pos, *lens, ctypes.byref(c),
               table)
    return None if q is None else out


def cache_read(p: CacheParams, cache: KVCache, cu_seqlens, cu_seqlens_k, block_table, *, rotary: Rotary = None,
               positions=None, keys: bool = True, values: bool = True, rows=None, k_out=None, v_out=None,
               cu_seqlens_host=None, cu_seqlens_k_host=None, stream=None):
    """fp2_cache_read: the last cu_seqlens tokens of each sequence as bf16 rows [rows, num_kv_heads, 128], the keys'
    turn by positions (int32 [rows]; None: indexes) taken back if rotary is given. How many rows there are is said
    by `rows`, by the outputs or by cu_seqlens_host. Returns (keys or None, values or None)."""
    a, batch = _Args(), p.batch
    if not keys and not values:
        raise ValueError("neither keys nor values")
    c = a.cache(p, cache, need_v=values)
    if rows is None:
        given = k_out if k_out is not None and keys else v_out if values else None
        if isinstance(given, torch.Tensor) and given.dim():
            rows = given.shape[0]
        elif cu_seqlens_host is not None:
            a.host("cu_seqlens_host", cu_seqlens_host, batch)
            rows = int(cu_seqlens_host[batch])
        else:
            raise ValueError("rows, k_out, v_out or cu_seqlens_host must say how many rows there are")
    lens = a.lengths(batch, cu_seqlens, cu_seqlens_k, cu_seqlens_host, cu_seqlens_k_host, rows)
    pos = a("positions", positions, _ONE_I32, rows, optional=True)
    table = a.table(batch, "block_table", block_table, p.max_pages_per_seq)
    args = None if rotary is None else _rotary_args(a, rotary)
    size, ko, vo = rows * p.num_kv_heads * HEAD_DIM, None, None
    if keys and k_out is not None:
        ko = a("k_out", k_out, _ONE_BF16, size)
    if values and v_out is not None:
        vo = a("v_out", v_out, _ONE_BF16, size)
    if cu_seqlens_host is None:     # (with it the call itself looks)
        if ko is not None and vo is not None and _share(ko, 2 * size, vo, 2 * size):
            raise ValueError("k_out must not overlap v_out")
        if pos is not None and any(o is not None and _share(o, 2 * size, pos, 4 * rows) for o in (ko, vo)):
            raise ValueError("k_out and v_out must not overlap positions")
    if (keys and k_out is None) or (values and v_out is None):
        shape = (rows, p.num_kv_heads, HEAD_DIM)
        with on_stream(stream):
            if keys and k_out is None:
                k_out = cache.k.new_empty(shape, dtype=torch.bfloat16)
                ko = k_out.data_ptr()
            if values and v_out is None:
                v_out = cache.k.new_empty(shape, dtype=torch.bfloat16)
                vo = v_out.data_ptr()
    if rows:
        a.call("fp2_cache_read", stream, ctypes.byref(p), args, pos, *lens, ctypes.byref(c), table, ko, vo)
    return k_out if keys else None, v_out if values else None


def cache_move(p: CacheParams, cache: KVCache, cu_seqlens_k, block_table, target_table=None, *, rotary: Rotary = None,
               moves=None, cu_seqlens_k_host=None, stream=None) -> None:
    """fp2_cache_move: the tokens of each sequence to the pages of target_table (int32 [batch, pages]), or in place
    if it is None, the keys turned by moves if rotary is given: int32 [batch], or [batch or 1, num_kv_heads or 1,
    max_kv_len (or more) or 1], in any strides."""
    a, batch = _Args(), p.batch
    c = a.cache(p, cache, need_v=target_table is not None)
    _, _, cuk, cuk_host = a.lengths(batch, None, cu_seqlens_k, None, cu_seqlens_k_host)
    table = a.table(batch, "block_table", block_table, p.max_pages_per_seq)
    pages, target = 0, None
    if target_table is not None:
        pages = target_table.shape[-1] if isinstance(target_table, torch.Tensor) and target_table.dim() else -1
        target = a.table(batch, "target_table", target_table, pages)
    args, by, strides = None, None, (0, 0, 0)
    if (rotary is None) != (moves is None):
        raise ValueError("rotary and moves go together")
    if rotary is not None:
        args = _rotary_args(a, rotary)
        if not isinstance(moves, torch.Tensor) or moves.dtype != torch.int32:
            raise ValueError("moves must be an int32 torch tensor")
        m = moves[:, None, None] if moves.dim() == 1 else moves
        want = (batch, p.num_kv_heads, p.max_kv_len)
        if m.dim() != 3 or any(n != 1 and n < w for n, w in zip(m.shape, want)) or m.shape[1] not in (1, want[1]):
            raise ValueError("moves must be int32 [batch] or [%d or 1, %d or 1, %d or 1], got %s"
                             % (*want, tuple(moves.shape)))
        a.place("moves", m, m.get_device())
        by = m.data_ptr()
        strides = tuple(s if n != 1 else 0 for n, s in zip(m.shape, m.stride()))
    a.call("fp2_cache_move", stream, ctypes.byref(p), args, by, *strides, cuk,
           cuk_host, ctypes.byref(c), table, target, pages)

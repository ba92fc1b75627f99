"""Serving-engine attention backends: the sparse extend (prefill) phase, and the
dense paged cache that decoding goes on from.

The shape a continuous-batching engine needs around fp2_prefill (Sec. 4: the
sparse operator serves every extend of a request, chunked prefill included,
while decode attention stays dense):

- ``BackendConfig``: the engine-level settings, fixed at start-up (head
  counts, page size, the per-forward bounds that size the buffers, the
  selection and correction settings).
- ``PrefillBackend``: one per stream. It owns a workspace and a block-mask
  buffer sized for the largest forward the config admits, allocated once and
  reused by every layer of every forward (the library never allocates).
- ``ForwardMetadata``: built once per forward by ``init_forward_metadata``
  from the extend lengths, the cached-prefix lengths and the page table, and
  shared by all layers: the length arrays are uploaded to the device once.
- ``forward_extend``: one layer's attention over the paged cache, through the
  C ABI. The K/V of the new tokens must already be in the cache.
- Block means across forwards: ``alloc_means_cache`` gives a layer's cache of
  pooled key/value means (one slot per 128-token block of the paged pool,
  about 2/(page * bytes per element) of the KV cache). Passed to
  ``forward_extend``, a forward pools only the blocks that are new or were
  incomplete, and copies the complete blocks of the cached prefix, whose
  means an earlier forward through the same cache wrote (chunked prefill, or
  prefix pages shared between requests).

Cached prefixes may have any length (a prefix-cache hit is page-granular);
``plan_forward`` checks the lengths against the configured bounds before
anything reaches the GPU.

``CacheConfig`` and ``CacheBackend`` are the same shape around the fp2_cache_*
operators: a forward of any mix of prompts, chunks and single tokens appends
the new keys and values to each layer's cache, attends over it and, where the
engine wants to shorten sequences later, adds up what every cached token
received; ``evict`` then keeps the heaviest ``budget`` tokens of each sequence
and KV head in new pages. One kernel serves a forward, by its longest extend: single
tokens beside a long chunk are faster in a forward of their own. A cache of codes with
a scale per head is what ``PrefillBackend`` reads, so a prompt may be extended sparsely
and decoded here.

With ``rotary`` (``make_rotary``) a forward takes queries and keys as the projection gives
them and turns them on the way in; an eviction with it turns the keys that stay to their
new indexes. ``read`` gives cached tokens back as bf16 rows (whole sequences too, however
many chunks they came in: ``init_read_metadata``), ``move`` takes them to other
pages or positions, and ``forward_cross`` attends to the states of an encoder (written with
``append``), or to a prefix that requests share, whatever their length; more queries than
``max_extend_len``, or than there are states, are allowed for by ``max_query_len``.
"""
from __future__ import annotations

import ctypes
import dataclasses
from typing import List, Optional, Sequence

import numpy as np

import paper_2608_19758_amd as fp2

BLOCK = fp2.BLOCK


@dataclasses.dataclass(frozen=True)
class BackendConfig:
    num_q_heads: int
    num_kv_heads: int
    page_size: int                 # tokens per KV page (> 0: paged pool)
    max_batch: int                 # sequences per forward
    max_extend_len: int            # new tokens of one sequence in one forward
    max_kv_len: int                # cached + new tokens of one sequence
    dtype: str = "bf16"            # "bf16" | "fp8"
    alpha: float = 0.1
    sink_blocks: int = 2
    window_blocks: int = 4
    recent_blocks: int = 0
    mean_correction: bool = True
    kv_splits: int = 0             # 0: cost-balanced plan on the device
    softmax_scale: float = 0.0     # <= 0: 1/sqrt(128)
    query_tile_rows: int = 0       # 0: query blocks of 128 positions; 128: 128-row tiles
    score_splits: int = 0          # 0: rows of few units split over workgroups; 1: never

    @property
    def max_pages_per_seq(self) -> int:
        return (self.max_kv_len + self.page_size - 1) // self.page_size

    def params(self, batch: int, max_extend: int, max_kv: int) -> "fp2.Params":
        return fp2.make_params(
            batch=batch, num_q_heads=self.num_q_heads, num_kv_heads=self.num_kv_heads,
            max_seq_len=max_extend, page_size=self.page_size,
            max_pages_per_seq=self.max_pages_per_seq, alpha=self.alpha,
            sink_blocks=self.sink_blocks, window_blocks=self.window_blocks,
            recent_blocks=self.recent_blocks, mean_correction=int(self.mean_correction),
            softmax_scale=self.softmax_scale, dtype=self.dtype, max_kv_len=max_kv,
            kv_splits=self.kv_splits, query_tile_rows=self.query_tile_rows,
            score_splits=self.score_splits)

    def worst_case_params(self) -> "fp2.Params":
        return self.params(self.max_batch, self.max_extend_len, self.max_kv_len)


@dataclasses.dataclass
class ForwardPlan:
    """Host part of a forward's metadata (no device memory)."""
    params: "fp2.Params"
    cu_q: np.ndarray               # int32 [batch + 1], query (new-token) rows
    cu_k: np.ndarray               # int32 [batch + 1], KV tokens (prefix + new)
    total_tokens: int


def plan_forward(cfg: BackendConfig, extend_lens: Sequence[int],
                 prefix_lens: Optional[Sequence[int]] = None) -> ForwardPlan:
    """Validate one forward against the config and build its parameters."""
    ext = [int(x) for x in extend_lens]
    pre = [0] * len(ext) if prefix_lens is None else [int(x) for x in prefix_lens]
    if len(pre) != len(ext):
        raise ValueError("extend_lens and prefix_lens differ in length")
    if len(ext) > cfg.max_batch:
        raise ValueError("batch %d > max_batch %d" % (len(ext), cfg.max_batch))
    for b, (e, p) in enumerate(zip(ext, pre)):
        if e < 0 or p < 0:
            raise ValueError("sequence %d: negative length" % b)
        if e > cfg.max_extend_len:
            raise ValueError("sequence %d: extend of %d > max_extend_len %d"
                             % (b, e, cfg.max_extend_len))
        if p + e > cfg.max_kv_len:
            raise ValueError("sequence %d: %d cached + %d new > max_kv_len %d"
                             % (b, p, e, cfg.max_kv_len))
    cu_q = np.zeros(len(ext) + 1, np.int32)
    cu_k = np.zeros(len(ext) + 1, np.int32)
    cu_q[1:] = np.cumsum(ext)
    cu_k[1:] = np.cumsum([p + e for p, e in zip(pre, ext)])
    max_e = max(ext, default=0)
    max_k = max((p + e for p, e in zip(pre, ext)), default=0)
    params = cfg.params(len(ext), max_e, max(max_k, max_e))
    return ForwardPlan(params=params, cu_q=cu_q, cu_k=cu_k, total_tokens=int(cu_q[-1]))


@dataclasses.dataclass
class ForwardMetadata:
    plan: ForwardPlan
    cu_q: object                   # device int32 [batch + 1]
    cu_k: object                   # device int32 [batch + 1]
    block_table: object            # device int32 [batch, max_pages_per_seq], dense
    pooled_blocks: object          # device int32 [batch]: cached complete prefix blocks

    @property
    def params(self):
        return self.plan.params


def _dense_table(block_table, n: int, w: int):
    """The first n rows of an engine's page table as a dense one of w pages."""
    import torch
    if not (isinstance(block_table, torch.Tensor) and block_table.is_cuda
            and block_table.dtype == torch.int32 and block_table.dim() == 2):
        raise ValueError("block_table must be a CUDA int32 tensor [batch, pages]")
    if block_table.shape[1] < w or block_table.shape[0] < n:
        raise ValueError("block_table is %s, the forward needs [>= %d, >= %d]"
                         % (tuple(block_table.shape), n, w))
    # the library reads row b at b * max_pages_per_seq: hand it a dense
    # table of exactly that width (a copy when the caller's is wider or strided)
    if block_table.shape[1] != w or not block_table.is_contiguous():
        block_table = block_table[:n, :w].contiguous()
    return block_table


class PrefillBackend:
    """Extend-phase attention of one stream (see the module docstring)."""

    def __init__(self, cfg: BackendConfig, device="cuda", stream=None):
        import torch
        self.cfg = cfg
        self.device = torch.device(device)
        self.stream = stream
        worst = cfg.worst_case_params()
        need = fp2.workspace_bytes(worst)
        if need == 0 and cfg.max_batch > 0:
            raise ValueError("configuration rejected by the library: " + fp2.last_error())
        self.workspace = torch.empty(max(1, need), dtype=torch.uint8, device=self.device)
        nq, nk = fp2.num_blocks(worst), fp2.num_key_blocks(worst)
        self._mask = torch.empty(max(1, cfg.max_batch * cfg.num_kv_heads * nq * nk),
                                 dtype=torch.uint8, device=self.device)

    def init_forward_metadata(self, extend_lens: Sequence[int], prefix_lens: Optional[Sequence[int]],
                              block_table, cached_prefix_lens: Optional[Sequence[int]] = None
                              ) -> ForwardMetadata:
        """cached_prefix_lens[b]: leading tokens of sequence b whose block means an
        earlier forward wrote to the means caches used with this metadata (None:
        none); only its complete blocks are taken from the cache."""
        import torch
        plan = plan_forward(self.cfg, extend_lens, prefix_lens)
        if fp2.workspace_bytes(plan.params) > self.workspace.numel():
            raise RuntimeError("forward needs more workspace than the configured worst case")
        n = len(plan.cu_q) - 1
        cached = [0] * n if cached_prefix_lens is None else [int(x) for x in cached_prefix_lens]
        if len(cached) != n:
            raise ValueError("cached_prefix_lens and extend_lens differ in length")
        kv = np.diff(plan.cu_k)
        for b, c in enumerate(cached):
            if c < 0 or c > kv[b]:
                raise ValueError("sequence %d: %d cached tokens outside [0, %d]" % (b, c, kv[b]))
        pooled = np.array([c // BLOCK for c in cached], np.int32)
        host = np.concatenate([plan.cu_q, plan.cu_k, pooled]).astype(np.int32)
        dev = torch.from_numpy(host).to(self.device)
        block_table = _dense_table(block_table, n, self.cfg.max_pages_per_seq)
        return ForwardMetadata(plan=plan, cu_q=dev[:n + 1], cu_k=dev[n + 1:2 * n + 2],
                               block_table=block_table, pooled_blocks=dev[2 * n + 2:])

    def alloc_means_cache(self, num_pages: int):
        """One layer's block-means cache for a pool of num_pages pages:
        (khat, vbar) bf16 [slots, num_kv_heads, 128]."""
        return fp2.alloc_means_cache(self.cfg.worst_case_params(), num_pages, self.device)

    def block_mask(self, meta: ForwardMetadata):
        """The selection mask written by the last forward_extend, as a view
        [batch, num_kv_heads, nbq, nbk] of the backend's buffer."""
        p = meta.params
        shape = (p.batch, p.num_kv_heads, max(1, fp2.num_blocks(p)), max(1, fp2.num_key_blocks(p)))
        n = int(np.prod(shape))
        return self._mask[:n].view(shape)

    def forward_extend(self, q, k_cache, v_cache, meta: ForwardMetadata, *, q_scale=None,
                       k_scale=None, v_scale=None, out=None, lse=None, want_lse=False,
                       means_cache=None):
        """One layer: q [total_new_tokens, Hq, 128] against the paged cache.
        means_cache: this layer's (khat, vbar) from alloc_means_cache, or None.
        Returns (out, lse or None)."""
        import torch
        p = meta.params
        if q.shape[0] != meta.plan.total_tokens:
            raise ValueError("q has %d rows, the forward has %d new tokens"
                             % (q.shape[0], meta.plan.total_tokens))
        if out is None:
            out = torch.empty((q.shape[0], p.num_q_heads, p.head_dim), dtype=torch.bfloat16,
                              device=q.device)
        if lse is None and want_lse:
            lse = torch.empty((q.shape[0], p.num_q_heads), dtype=torch.float32, device=q.device)
        fp2.prefill(p, q, k_cache, v_cache, meta.cu_q, meta.block_table,
                    cu_seqlens_host=meta.plan.cu_q, cu_seqlens_k=meta.cu_k,
                    cu_seqlens_k_host=meta.plan.cu_k, q_scale=q_scale, k_scale=k_scale,
                    v_scale=v_scale, out=out, lse=lse, block_mask=self.block_mask(meta),
                    workspace=self.workspace, stream=self.stream,
                    means_cache=None if means_cache is None
                    else (means_cache[0], means_cache[1], meta.pooled_blocks))
        return out, lse

    def forward_decode(self, *args, **kwargs):
        raise NotImplementedError("decode attention stays dense; this backend serves extends")


@dataclasses.dataclass(frozen=True)
class CacheConfig:
    num_q_heads: int
    num_kv_heads: int
    page_size: int                 # tokens per KV page
    max_batch: int                 # sequences per forward
    max_extend_len: int            # new tokens of one sequence in one forward
    max_kv_len: int                # cached + new tokens of one sequence
    dtype: str = "bf16"            # of the cache: "bf16" | "fp8"
    scale_tokens: int = 0          # fp8: tokens per power-of-two scale, 0: a scale per head
    sink_tokens: int = 0           # first tokens that stay visible and are never evicted
    window_tokens: int = 0         # 0: every earlier token is visible
    softmax_scale: float = 0.0     # <= 0: 1/sqrt(128)
    max_query_len: int = 0         # queries of one sequence in a cross attention, whatever max_kv_len; 0: max_extend_len

    @property
    def max_pages_per_seq(self) -> int:
        return (self.max_kv_len + self.page_size - 1) // self.page_size

    def params(self, batch: int, max_extend: int, max_kv: int) -> "fp2.CacheParams":
        return fp2.make_cache_params(
            batch=batch, num_q_heads=self.num_q_heads, num_kv_heads=self.num_kv_heads,
            max_seq_len=max_extend, max_kv_len=max_kv, page_size=self.page_size,
            max_pages_per_seq=self.max_pages_per_seq, dtype=self.dtype,
            scale_tokens=self.scale_tokens, sink_tokens=self.sink_tokens,
            window_tokens=self.window_tokens, softmax_scale=self.softmax_scale)

    def worst_case_params(self) -> "fp2.CacheParams":
        return self.params(self.max_batch, self.max_extend_len, self.max_kv_len)


def plan_cross(cfg: CacheConfig, query_lens: Sequence[int], state_lens: Sequence[int]) -> ForwardPlan:
    """Validate one cross attention against the config and build its parameters."""
    new, kv = [int(x) for x in query_lens], [int(x) for x in state_lens]
    if len(new) != len(kv):
        raise ValueError("query_lens and state_lens differ in length")
    if len(new) > cfg.max_batch:
        raise ValueError("batch %d > max_batch %d" % (len(new), cfg.max_batch))
    most, name = (cfg.max_query_len, "max_query_len") if cfg.max_query_len else (cfg.max_extend_len, "max_extend_len")
    for b, (n, t) in enumerate(zip(new, kv)):
        if not 0 <= n <= most:
            raise ValueError("sequence %d: %d queries outside [0, %s = %d]" % (b, n, name, most))
        if not 0 <= t <= cfg.max_kv_len:
            raise ValueError("sequence %d: %d states outside [0, max_kv_len = %d]" % (b, t, cfg.max_kv_len))
    params = dataclasses.replace(cfg, sink_tokens=0, window_tokens=0).params(len(new), max(new, default=0),
                                                                             max(kv, default=0))
    cu = [np.concatenate([[0], np.cumsum(x)]).astype(np.int32) for x in (new, kv)]
    return ForwardPlan(params=params, cu_q=cu[0], cu_k=cu[1], total_tokens=int(cu[0][-1]))


def plan_read(cfg: CacheConfig, read_lens: Sequence[int],
              prefix_lens: Optional[Sequence[int]] = None) -> ForwardPlan:
    """Validate one reading back: the last read_lens tokens of sequences, each behind prefix_lens others. Unlike
    a forward's new tokens they are bounded by max_kv_len alone."""
    lens = [int(x) for x in read_lens]
    for b, n in enumerate(lens):
        if n > cfg.max_kv_len:
            raise ValueError("sequence %d: %d tokens > max_kv_len %d" % (b, n, cfg.max_kv_len))
    return plan_forward(dataclasses.replace(cfg, max_extend_len=cfg.max_kv_len), lens, prefix_lens)


@dataclasses.dataclass
class CacheMetadata:
    plan: ForwardPlan
    lengths: object                # device int32: cu_q and cu_k side by side
    block_table: object            # device int32 [batch or more, max_pages_per_seq], dense
    replayed: bool = False         # lengths and table are the metadata's own, and may be updated
    rows: Optional[int] = None     # of the tensors of the forwards captured with it, the fewest
    cross: bool = False            # of a cross attention
    read: bool = False             # of tokens to read back, which no forward appends

    @property
    def params(self):
        return self.plan.params

    @property
    def cu_q(self):
        return self.lengths[:len(self.plan.cu_q)]

    @property
    def cu_k(self):
        return self.lengths[len(self.plan.cu_q):]


class CacheBackend:
    """Attention of one stream over paged caches, decoding included (see the
    module docstring). It owns one workspace that fits every forward; calls
    that overlap, and graphs that may, need backends of their own. Work runs
    on `stream` (None: the current one of the device); the caller orders its
    own tensors with it."""

    def __init__(self, cfg: CacheConfig, device="cuda", stream=None):
        import torch
        self.cfg = cfg
        self.device = torch.device(device)
        self.stream = stream
        if not 0 <= cfg.max_extend_len <= cfg.max_kv_len:
            raise ValueError("max_extend_len %d outside [0, max_kv_len = %d]"
                             % (cfg.max_extend_len, cfg.max_kv_len))
        # a call without new tokens checks its parameters and has nothing to do
        idle = cfg.params(cfg.max_batch, 0, cfg.max_kv_len)
        if fp2.lib().fp2_cache_append(ctypes.byref(idle), *[None] * 9):
            raise ValueError("configuration rejected by the library: " + fp2.last_error())
        # nor has one without sequences, which checks the bound of the queries
        none = dataclasses.replace(cfg, sink_tokens=0, window_tokens=0).params(0, cfg.max_query_len, cfg.max_kv_len)
        if fp2.lib().fp2_cache_cross(ctypes.byref(none), *[None] * 10, 0, None):
            raise ValueError("max_query_len rejected by the library: " + fp2.last_error())
        with fp2.cache.on_stream(stream):
            self.workspace = torch.empty(fp2.CACHE_WORKSPACE_MAX, dtype=torch.uint8, device=self.device)

    def alloc_cache(self, num_pages: int, k_scale=None, v_scale=None) -> "fp2.KVCache":
        """One layer's empty cache of num_pages pages."""
        with fp2.cache.on_stream(self.stream):
            return fp2.alloc_cache(self.cfg.worst_case_params(), num_pages, self.device, k_scale, v_scale)

    def alloc_weights(self):
        """One layer's weights of empty sequences: zeros [max_batch, num_kv_heads, max_kv_len]."""
        import torch
        c = self.cfg
        with fp2.cache.on_stream(self.stream):
            return torch.zeros((c.max_batch, c.num_kv_heads, c.max_kv_len), device=self.device)

    def init_forward_metadata(self, extend_lens: Sequence[int], prefix_lens: Optional[Sequence[int]],
                              block_table, replayed: bool = False) -> CacheMetadata:
        """Once per forward, for all layers. replayed: the forward is captured in a graph
        and replayed after update_forward_metadata; its bounds are then the longest of
        these extends and the config's max_kv_len instead of these lengths'."""
        return self._metadata(plan_forward(self.cfg, extend_lens, prefix_lens), block_table, replayed)

    def init_cross_metadata(self, query_lens: Sequence[int], state_lens: Sequence[int], block_table,
                            replayed: bool = False) -> CacheMetadata:
        """The same for cross attention: queries (up to max_query_len), and cached states, of each sequence."""
        return self._metadata(plan_cross(self.cfg, query_lens, state_lens), block_table, replayed, cross=True)

    def init_read_metadata(self, read_lens: Sequence[int], prefix_lens: Optional[Sequence[int]], block_table,
                           replayed: bool = False) -> CacheMetadata:
        """The same for reading back (or moving): the last read_lens tokens of each sequence, up to max_kv_len;
        without prefix_lens whole sequences."""
        return self._metadata(plan_read(self.cfg, read_lens, prefix_lens), block_table, replayed, read=True)

    def _metadata(self, plan, block_table, replayed, cross=False, read=False):
        import torch
        if replayed:
            kv, new = self.cfg.max_kv_len, plan.params.max_seq_len
            plan.params = self.cfg.params(plan.params.batch, new, kv)
            if cross:
                plan.params.sink_tokens = plan.params.window_tokens = 0
        with fp2.cache.on_stream(self.stream):
            lengths = torch.from_numpy(np.concatenate([plan.cu_q, plan.cu_k])).to(self.device)
            table = _dense_table(block_table, len(plan.cu_q) - 1, self.cfg.max_pages_per_seq)
            if replayed:
                table = table.clone()
        return CacheMetadata(plan=plan, lengths=lengths, block_table=table, replayed=replayed, cross=cross,
                             read=read)

    def update_forward_metadata(self, meta: CacheMetadata, extend_lens: Sequence[int],
                                prefix_lens: Optional[Sequence[int]], block_table) -> None:
        """Other lengths and pages for a captured forward (metadata made with
        replayed=True): as many sequences, extends within the first one's bound, and no more new
        tokens in all than the captured tensors have rows. For a cross attention: its queries and
        states; for a read: its tokens and those before them."""
        import torch
        plan = (plan_cross if meta.cross else plan_read if meta.read else plan_forward)(self.cfg, extend_lens, prefix_lens)
        p = meta.params
        if not meta.replayed:
            raise ValueError("the metadata was not made with replayed=True")
        if plan.params.batch != p.batch or plan.params.max_seq_len > p.max_seq_len:
            raise ValueError("%d sequences with extends up to %d do not fit a forward of %d with up to %d"
                             % (plan.params.batch, plan.params.max_seq_len, p.batch, p.max_seq_len))
        if meta.rows is not None and plan.total_tokens > meta.rows:
            raise ValueError("%d new tokens, the captured forward's tensors have %d rows"
                             % (plan.total_tokens, meta.rows))
        plan.params = p
        with fp2.cache.on_stream(self.stream):
            table = _dense_table(block_table, p.batch, self.cfg.max_pages_per_seq)   # refused before any change
            meta.lengths.copy_(torch.from_numpy(np.concatenate([plan.cu_q, plan.cu_k])))
            meta.block_table[:p.batch].copy_(table[:p.batch])
        meta.plan = plan

    def _check_rows(self, meta: CacheMetadata, *named) -> None:
        """Tensors (name, tensor or None) against the forward's tokens; those of a captured forward bound
        the later ones."""
        given = [(n, t) for n, t in named if t is not None]
        for name, t in given:
            if t.shape[0] < meta.plan.total_tokens:
                raise ValueError("%s has %d rows, the forward has %d new tokens"
                                 % (name, t.shape[0], meta.plan.total_tokens))
        if meta.replayed:
            import torch
            with fp2.cache.on_stream(self.stream):
                captured = torch.cuda.is_current_stream_capturing()
            if captured:     # later lengths are held to these tensors
                rows = [t.shape[0] for _, t in given] + [meta.rows] * (meta.rows is not None)
                meta.rows = min(rows)

    def _lengths(self, meta: CacheMetadata, cross: bool = False, appends: bool = False):
        if meta.cross != cross or (meta.read and appends):
            raise ValueError("metadata of a %s" % ("cross attention" if meta.cross else "read" if meta.read else "forward"))
        return ((meta.cu_q, meta.cu_k, meta.block_table),
                dict(cu_seqlens_host=meta.plan.cu_q, cu_seqlens_k_host=meta.plan.cu_k, stream=self.stream))

    def forward(self, q, k_new, v_new, cache: "fp2.KVCache", meta: CacheMetadata, *, out=None, lse=None,
                want_lse=False, weights=None, rotary: Optional["fp2.Rotary"] = None, positions=None):
        """One layer: k_new and v_new bf16 [new tokens, Hkv, 128] go into the cache, q
        [new tokens, Hq, 128] attends over it. With rotary both come as the projection gives them (parts of
        one matrix will do) and are turned by positions (device int32 [new tokens]; None: a token's index in
        its sequence). weights (as from alloc_weights): what the cached tokens received of these queries is
        added to it, row b for sequence b. Returns (out, lse or None)."""
        lens, host = self._lengths(meta, appends=True)
        if rotary is None and positions is not None:
            raise ValueError("positions without rotary")
        self._check_rows(meta, ("q", q), ("k_new", k_new), ("v_new", v_new), ("positions", positions))
        p = meta.params
        if rotary is None:
            fp2.cache_append(p, k_new, v_new, cache, *lens, **host)
        else:
            q = fp2.cache_append_rotary(p, rotary, q, k_new, v_new, cache, *lens, positions=positions, **host)
        out, lse = fp2.cache_attend(p, q, cache, *lens, out=out, lse=lse,
                                    want_lse=want_lse or weights is not None,
                                    workspace=self.workspace, **host)
        if weights is not None:
            fp2.cache_weights(p, q, lse, cache, *lens, weights=weights, weights_in=weights,
                              workspace=self.workspace, **host)
        return out, lse

    def append(self, k_new, v_new, cache: "fp2.KVCache", meta: CacheMetadata) -> None:
        """One layer: keys and values into the cache without queries (an encoder's states)."""
        lens, host = self._lengths(meta, appends=True)
        self._check_rows(meta, ("k_new", k_new), ("v_new", v_new))
        fp2.cache_append(meta.params, k_new, v_new, cache, *lens, **host)

    def forward_cross(self, q, cache: "fp2.KVCache", meta: CacheMetadata, *, out=None, lse=None, want_lse=False):
        """One layer of cross attention (metadata of init_cross_metadata): every query of q [queries, Hq, 128]
        over all states of its sequence; zeros where there are none. Returns (out, lse or None)."""
        lens, host = self._lengths(meta, cross=True)
        self._check_rows(meta, ("q", q))
        return fp2.cache_cross(meta.params, q, cache, *lens, out=out, lse=lse, want_lse=want_lse,
                               workspace=self.workspace, **host)

    def read(self, cache: "fp2.KVCache", meta: CacheMetadata, *, rotary: Optional["fp2.Rotary"] = None, positions=None):
        """The tokens of init_read_metadata (or a forward's new ones) out of one layer's cache, (keys, values) bf16
        [tokens, Hkv, 128]; with rotary the keys' turn by positions (device int32 [tokens]; None: indexes) is
        taken back."""
        lens, host = self._lengths(meta)
        if meta.replayed:     # the rows of a captured read are those of now
            self._check_rows(meta, ("rows", np.empty((meta.plan.total_tokens, 0))))
        return fp2.cache_read(meta.params, cache, *lens, rotary=rotary, positions=positions, **host)

    def move(self, cache: "fp2.KVCache", meta: CacheMetadata, target_table=None, *,
             rotary: Optional["fp2.Rotary"] = None, moves=None) -> None:
        """One layer: the sequences' tokens to the pages of target_table (int32 [batch, pages]; None: in place),
        their keys turned by moves (fp2.cache_move) where rotary is given."""
        lens, host = self._lengths(meta)
        fp2.cache_move(meta.params, cache, *lens[1:], target_table, rotary=rotary, moves=moves,
                       cu_seqlens_k_host=host["cu_seqlens_k_host"], stream=self.stream)

    def evict(self, cache: "fp2.KVCache", weights, meta: CacheMetadata, target_table, *, budget: int,
              recent_tokens: int = 0, rotary: Optional["fp2.Rotary"] = None):
        """One layer, after a forward: the sequences of `meta` are cut to `budget` tokens per
        KV head, in the pages of target_table (int32 [batch, pages]). With rotary the keys that stay, which
        were turned by their indexes, are turned to their new ones (else later forwards need positions that
        go on from the old ones). Returns (the tokens that stay, int32 [batch, Hkv, budget], their weights);
        the sequences' new lengths are evicted_lens(meta, budget)."""
        _, host = self._lengths(meta)
        p = meta.params
        kept, cu_k, w = fp2.cache_evict(p, cache, weights, meta.cu_k, meta.block_table, target_table,
                                        budget=budget, recent_tokens=recent_tokens,
                                        cu_seqlens_k_host=host["cu_seqlens_k_host"], stream=self.stream)
        if rotary is not None and p.batch > 0 and p.max_kv_len > 0:
            import torch
            stay = min(budget, p.max_kv_len)
            short = self.cfg.params(p.batch, 0, stay)
            short.max_pages_per_seq = target_table.shape[1]
            with fp2.cache.on_stream(self.stream):
                moves = torch.arange(budget, dtype=torch.int32, device=kept.device) - kept
            fp2.cache_move(short, cache, cu_k, target_table, rotary=rotary, moves=moves, stream=self.stream)
        return kept, w


def evicted_lens(meta: CacheMetadata, budget: int) -> List[int]:
    """Cached tokens of each sequence after an eviction to `budget`."""
    return [min(int(n), budget) for n in np.diff(meta.plan.cu_k)]

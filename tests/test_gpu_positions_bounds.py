"""Reading back, appending, moving and cross attention on the GPU beyond a forward's bounds, and in
calls large enough that their workgroups take several shares of work each."""
import numpy as np
import pytest
import torch

import paper_2608_19758_amd as fp2
from paper_2608_19758_amd import serving
from tests import cache_ref as ref
from tests import positions_ref as pos_ref
from tests.test_gpu_cache import close, cu_of, dev
from tests.test_gpu_cache_serving import HKV, HQ, PAGE, config, equal, rows, scales, tables
from tests.test_gpu_positions import run_move
from tests.test_gpu_positions_serving import spoil, view

pytestmark = pytest.mark.gpu


# ---- sequences longer than a forward's chunk

@pytest.mark.parametrize("form", ["bf16", "head", 16])
def test_read_of_whole_sequences(form):
    """Sequences that came in several chunks, read back in one call: each key and value against what the cache
    holds, the last tokens of some as well; moved in place by the same metadata."""
    cfg = config(form, max_extend_len=200)
    be = serving.CacheBackend(cfg)
    (table,), pages = tables(cfg, 1, 11)
    g = torch.Generator().manual_seed(11)
    cache = be.alloc_cache(pages, *scales(form))
    r = fp2.make_rotary(128)
    freq = fp2.rotary_frequencies(128)[0]
    lens = [0, 0, 0]
    for ext in ([200, 0, 7], [200, 0, 0], [187, 0, 1]):
        be.forward(*rows(g, sum(ext)), cache, be.init_forward_metadata(ext, lens, table), rotary=r)
        lens = [a + e for a, e in zip(lens, ext)]
    c = view(cfg, lens, cache, table, form)
    for part, pre in ((lens, None), ([450, 0, 3], [137, 0, 5])):
        k, v = be.read(cache, be.init_read_metadata(part, pre, table), rotary=r)
        torch.cuda.synchronize()
        index = [np.arange(n - m, n) for n, m in zip(lens, part)]
        slots = np.concatenate([c.slots(b, i) for b, i in enumerate(index)])
        raw = [np.stack([c.values(n, slots, h) for h in range(HKV)], 1) for n in "kv"]
        want, err = pos_ref.turn(raw[0], np.repeat(np.concatenate(index)[:, None], HKV, 1), freq, False, back=True)
        pos_ref.check_bf16(k, want, err, "k")
        pos_ref.check_bf16(v, raw[1], 0 * raw[1], "v")
    # and turned on, in place, by as many positions as bring each back: bf16 rows are off by two roundings of 2^-8
    # (and the turns' own), which a turn spreads over a pair
    if form == "bf16":
        meta = be.init_read_metadata(lens, None, table)
        for by in (7, -7):
            be.move(cache, meta, rotary=r, moves=torch.full((3,), by, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        was, now = c, view(cfg, lens, cache, table, form)
        for b, n in enumerate(lens):
            for h in range(HKV):
                x, y = (t.values("k", t.slots(b, np.arange(n)), h) for t in (was, now))
                pair = np.abs(x) + np.abs(np.concatenate([x[:, 64:], x[:, :64]], 1))
                assert (np.abs(y - x) <= 2 * 1.02 * 2.0 ** -8 * pair + 1e-6).all()


def test_captured_read_of_whole_sequences():
    """Captured with the most tokens and replayed with fewer, other lengths and pages."""
    cfg = config("bf16", max_extend_len=100)
    be, eager = serving.CacheBackend(cfg), serving.CacheBackend(cfg)
    (table,), pages = tables(cfg, 1, 12)
    g = torch.Generator().manual_seed(12)
    cache = be.alloc_cache(pages)
    cache.k.copy_(torch.randn(cache.k.shape, generator=g).bfloat16())
    cache.v.copy_(torch.randn(cache.v.shape, generator=g).bfloat16())
    r = fp2.make_rotary(64, interleaved=True)
    meta = be.init_read_metadata([900, 300, 0], None, table, replayed=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        k, v = be.read(cache, meta, rotary=r)
    for order, part, pre in (([0, 1, 2], [900, 300, 0], None), ([2, 1, 0], [3, 800, 250], [20, 224, 0]),
                             ([1, 0, 2], [0, 0, 1], [5, 0, 1023]), ([0, 1, 2], [900, 300, 0], None)):
        tab = table[order]
        be.update_forward_metadata(meta, part, pre, tab)
        graph.replay()
        spoil()
        wk, wv = eager.read(cache, eager.init_read_metadata(part, pre, tab), rotary=r)
        torch.cuda.synchronize()
        n = sum(part)
        assert torch.equal(k[:n], wk) and torch.equal(v[:n], wv)
    for part in ([901, 0, 0], [900, 300, 1], [1, 1]):
        with pytest.raises(ValueError):
            be.update_forward_metadata(meta, part, None, table)


@pytest.mark.parametrize("form", ["bf16", "head", 32])
def test_cross_of_more_queries_than_states(form):
    """A cache of short states under queries of many more: eager, and captured and replayed."""
    cfg = config(form, max_extend_len=128, max_kv_len=128, max_query_len=1500)
    be, eager = serving.CacheBackend(cfg), serving.CacheBackend(cfg)
    (table,), pages = tables(cfg, 1, 13)
    g = torch.Generator().manual_seed(13)
    cache = be.alloc_cache(pages, *scales(form))
    states = [77, 0, 128]
    _, k, v = rows(g, sum(states))
    be.append(k, v, cache, be.init_forward_metadata(states, None, table))
    for new in ([1500, 3, 129], [2, 0, 1]):
        q = rows(g, sum(new))[0]
        out, lse = be.forward_cross(q, cache, be.init_cross_metadata(new, states, table), want_lse=True)
        torch.cuda.synchronize()
        o, tol, z, ztol = pos_ref.cross(view(cfg, states, cache, table, form), q.cpu(), new)
        close(out, o, tol, "out")
        close(lse, z, ztol, "lse")
    new = [400, 300, 200]
    meta = be.init_cross_metadata(new, states, table, replayed=True)
    q, out = rows(g, sum(new))[0], torch.zeros((sum(new), HQ, 128), dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        be.forward_cross(q, cache, meta, out=out)
    for order, now in (([0, 1, 2], new), ([2, 0, 1], [400, 200, 300]), ([1, 2, 0], [1, 400, 0]), ([0, 1, 2], new)):
        tab, kv = table[order], [states[i] for i in order]
        be.update_forward_metadata(meta, now, kv, tab)
        graph.replay()
        spoil()
        want, _ = eager.forward_cross(q, cache, eager.init_cross_metadata(now, kv, tab, replayed=True))
        torch.cuda.synchronize()
        assert torch.equal(out[:sum(now)], want[:sum(now)])
    with pytest.raises(ValueError):
        be.update_forward_metadata(meta, [401, 0, 0], states, table)
    with pytest.raises(ValueError, match="max_query_len"):
        be.init_cross_metadata([1501], [77], table)


# ---- more sequences than a wave has lanes, each block by itself

@pytest.mark.parametrize("form,page", [("bf16", 16), ("head", 24), (16, 48), (32, 32), (64, 64), (128, 128)])
@pytest.mark.parametrize("kind", ["copy", "one", "each"])
def test_move_of_many_sequences(form, page, kind):
    """200 sequences, a quarter of them empty: every row, block and scale against the definition."""
    g = np.random.default_rng(30)
    lens = [int(n) for n in g.integers(0, 60, 200) * (g.random(200) < 0.75)]
    lens[150] = 300
    run_move(form, page, kind, lens=lens)
    if kind != "copy":
        run_move(form, page, kind, lens=lens, in_place=True)


# ---- calls whose workgroups take several shares of the work: bit for bit what calls of a few sequences give,
# in which each workgroup has one at most (the tests above and beside this file hold those to the definition)

MOST = 400      # tokens of a sequence, at most


def pools(form, lens, hkv, page, seed):
    """A cache of random rows, and its table of shuffled pages."""
    g = torch.Generator("cuda").manual_seed(seed)
    width = -(-MOST // page)
    need = [-(-n // page) for n in lens]
    order = np.random.default_rng(seed).permutation(sum(need)).astype(np.int32)
    table = np.full((len(lens), width), 2 ** 30, np.int32)
    for b, (n, at) in enumerate(zip(need, np.cumsum([0] + need))):
        table[b, :n] = order[at:at + n]
    slots = sum(need) * page
    x = [torch.randn((slots, hkv, 128), device="cuda", generator=g) for _ in "kv"]
    if form == "bf16":
        return fp2.KVCache(*(t.bfloat16() for t in x)), table
    codes = [(t * 100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for t in x]
    if form == "head":
        return fp2.KVCache(*codes, *(torch.rand(hkv, device="cuda", generator=g) * 0.01 + 0.005 for _ in "kv")), table
    return fp2.KVCache(*codes, *(torch.randint(110, 130, (slots // form, hkv), dtype=torch.uint8, device="cuda", generator=g)
                                 for _ in "kv")), table


def copy_of(c):
    return fp2.KVCache(*(None if x is None else x.clone() for x in (c.k, c.v, c.k_scale, c.v_scale)))


def lengths_of(n, most, long, seed):
    """Most of them up to `most`, one in ten empty, one in thirty up to `long`."""
    g = np.random.default_rng(seed)
    a = g.integers(1, most + 1, n)
    a[g.random(n) < 0.1] = 0
    far = g.random(n) < 1 / 30
    a[far] = g.integers(most, long + 1, far.sum())
    a[n // 2] = long
    return [int(x) for x in a]


def call_of(form, lens, new, hq, hkv, page, width):
    return fp2.make_cache_params(batch=len(lens), num_q_heads=hq, num_kv_heads=hkv, max_seq_len=new, max_kv_len=MOST,
                                 page_size=page, max_pages_per_seq=width, dtype="bf16" if form == "bf16" else "fp8",
                                 scale_tokens=form if isinstance(form, int) else 0)


LARGE = [("bf16", 16), ("head", 16), (16, 16), (32, 32), (64, 64), (128, 128)]


@pytest.mark.parametrize("form,page", LARGE)
def test_large_append(form, page):
    """3000 sequences of 8 heads: 7000 runs of tokens and more, in 2048 workgroups of keys and values; 20000 runs of
    eight queries of 8 heads in 16384 waves."""
    hq, hkv, n = 16, 8, 3000
    new = lengths_of(n, 36, 300, 40)
    lens = [a + int(b) for a, b in zip(new, np.random.default_rng(41).integers(0, 90, n))]
    cache, table = pools(form, lens, hkv, page, 42)
    few, r, total = copy_of(cache), fp2.make_rotary(96), sum(new)
    assert sum(m // 8 + 1 for m in new) * 2 > 16384
    g = torch.Generator("cuda").manual_seed(43)
    q, k, v = (torch.randn((total, h, 128), device="cuda", generator=g).bfloat16() for h in (hq, hkv, hkv))
    cu, cuk, tab = cu_of(new), cu_of(lens), dev(table)
    print("large append %s, %d tokens" % (form, total), flush=True)
    out = fp2.cache_append_rotary(call_of(form, lens, 300, hq, hkv, page, table.shape[1]), r, q, k, v, cache, dev(cu),
                                  dev(cuk), tab)
    for b in range(0, n, 50):
        part = slice(b, min(b + 50, n))
        rows_ = slice(int(cu[b]), int(cu[part.stop]))
        if rows_.start == rows_.stop:
            continue
        got = fp2.cache_append_rotary(call_of(form, lens[part], 300, hq, hkv, page, table.shape[1]), r, q[rows_], k[rows_],
                                      v[rows_], few, dev(cu_of(new[part])), dev(cu_of(lens[part])), tab[part].contiguous())
        assert torch.equal(out[rows_], got)
    torch.cuda.synchronize()
    equal(cache, few)


@pytest.mark.parametrize("form,page", [("bf16", 16), ("head", 16), (16, 16), (64, 64)])
def test_large_read(form, page):
    """14000 sequences: 70000 runs of 16 tokens' keys or values in 65536 waves."""
    hkv, n = 2, 14000
    lens = lengths_of(n, 16, 300, 50)
    new = [max(m - int(x), 0) for m, x in zip(lens, np.random.default_rng(51).integers(0, 9, n))]
    cache, table = pools(form, lens, hkv, page, 52)
    r, total = fp2.make_rotary(128, interleaved=True), sum(new)
    assert (total // 16 + 2 * n) * 2 > 65536
    cu, cuk, tab = cu_of(new), cu_of(lens), dev(table)
    print("large read %s, %d tokens" % (form, total), flush=True)
    k, v = fp2.cache_read(call_of(form, lens, 300, hkv, hkv, page, table.shape[1]), cache, dev(cu), dev(cuk), tab, rotary=r,
                          rows=total)
    for b in range(0, n, 1000):
        part = slice(b, min(b + 1000, n))
        rows_ = slice(int(cu[b]), int(cu[part.stop]))
        wk, wv = fp2.cache_read(call_of(form, lens[part], 300, hkv, hkv, page, table.shape[1]), cache, dev(cu_of(new[part])),
                                dev(cu_of(lens[part])), tab[part].contiguous(), rotary=r, rows=rows_.stop - rows_.start)
        assert torch.equal(k[rows_], wk) and torch.equal(v[rows_], wv)
    # values by themselves: a number times a power of two is exact, times a head's scale rounded to fp32 and then bf16
    at = np.concatenate([np.arange(m - x, m) for m, x in zip(lens, new)])
    slots = dev(table[np.repeat(np.arange(n), new), at // page].astype(np.int64) * page + at % page)
    want = cache.v[slots]
    if form != "bf16":
        want = want.view(torch.float8_e4m3fn).float()
        want = want * (cache.v_scale if form == "head" else (cache.v_scale[slots // form].int() << 23).view(torch.float32))[..., None]
    torch.cuda.synchronize()
    assert torch.equal(v, want.bfloat16())


@pytest.mark.parametrize("form,page", LARGE)
@pytest.mark.parametrize("in_place", [True, False])
def test_large_move(form, page, in_place):
    """6000 sequences of 8 heads, at least as many runs of tokens, in 2048 workgroups; with a number of positions for
    each sequence, and for each head and token."""
    hkv, n = 8, 6000
    lens = lengths_of(n, 40, 300, 60)
    cache, table = pools(form, lens, hkv, page, 61)
    to = None
    if not in_place:       # a pool twice as large, the targets in its second half
        grow = lambda x: None if x is None else x if x.dim() == 1 else torch.cat([x, torch.zeros_like(x)])      # noqa: E731
        half = cache.k.shape[0] // page
        cache = fp2.KVCache(*(grow(x) for x in (cache.k, cache.v, cache.k_scale, cache.v_scale)))
        to = dev(np.where(table == 2 ** 30, table, table + half).astype(np.int32))
    few, r, cuk, tab = copy_of(cache), fp2.make_rotary(128), cu_of(lens), dev(table)
    g = torch.Generator("cuda").manual_seed(62)
    for moves in (torch.randint(-9000, 9000, (n,), dtype=torch.int32, device="cuda", generator=g),
                  torch.randint(-9000, 9000, (n, hkv, MOST), dtype=torch.int32, device="cuda", generator=g)):
        print("large move %s, %d tokens, moves %s" % (form, sum(lens), tuple(moves.shape)), flush=True)
        fp2.cache_move(call_of(form, lens, 0, hkv, hkv, page, table.shape[1]), cache, dev(cuk), tab, to, rotary=r, moves=moves)
        for b in range(0, n, 80):
            part = slice(b, min(b + 80, n))
            fp2.cache_move(call_of(form, lens[part], 0, hkv, hkv, page, table.shape[1]), few, dev(cu_of(lens[part])),
                           tab[part].contiguous(), None if to is None else to[part].contiguous(), rotary=r, moves=moves[part])
        torch.cuda.synchronize()
        equal(cache, few)


# ---- queries turned in place on the way into the cache, and as codes on into the sparse prefill

@pytest.mark.parametrize("new", [[1] * 5, [2, 0, 1, 2, 1], [4, 3, 0, 1, 4], [8, 1, 0, 5, 7], [16, 9, 0, 1, 12],
                                 [32, 17, 0, 3, 20], [40, 33, 0, 1, 250]])
@pytest.mark.parametrize("dim,interleaved", [(128, False), (64, True), (100, False)])
def test_append_turns_queries_in_place(new, dim, interleaved):
    """As to rows of their own: dense queries, and those of a wider matrix, whose other columns stay."""
    hq, hkv, page = 8, 2, 16
    lens = [n + 13 * b for b, n in enumerate(new)]
    total, r = sum(new), fp2.make_rotary(dim, interleaved=interleaved)
    g = torch.Generator().manual_seed(70)
    m = torch.randn((total + 2, hq + 2 * hkv, 128), generator=g).bfloat16().cuda()
    parts = lambda x: (x[:total, :hq], x[:total, hq:hq + hkv], x[:total, hq + hkv:])        # noqa: E731
    cache, table = pools(16, lens, hkv, page, 71)
    p = fp2.make_cache_params(batch=5, num_q_heads=hq, num_kv_heads=hkv, max_seq_len=max(new), max_kv_len=max(lens),
                              page_size=page, max_pages_per_seq=table.shape[1], dtype="fp8", scale_tokens=16)
    args = dev(cu_of(new)), dev(cu_of(lens)), dev(table)
    print("in place, new %s dim %d" % (new, dim), flush=True)
    first, second, third = cache, copy_of(cache), copy_of(cache)
    before = m.clone()
    want = fp2.cache_append_rotary(p, r, *parts(m), first, *args)
    assert torch.equal(m, before)
    q, k, v = parts(m)
    dense = q.contiguous()
    assert fp2.cache_append_rotary(p, r, dense, k, v, second, *args, out=dense) is dense
    assert torch.equal(dense, want)
    assert fp2.cache_append_rotary(p, r, q, k, v, third, *args, out=q, cu_seqlens_host=cu_of(new)) is q
    torch.cuda.synchronize()
    assert torch.equal(q, want) and torch.equal(m[:, hq:], before[:, hq:]) and torch.equal(m[total:], before[total:])
    equal(first, second)
    equal(first, third)


def test_codes_of_turned_queries_into_the_sparse_prefill():
    """A prompt whose keys an append turns into a cache with a scale per head, its queries turned to codes, all
    blocks kept: against dense attention over what cache and codes hold. The bar is that of the sparse kernels'
    parity tests in codes, 6e-2."""
    n, cfg = 500, config("head")
    sparse = serving.PrefillBackend(serving.BackendConfig(
        num_q_heads=HQ, num_kv_heads=HKV, page_size=PAGE, max_batch=1, max_extend_len=600, max_kv_len=1024,
        dtype="fp8", window_blocks=8))
    be = serving.CacheBackend(cfg)
    (table,), pages = tables(cfg, 1, 14)
    g = torch.Generator().manual_seed(14)
    q, k, v = rows(g, n)
    r, freq = fp2.make_rotary(128), fp2.rotary_frequencies(128)[0]
    cache, scale = be.alloc_cache(pages, *scales("head")), torch.full((HQ,), 0.0125, device="cuda")
    meta = be.init_forward_metadata([n], None, table)
    codes = fp2.cache_append_rotary(meta.params, r, q, k, v, cache, meta.cu_q, meta.cu_k, meta.block_table, q_scale=scale)
    alone = fp2.rotary(r, q, torch.arange(n, dtype=torch.int32, device="cuda"), q_scale=scale)
    out, _ = sparse.forward_extend(codes, cache.k, cache.v, sparse.init_forward_metadata([n], None, table), q_scale=scale,
                                   k_scale=cache.k_scale, v_scale=cache.v_scale)
    torch.cuda.synchronize()
    assert torch.equal(codes, alone)
    by = float(np.float32(0.0125))
    want, err = pos_ref.turn(q.double().cpu().numpy(), np.repeat(np.arange(n)[:, None], HQ, 1), freq, False)
    pos_ref.check_codes(codes, want / by, err / by + np.abs(want / by) * pos_ref.U, "codes")
    turned = torch.from_numpy(ref.VALUES[codes.cpu().numpy()] * by)
    o = ref.attend(view(cfg, [n], cache, table, "head"), turned, [n])[0]
    assert np.abs(out.double().cpu().numpy() - o).max() <= 6e-2

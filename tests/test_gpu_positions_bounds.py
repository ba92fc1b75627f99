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
from tests.test_gpu_cache_serving import HKV, HQ, config, rows, scales, tables
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

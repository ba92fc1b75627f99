"""Rotary positions and cross attention as an engine uses them: forwards that turn what they
append, eviction to new indexes, a cache read back and moved, an encoder's states; captured and
replayed, on streams of their own, two calls at once."""
import numpy as np
import pytest
import torch

import paper_2608_19758_amd as fp2
from paper_2608_19758_amd import serving
from tests import cache_ref as ref
from tests import positions_ref as pos_ref
from tests.test_gpu_cache import close, cu_of, dev
from tests.test_gpu_cache_serving import HKV, HQ, PAGE, config, equal, rows, scales, tables

pytestmark = pytest.mark.gpu


def spoil():
    """Work of the program's own between replays."""
    float(torch.randn(1 << 18, device="cuda").sum())


def view(cfg, lens, cache, table, form):
    """The reference's view of a cache."""
    c = ref.Cache([1] * len(lens), HKV, form, PAGE, room=cfg.max_kv_len - 1)
    c.lens, c.table = list(lens), table.cpu().numpy()
    c.k, c.v = cache.k.cpu(), cache.v.cpu()
    c.ks, c.vs = (None if x is None else x.cpu() for x in (cache.k_scale, cache.v_scale))
    return c


def turned(r, q, at):
    return fp2.rotary(r, q, dev(np.asarray(at, np.int32)))


@pytest.mark.parametrize("form", ["bf16", "head", 16, 64])
@pytest.mark.parametrize("own_stream", [False, True])
def test_forwards_evict_and_go_on(form, own_stream):
    """Prompt, steps, eviction that turns the keys to their new indexes, and steps behind it: each output against
    the definition over what the cache holds, and the keys against what their tokens had."""
    cfg = config(form, sink_tokens=4)
    stream = torch.cuda.Stream() if own_stream else None
    be = serving.CacheBackend(cfg, stream=stream)
    (table, target), pages = tables(cfg, 2, 3)
    g = torch.Generator().manual_seed(1)
    cache, w = be.alloc_cache(pages, *scales(form)), be.alloc_weights()
    r = fp2.make_rotary(96, interleaved=True)
    freq = fp2.rotary_frequencies(96)[0]
    lens, keys = [0, 0], [[], []]
    for ext in ([300, 71], [1, 3], [17, 0]):
        x = rows(g, sum(ext))
        torch.cuda.synchronize()
        meta = be.init_forward_metadata(ext, lens, table)
        out, lse = be.forward(*x, cache, meta, want_lse=True, weights=w, rotary=r)
        torch.cuda.synchronize()
        index = np.concatenate([np.arange(a, a + e) for a, e in zip(lens, ext)])
        lens = [a + e for a, e in zip(lens, ext)]
        for b, part in enumerate(np.split(x[1].double().cpu().numpy(), np.cumsum(ext)[:-1])):
            keys[b].append(part)
        c = view(cfg, lens, cache, table, form)
        q = turned(r, x[0], index)
        torch.cuda.synchronize()
        o, tol, z, ztol, _ = ref.attend(c, q.cpu(), ext)
        close(out, o, tol, "out")
        close(lse, z, ztol, "lse")
    budget = 128
    old = view(cfg, lens, cache, table, form)
    kept, left = be.evict(cache, w, meta, target[:, :cfg.max_pages_per_seq].contiguous(), budget=budget, recent_tokens=16,
                          rotary=r)
    torch.cuda.synchronize()
    kept = kept.cpu().numpy()
    stay = serving.evicted_lens(meta, budget)
    assert stay == [128, 74]
    c = view(cfg, stay, cache, target, form)
    for b, n in enumerate(stay):
        for h in range(HKV):
            at = kept[b, h, :n]
            raw = np.concatenate(keys[b])[at, h]
            want, _ = pos_ref.turn(raw, np.arange(n), freq, True)
            got = c.values("k", c.slots(b, np.arange(n)), h)
            was = old.values("k", old.slots(b, at), h)
            # Each rounding of a code is off by at most half a step: 2^-4 of a number (bf16 2^-8), or, among the
            # subnormal ones, half of 2^-9 scales. The first by its own value, turned; those of the eviction (a
            # block's codes may round again where its scale changes) and of the move by theirs. A turn spreads an
            # error over its pair: at most the sum of both.
            eps = 2.0 ** -8 if form == "bf16" else 2.0 ** -4
            step = 0.0
            if form == "head":
                step = 2.0 ** -10 * float(c.ks[h])
            elif form != "bf16":
                step = 2.0 ** -10 * 2.0 ** (np.maximum.reduce(
                    [c.ks[c.slots(b, np.arange(n)) // c.sb, h].numpy().astype(int),
                     old.ks[old.slots(b, at) // old.sb, h].numpy().astype(int)])[:, None] - 127.0)
            big = np.abs(raw) + np.abs(was) + np.abs(got)
            pair = big.copy()
            pair[:, 0:96:2] += big[:, 1:96:2]
            pair[:, 1:96:2] += big[:, 0:96:2]
            assert (np.abs(got - want) <= 2 * eps * pair + 6 * step + 1e-6).all()
    # and on: positions go on from the new lengths
    for ext in ([1, 1], [5, 2]):
        x = rows(g, sum(ext))
        meta = be.init_forward_metadata(ext, stay, target)
        torch.cuda.synchronize()
        out, _ = be.forward(*x, cache, meta, weights=left, rotary=r)
        torch.cuda.synchronize()
        index = np.concatenate([np.arange(a, a + e) for a, e in zip(stay, ext)])
        stay = [a + e for a, e in zip(stay, ext)]
        q = turned(r, x[0], index)
        torch.cuda.synchronize()
        o, tol, _, _, _ = ref.attend(view(cfg, stay, cache, target, form), q.cpu(), ext)
        close(out, o, tol, "out behind the eviction")


@pytest.mark.parametrize("form", ["bf16", 64])
@pytest.mark.parametrize("new", [1, 40])
def test_captured_forward(form, new):
    """A forward with positions, captured once and replayed with other lengths, pages and positions."""
    cfg = config(form)
    be, eager = serving.CacheBackend(cfg), serving.CacheBackend(cfg)
    (table,), pages = tables(cfg, 1, 4)
    g = torch.Generator().manual_seed(2)
    a, b = (be.alloc_cache(pages) for _ in "ab")
    r = fp2.make_rotary(128)
    lens = [70, 300, 3]
    x = rows(g, sum(lens))
    for e, cache in ((be, a), (eager, b)):
        e.forward(*x, cache, e.init_forward_metadata(lens, None, table), rotary=r)
    ext = [new] * 3
    meta = be.init_forward_metadata(ext, lens, table, replayed=True)
    static, out = rows(g, 3 * new), torch.zeros((3 * new, HQ, 128), dtype=torch.bfloat16, device="cuda")
    positions = torch.zeros(3 * new, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        be.forward(*static, a, meta, out=out, rotary=r, positions=positions)
    for step in range(5):
        now = [new, max(new - step, 0), new] if new > 1 else ext
        total = sum(now)
        be.update_forward_metadata(meta, now, lens, table)
        x = rows(g, total)
        at = torch.cat([torch.arange(n, n + m) + 1000 * step for n, m in zip(lens, now)]).int().cuda()
        for s, t in zip(static, x):
            s[:total].copy_(t)
        positions[:total].copy_(at)
        graph.replay()
        spoil()
        m2 = eager.init_forward_metadata(now, lens, table, replayed=True)
        want, _ = eager.forward(*x, b, m2, rotary=r, positions=at)
        torch.cuda.synchronize()
        assert torch.equal(out[:total], want), step
        equal(a, b)
        lens = [n + m for n, m in zip(lens, now)]
    with pytest.raises(ValueError, match="rows"):
        be.forward(*static, a, meta, rotary=r, positions=positions[:1])
    with pytest.raises(ValueError, match="without rotary"):
        be.forward(*static, a, meta, positions=positions)


@pytest.mark.parametrize("form", ["bf16", "head", 32])
def test_cross(form):
    """An encoder's states written once; decoder prompts and steps over them, captured steps among them."""
    cfg = config(form, window_tokens=100, sink_tokens=2)
    be, eager = serving.CacheBackend(cfg), serving.CacheBackend(cfg)
    (table,), pages = tables(cfg, 1, 5)
    g = torch.Generator().manual_seed(3)
    cache = be.alloc_cache(pages, *scales(form))
    states = [600, 0, 77]
    _, k, v = rows(g, sum(states))
    be.append(k, v, cache, be.init_forward_metadata(states, None, table))
    for new in ([100, 9, 600], [1, 1, 1], [0, 3, 2]):
        q = rows(g, sum(new))[0]
        out, lse = be.forward_cross(q, cache, be.init_cross_metadata(new, states, table), want_lse=True)
        torch.cuda.synchronize()
        o, tol, z, ztol = pos_ref.cross(view(cfg, states, cache, table, form), q.cpu(), new)
        close(out, o, tol, "out")
        close(lse, z, ztol, "lse")
    for n in (1, 70):
        new = [n] * 3
        meta = be.init_cross_metadata(new, states, table, replayed=True)
        q, out = rows(g, 3 * n)[0], torch.zeros((3 * n, HQ, 128), dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            be.forward_cross(q, cache, meta, out=out)
        for order, now in (([0, 1, 2], new), ([2, 0, 1], new), ([1, 2, 0], [n, max(n - 5, 1), n]), ([0, 1, 2], new)):
            tab, kv = table[order], [states[i] for i in order]
            be.update_forward_metadata(meta, now, kv, tab)
            graph.replay()
            spoil()
            want, _ = eager.forward_cross(q, cache, eager.init_cross_metadata(now, kv, tab, replayed=True))
            torch.cuda.synchronize()
            assert torch.equal(out[:sum(now)], want[:sum(now)])
    meta = be.init_cross_metadata([1, 1, 1], states, table)
    with pytest.raises(ValueError, match="cross"):
        be.forward(q, k, v, cache, meta)
    with pytest.raises(ValueError, match="forward"):
        be.forward_cross(q, cache, be.init_forward_metadata([1], [5], table))
    with pytest.raises(ValueError, match="rows"):
        be.forward_cross(q[:2], cache, meta)


@pytest.mark.parametrize("form", ["bf16", 16])
def test_document_taken_over_at_another_offset(form):
    """A cached document moved behind a prompt of another request: attention over both equals the one over a cache
    that was filled in order, within the roundings of the keys; and it reads back as it was."""
    cfg = config(form)
    be = serving.CacheBackend(cfg)
    (table, other), pages = tables(cfg, 2, 6)
    g = torch.Generator().manual_seed(4)
    r = fp2.make_rotary(128, base=500000.0)
    cache = be.alloc_cache(pages)
    doc, front = 130, 3 * PAGE
    _, k, v = rows(g, doc)
    meta = be.init_forward_metadata([doc], None, table)
    be.forward(torch.zeros((doc, HQ, 128), dtype=torch.bfloat16, device="cuda"), k, v, cache, meta, rotary=r)
    plain, values = be.read(cache, meta, rotary=r)
    torch.cuda.synchronize()
    eps = 2.0 ** -8 if form == "bf16" else 2.0 ** -4
    assert float((values.double() - v.double()).abs().max()) <= (0 if form == "bf16" else eps * float(v.abs().max()))
    kd = k.double()
    pair = kd.abs() + torch.cat([kd[..., 64:], kd[..., :64]], -1).abs()
    # rounded as a code and, once more, as a bf16 row; half a step of a block's smallest codes is 2^-10 of its scale,
    # at most 2^-9 of the block's largest value / 448 (the scale is below twice that)
    bound = (eps + 2.0 ** -8) * (1 + eps) * pair + (0 if form == "bf16" else 4 * 2.0 ** -10 * 2 * 1.5 * float(k.abs().max()) / 448)
    assert bool(((plain.double() - kd).abs() <= bound).all())
    # the document's pages behind three others of another sequence
    moved = be.init_forward_metadata([doc], None, table)
    be.move(cache, moved, other[:1, 3:3 + cfg.max_pages_per_seq].contiguous(), rotary=r,
            moves=torch.tensor([front], dtype=torch.int32, device="cuda"))
    x = rows(g, front)
    be.forward(*x, cache, be.init_forward_metadata([front], None, other), rotary=r)
    torch.cuda.synchronize()
    slots = view(cfg, [front + doc], cache, other, form)
    freq = fp2.rotary_frequencies(128, 500000.0)[0]
    want, _ = pos_ref.turn(k.double().cpu().numpy(), np.repeat(np.arange(front, front + doc)[:, None], HKV, 1), freq, False)
    for h in range(HKV):
        got = slots.values("k", slots.slots(0, np.arange(front, front + doc)), h)
        p = pair[:, h].cpu().numpy()
        step = 0 if form == "bf16" else 4 * 2.0 ** -10 * 2 * 1.5 * float(k.abs().max()) / 448
        assert (np.abs(got - want[:, h]) <= 2.1 * eps * (1 + 2 * eps) * p + 2 * step + 1e-6).all()
    q = rows(g, 1)
    out, _ = be.forward(*q, cache, be.init_forward_metadata([1], [front + doc], other), rotary=r)
    torch.cuda.synchronize()
    t = turned(r, q[0], [front + doc])
    torch.cuda.synchronize()
    o, tol, _, _, _ = ref.attend(view(cfg, [front + doc + 1], cache, other, form), t.cpu(), [1])
    close(out, o, tol, "out")


def test_calls_on_two_streams():
    """Calls that overlap, on streams of their own, with workspaces of their own."""
    g = torch.Generator().manual_seed(5)
    r = fp2.make_rotary(128)
    c = ref.Cache([4000, 700], 4, 64, 64, seed=20)
    q = torch.randn((300, 16, 128), generator=g).bfloat16().cuda()
    cache = fp2.KVCache(dev(c.k), dev(c.v), dev(c.ks), dev(c.vs))
    cu, cuk, table = dev(cu_of([200, 100])), dev(cu_of(c.lens)), dev(c.table)
    at = torch.arange(300, dtype=torch.int32, device="cuda")
    p = fp2.make_cache_params(batch=2, num_q_heads=16, num_kv_heads=4, max_seq_len=200, max_kv_len=4000, page_size=64,
                              max_pages_per_seq=c.width, dtype="fp8", scale_tokens=64)

    def work(stream):
        turned = fp2.rotary(r, q, at, stream=stream)
        out, _ = fp2.cache_cross(p, turned, cache, cu, cuk, table, stream=stream)
        k, v = fp2.cache_read(p, cache, cu, cuk, table, rows=300, rotary=r, stream=stream)
        return turned, out, k, v

    want = work(None)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(4):
        got = [work(s) for s in streams]
        torch.cuda.synchronize()
        for one in got:
            for x, y in zip(one, want):
                assert torch.equal(x, y)


def test_slots_past_4_gib():
    """Rows whose places in the pool pass 32 bits."""
    slots = (1 << 25) + 64            # of 128 bf16: 8 GiB a pool
    r = fp2.make_rotary(128)
    k = torch.zeros((slots, 1, 128), dtype=torch.bfloat16, device="cuda")
    cache = fp2.KVCache(k, torch.zeros_like(k))
    p = fp2.make_cache_params(batch=1, num_q_heads=1, num_kv_heads=1, max_seq_len=64, max_kv_len=64, page_size=64)
    table = torch.tensor([[slots // 64 - 1]], dtype=torch.int32, device="cuda")
    low = torch.tensor([[1]], dtype=torch.int32, device="cuda")
    x = torch.randn((64, 1, 128)).bfloat16().cuda()
    cu = dev(cu_of([64]))
    q = fp2.cache_append_rotary(p, r, x, x, x, cache, cu, cu, table)
    assert torch.equal(cache.k[-64:], q) and torch.equal(cache.v[-64:], x)
    fp2.cache_move(p, cache, cu, table, low)
    assert torch.equal(cache.k[64:128], q) and torch.equal(cache.v[64:128], x)
    got, v = fp2.cache_read(p, cache, cu, cu, table, rows=64)
    assert torch.equal(got, q) and torch.equal(v, x)
    far, _ = fp2.cache_cross(p, q, cache, cu, cu, table)
    near, _ = fp2.cache_cross(p, q, cache, cu, cu, low)
    assert torch.equal(far, near)
    q1 = q[:1].contiguous()
    one = fp2.make_cache_params(batch=1, num_q_heads=1, num_kv_heads=1, max_seq_len=1, max_kv_len=64, page_size=64)
    far, _ = fp2.cache_cross(one, q1, cache, dev(cu_of([1])), cu, table)
    assert torch.equal(far, fp2.cache_cross(one, q1, cache, dev(cu_of([1])), cu, low)[0])


def test_more_sequences_than_lanes():
    """Hundreds of sequences, many of them without tokens."""
    g = np.random.default_rng(6)
    lens = [int(n) for n in g.integers(0, 40, 300)]
    lens[150] = 700
    new = [min(n, int(m)) for n, m in zip(lens, g.integers(0, 30, 300))]
    r = fp2.make_rotary(64)
    freq = fp2.rotary_frequencies(64)[0]
    c = ref.Cache(lens, 2, 16, 16, seed=21)
    p = fp2.make_cache_params(batch=300, num_q_heads=4, num_kv_heads=2, max_seq_len=max(new), max_kv_len=700, page_size=16,
                              max_pages_per_seq=c.width, dtype="fp8", scale_tokens=16)
    cache = fp2.KVCache(dev(c.k), dev(c.v), dev(c.ks), dev(c.vs))
    cu, cuk, table = dev(cu_of(new)), dev(cu_of(lens)), dev(c.table)
    k, _ = fp2.cache_read(p, cache, cu, cuk, table, rows=sum(new), rotary=r)
    slots = np.concatenate([c.slots(b, np.arange(n - m, n)) for b, (n, m) in enumerate(zip(lens, new))])
    index = np.concatenate([np.arange(n - m, n) for n, m in zip(lens, new)])
    raw = np.stack([c.values("k", slots, h) for h in range(2)], 1)
    want, err = pos_ref.turn(raw, np.repeat(index[:, None], 2, 1), freq, False, back=True)
    pos_ref.check_bf16(k, want, err, "k")
    for many in (new, [3 * n + (i % 7) for i, n in enumerate(new)]):
        pc = fp2.make_cache_params(batch=300, num_q_heads=4, num_kv_heads=2, max_seq_len=max(many), max_kv_len=700,
                                   page_size=16, max_pages_per_seq=c.width, dtype="fp8", scale_tokens=16)
        q = torch.randn((sum(many), 4, 128), generator=torch.Generator().manual_seed(7)).bfloat16()
        out, lse = fp2.cache_cross(pc, dev(q), cache, dev(cu_of(many)), cuk, table, want_lse=True)
        torch.cuda.synchronize()
        o, tol, z, ztol = pos_ref.cross(c, q, many)
        close(out, o, tol, "out")
        close(lse, z, ztol, "lse")
    before = cache.k.clone()
    moves = torch.full((300,), 11, dtype=torch.int32, device="cuda")
    fp2.cache_move(p, cache, cuk, table, rotary=r, moves=moves)
    k2, _ = fp2.cache_read(p, cache, cuk, cuk, table, rows=sum(lens))
    slots = np.concatenate([c.slots(b, np.arange(n)) for b, n in enumerate(lens)])
    raw = np.stack([c.values("k", slots, h) for h in range(2)], 1)
    want, _ = pos_ref.turn(raw, np.full((len(slots), 2), 11), freq, False)
    # one rounding to a code of a block whose scale is at most 2 / 448 of its largest value
    size = np.abs(want).max()
    assert np.abs(k2.double().cpu().numpy() - want).max() <= 2.0 ** -4 * size + 2.0 ** -8 * size
    assert not torch.equal(before, cache.k)


def test_captured_rotary_read_and_move():
    """The calls themselves in a graph: other positions, lengths and moves at each replay."""
    r = fp2.make_rotary(128, interleaved=True)
    c = ref.Cache([300, 100], 2, "bf16", 16, seed=22)
    p = fp2.make_cache_params(batch=2, num_q_heads=4, num_kv_heads=2, max_seq_len=300, max_kv_len=300, page_size=16,
                              max_pages_per_seq=c.width)
    cache = fp2.KVCache(dev(c.k), dev(c.v))
    start = cache.k.clone()
    q = torch.randn((50, 4, 128)).bfloat16().cuda()
    at, by = torch.zeros(50, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    cu, cuk, table = torch.zeros(3, dtype=torch.int32, device="cuda"), dev(cu_of(c.lens)), dev(c.table)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        turned = fp2.rotary(r, q, at)
        fp2.cache_move(p, cache, cuk, table, rotary=r, moves=by)
        k, v = fp2.cache_read(p, cache, cu, cuk, table, rows=400)
    for step, new in enumerate(([300, 100], [5, 0], [0, 99], [128, 64], [300, 100])):
        cache.k.copy_(start)
        at.copy_(torch.arange(50) * (step + 1))
        by.fill_(7 * step - 10)
        cu.copy_(dev(cu_of(new)))
        graph.replay()
        spoil()
        got = [turned.clone(), k.clone(), v.clone(), cache.k.clone()]
        cache.k.copy_(start)
        n = sum(new)
        want = fp2.rotary(r, q, at)
        fp2.cache_move(p, cache, cuk, table, rotary=r, moves=by)
        wk, wv = fp2.cache_read(p, cache, cu, cuk, table, rows=400)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want) and torch.equal(got[1][:n], wk[:n]) and torch.equal(got[2][:n], wv[:n])
        assert torch.equal(got[3].view(torch.int16), cache.k.view(torch.int16))

"""The paged cache's operators on the GPU against their definitions in 64 bits
(tests/cache_ref.py): every form of cache, single tokens to prompts, windows and
first tokens, odd sizes, infinities and NaN in places that no query sees."""
import numpy as np
import pytest
import torch

import paper_2608_19758_amd as fp2
from tests import cache_ref as ref

pytestmark = pytest.mark.gpu


def dev(x):
    return None if x is None else (torch.from_numpy(x) if isinstance(x, np.ndarray) else x).cuda()


def cu_of(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def params(c, hq, new, window=0, sink=0, splits=0, max_new=None, max_kv=None, scale=0.0):
    return fp2.make_cache_params(
        batch=len(c.lens), num_q_heads=hq, num_kv_heads=c.hkv, max_seq_len=max_new or max(new),
        max_kv_len=max_kv or max(c.lens), page_size=c.page, max_pages_per_seq=c.width,
        dtype="bf16" if c.form == "bf16" else "fp8", scale_tokens=c.sb, sink_tokens=sink,
        window_tokens=window, kv_splits=splits, softmax_scale=scale)


def on_gpu(c):
    return fp2.KVCache(dev(c.k), dev(c.v), dev(c.ks), dev(c.vs))


def same(got, want, what):
    got, want = got.cpu(), want
    if got.dtype == torch.bfloat16:
        got, want = got.view(torch.int16), want.view(torch.int16)
    assert torch.equal(got, want), "%s differs at %d of %d" % (what, int((got != want).sum()), got.numel())


def close(got, want, tol, what):
    got = got.double().cpu().numpy() if isinstance(got, torch.Tensor) else got
    fin = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what + ": NaN in other places"
    assert np.array_equal(got[~fin & ~np.isnan(want)], want[~fin & ~np.isnan(want)]), what + ": infinities"
    over = np.abs(got[fin] - want[fin]) / tol[fin]
    print("%s: largest error %.3f of its bound" % (what, over.max() if over.size else 0), flush=True)
    assert not (over > 1).any(), what


def run_attend(c, hq, new, window=0, sink=0, splits=0, seed=1, scale=0.0, pad=3, weights=True):
    """Attention and weights of random queries against the definition."""
    print("attend lens %s new %s hkv %d hq %d %s page %d window %d sink %d splits %d"
          % (c.lens, new, c.hkv, hq, c.form, c.page, window, sink, splits), flush=True)
    g = torch.Generator().manual_seed(seed)
    q = torch.randn((sum(new) + pad, hq, 128), generator=g).bfloat16()
    n = sum(new)
    p = params(c, hq, new, window, sink, splits, scale=scale)
    cu, cuk = cu_of(new), cu_of(c.lens)
    out = torch.full((n + pad, hq, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n + pad, hq), 7.0, device="cuda")
    args = (dev(cu), dev(cuk), dev(c.table))
    ws = fp2.alloc_cache_workspace(p)
    ws.fill_(0xff)                                     # what a workspace holds does not matter
    cache = on_gpu(c)
    fp2.cache_attend(p, dev(q), cache, *args, out=out, lse=lse, workspace=ws, cu_seqlens_host=cu,
                     cu_seqlens_k_host=cuk)
    torch.cuda.synchronize()
    o, tol, z, ztol, _ = ref.attend(c, q[:n], new, window, sink, scale or None)
    close(out[:n], o, tol, "out")
    close(lse[:n], z, ztol, "lse")
    assert bool((out[n:] == 7).all()) and bool((lse[n:] == 7).all())     # rows behind the last sequence
    if not weights:
        return out, lse
    stride = max(c.lens) + 5
    before = torch.rand((len(c.lens), c.hkv, stride), generator=g)
    w = dev(before).clone()
    fp2.cache_weights(p, dev(q), lse, cache, *args, weights=w, weights_in=w)
    fresh = fp2.cache_weights(p, dev(q), lse, cache, *args, weights=torch.full_like(w, -1.0))
    moved = fp2.cache_weights(p, dev(q), lse, cache, *args, weights_in=dev(before))
    _, _, _, _, want = ref.attend(c, q[:n], new, window, sink, scale or None,
                                  lse[:n].double().cpu().numpy())
    for b, L in enumerate(c.lens):
        close(fresh[b, :, :L], want[b][0], want[b][1] + 1e-30, "weights of %d" % b)
        both = want[b][0] + before[b, :, :L].double().numpy()
        other = moved[b].cpu()
        assert torch.equal(other[:, L:], before[b, :, L:])
        close(other[:, :L], both, want[b][1] + 2 * ref.U32 * both, "weights of %d added elsewhere" % b)
        close(w[b, :, :L], both, want[b][1] + 2 * ref.U32 * both, "added weights of %d" % b)
        assert not bool(fresh[b, :, L:].any()) and torch.equal(w[b, :, L:].cpu(), before[b, :, L:])
    return out, lse


FORMS = ["bf16", "head", 16, 64]


@pytest.mark.parametrize("form", FORMS + [32, 128])
def test_single_tokens(form):
    c = ref.Cache([1, 2, 31, 32, 33, 129, 700], 2, form, 128, seed=1, spread=1.0)
    run_attend(c, 8, [1] * 7)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("g", [1, 2, 8])
def test_groups_and_drafts(form, g):
    """Several new tokens a sequence: 1 to 64 packed rows, sequences without any among them."""
    new = [8, 1, 0, 5, 3]
    c = ref.Cache([900, 1, 50, 64, 3], 3, form, 64, seed=2)
    run_attend(c, 3 * g, new)


@pytest.mark.parametrize("form,page", [("bf16", 1), ("bf16", 24), ("head", 5), ("head", 48), ("bf16", 4096),
                                       (16, 48), (32, 96), (64, 192)])
def test_pages(form, page):
    c = ref.Cache([333, 97, 16], 2, form, page, seed=3)
    run_attend(c, 8, [1, 4, 2])


@pytest.mark.parametrize("window,sink", [(1, 0), (1, 1), (17, 4), (64, 0), (100, 40), (33, 200), (5000, 4)])
@pytest.mark.parametrize("form", ["bf16", 16])
def test_windows(form, window, sink):
    c = ref.Cache([450, 97, 1, 230], 2, form, 16, seed=4)
    run_attend(c, 8, [1, 6, 1, 2], window, sink)


@pytest.mark.parametrize("form", ["bf16", "head", 64])
@pytest.mark.parametrize("splits", [0, 1, 7, 32])
def test_parts(form, splits):
    """Keys cut into parts: by the work of the call, into fixed numbers, or not at all."""
    c = ref.Cache([5000, 1300, 0, 60], 1, form, 64, seed=5)
    run_attend(c, 4, [1, 2, 0, 1], splits=splits)
    run_attend(c, 4, [1, 2, 0, 1], 900, 70, splits=splits)


def test_many_sequences():
    """More sequences than a wave holds lengths of."""
    lens = list(np.random.default_rng(7).integers(1, 400, 150))
    lens[70] = 3000
    c = ref.Cache(lens, 1, 16, 16, seed=6)
    run_attend(c, 2, [1] * 150)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("hq,hkv", [(8, 2), (2, 2), (8, 1)])
def test_prompts(form, hq, hkv):
    """Many rows: whole prompts and chunks behind a prefix."""
    c = ref.Cache([300, 517, 70, 9], hkv, form, 64, seed=8, spread=0.5)
    run_attend(c, hq, [300, 131, 0, 1])


@pytest.mark.parametrize("window,sink", [(1, 0), (40, 3), (64, 64), (130, 70), (257, 0)])
@pytest.mark.parametrize("form", ["bf16", 16])
def test_prompt_windows(form, window, sink):
    c = ref.Cache([600, 411], 2, form, 48, seed=9)
    run_attend(c, 8, [600, 200], window, sink)


@pytest.mark.parametrize("form,page", [("bf16", 1), ("bf16", 80), ("head", 24), (32, 32)])
def test_prompt_pages_and_parts(form, page):
    c = ref.Cache([1800], 1, form, page, seed=10)
    for splits in (0, 1, 5):
        run_attend(c, 4, [100], splits=splits)


def test_softmax_scale_and_large_scores():
    c = ref.Cache([200], 2, "bf16", 16, seed=11)
    c.k *= 6
    run_attend(c, 8, [3], scale=0.5)
    run_attend(c, 8, [100], scale=0.5)


@pytest.mark.parametrize("form", ["bf16", "head", 16])
@pytest.mark.parametrize("new", [1, 4, 90])
def test_odd_values_reach_only_rows_that_see_them(form, new):
    """Infinities and NaN among the values: rows that see the token get them, others do not,
    also where they share a tile. Keys of NaN outside the window reach nobody."""
    L, window = 400, 120
    c = ref.Cache([L], 2, form, 16, seed=12)
    nan, inf = (float("nan"), float("inf")) if form == "bf16" else (0x7f, 0xff)
    P = L - new
    at = {L - 1: inf, P: nan} if new > 1 else {}
    at.update({P - window: nan, P - window - 3: inf})      # just outside the first row's window
    if new == 90:
        at[P - window + 40] = nan                          # leaves the window while the rows go on
    for t, x in at.items():
        c.v[c.slots(0, t), :, 3:90:7] = x
    for t in range(5, P - window):
        c.k[c.slots(0, t)] = nan
    run_attend(c, 8, [new], window, 5, weights=False)


def test_queries_of_one_call_do_not_depend_on_others():
    """kv_splits 1: the rows of a sequence are the same alone and in a batch."""
    c = ref.Cache([700, 300], 2, 64, 64, seed=13)
    out, _ = run_attend(c, 8, [2, 3], splits=1, pad=0, weights=False)
    g = torch.Generator().manual_seed(1)
    q = torch.randn((5, 8, 128), generator=g).bfloat16()
    p = fp2.make_cache_params(batch=1, num_q_heads=8, num_kv_heads=2, max_seq_len=3, max_kv_len=700,
                              page_size=64, dtype="fp8", scale_tokens=64, kv_splits=1)
    one, _ = fp2.cache_attend(p, dev(q[2:]), on_gpu(c), dev(cu_of([3])), dev(cu_of([300])),
                              dev(c.table[1:, :p.max_pages_per_seq].copy()))
    assert torch.equal(one, out[2:])


# ---- append

def grown(lens, new, form, page, hkv=3, seed=0, odd=False, size=1.0):
    c = ref.Cache(lens, hkv, form, page, room=max(new), seed=seed, spread=1.5)
    c.lens = [a + b for a, b in zip(lens, new)]
    r = np.random.default_rng(seed + 100)
    x = [r.standard_normal((sum(new) + 2, hkv, 128)) * np.exp(2 * r.standard_normal((sum(new) + 2, hkv, 1))) * size
         for _ in "kv"]
    if odd:
        for y in x:
            y[::3, 0, 5], y[1::3, 1, 9], y[::4, 2, 0] = np.nan, np.inf, -np.inf
            y[2::5] = 0.0
    return c, torch.from_numpy(x[0]).bfloat16(), torch.from_numpy(x[1]).bfloat16()


def run_append(c, k, v, new):
    print("append lens %s new %s %s page %d" % (c.lens, new, c.form, c.page), flush=True)
    want = ref.append(c, k, v, new)
    cache = on_gpu(c)
    fp2.cache_append(params(c, c.hkv, new), dev(k), dev(v), cache, dev(cu_of(new)), dev(cu_of(c.lens)), dev(c.table),
                     cu_seqlens_host=cu_of(new), cu_seqlens_k_host=cu_of(c.lens))
    torch.cuda.synchronize()
    same(cache.k, want["k"], "k")
    same(cache.v, want["v"], "v")
    if c.ks is not None:
        same(cache.k_scale, want["ks"], "k_scale")
        same(cache.v_scale, want["vs"], "v_scale")
    return cache


@pytest.mark.parametrize("form,page", [("bf16", 1), ("bf16", 64), ("head", 7), (16, 16), (16, 48), (32, 64),
                                       (64, 64), (128, 128), (64, 192)])
@pytest.mark.parametrize("odd", [False, True])
def test_append(form, page, odd):
    """Whole pools compared: the new rows, the old rows of a first block, and nothing else."""
    for lens, new in (([0, 5, 130, 63], [1, 1, 1, 1]), ([0, 17, 200, 64], [300, 0, 129, 70]),
                      ([127, 1], [2, 15])):
        c, k, v = grown(lens, new, form, page, seed=len(lens), odd=odd)
        run_append(c, k, v, new)


@pytest.mark.parametrize("form,page", [("bf16", 24), ("head", 16), (16, 64), (32, 96), (128, 128)])
@pytest.mark.parametrize("new", [16, 17])
def test_append_few_tokens(form, page, new):
    """Few new tokens of many sequences, over the edges of blocks, with scales that grow and that do not."""
    lens = [0, 1, 15, 16, 31, 113, 120, 127, 128, 250]
    count = [new, 16, 1, 0, 16, 16, 9, 1, 16, 7]
    for size in (0.01, 1, 30.0):
        c, k, v = grown(lens, count, form, page, seed=31, size=size)
        run_append(c, k, v, count)


@pytest.mark.parametrize("size", [1e-36, 1e-30, 1e30, 1e38])
def test_append_extreme_sizes(size):
    c, k, v = grown([0, 20], [40, 3], 16, 16, size=size)
    run_append(c, k, v, [40, 3])


def test_append_keeps_what_a_growing_scale_can():
    """Token by token with growing values: codes are moved by powers of two, so a value loses only what
    falls below 2^-6 of the scale."""
    n = 32
    c = ref.Cache([0], 1, 32, 32, room=n, seed=3)
    x = torch.randn(n, 1, 128, generator=torch.Generator().manual_seed(2)).bfloat16() * \
        (2.0 ** (torch.arange(n) / 4))[:, None, None].bfloat16()
    x = x.bfloat16()
    cache = on_gpu(c)
    for t in range(n):
        c.lens = [t + 1]
        fp2.cache_append(params(c, 1, [1], max_kv=n), dev(x[t:t + 1]), dev(x[t:t + 1]), cache, dev(cu_of([1])),
                         dev(cu_of([t + 1])), dev(c.table))
    torch.cuda.synchronize()
    c.k, c.ks = cache.k.cpu(), cache.k_scale.cpu()
    got = c.values("k", c.slots(0, np.arange(n)), 0)
    step = 2.0 ** (int(c.ks[c.slots(0, 0) // 32, 0]) - 127)
    # one rounding to 4 bits, 2^-4 of the value, and where the value is below 2^-6 of the scale one to a
    # multiple of 2^-9 of each of the scales passed: less than 2^-9 of the last in all
    bound = np.abs(x[:, 0].double().numpy()) * 2.0 ** -4 + step * 2.0 ** -9
    assert (np.abs(got - x[:, 0].double().numpy()) <= bound).all()


# ---- eviction

def run_evict(c, weights, budget, sink, recent):
    print("evict lens %s budget %d sink %d recent %d %s page %d" % (c.lens, budget, sink, recent, c.form, c.page),
          flush=True)
    stay = max(1, min(budget, max(c.lens)))
    width = -(-stay // c.page)
    extra = len(c.lens) * width
    # pages behind the pool's own take what stays
    target = (c.pages + np.random.default_rng(1).permutation(extra)).astype(np.int32).reshape(len(c.lens), width)
    grow = lambda x, rows, fill: None if x is None else torch.cat(           # noqa: E731
        [x, torch.full((rows,) + tuple(x.shape[1:]), fill, dtype=x.dtype)])
    rows = extra * c.page
    c.k, c.v = grow(c.k, rows, 5), grow(c.v, rows, 6)
    if c.sb:
        c.ks, c.vs = grow(c.ks, rows // c.sb, 9), grow(c.vs, rows // c.sb, 9)
    kept, left, want = ref.evict(c, weights, target, budget, sink, recent)
    cache = on_gpu(c)
    p = params(c, c.hkv, [0], sink=sink, max_new=0)
    got, cu, w = fp2.cache_evict(p, cache, dev(weights), dev(cu_of(c.lens)), dev(c.table), dev(target),
                                 budget=budget, recent_tokens=recent, cu_seqlens_k_host=cu_of(c.lens))
    torch.cuda.synchronize()
    assert np.array_equal(got.cpu().numpy(), kept), "kept"
    assert np.array_equal(cu.cpu().numpy(), cu_of([min(n, budget) for n in c.lens]))
    assert np.array_equal(w.cpu().numpy(), left, equal_nan=True), "weights"
    for n, t in (("k", cache.k), ("v", cache.v), ("ks", cache.k_scale), ("vs", cache.v_scale)):
        if t is not None:
            same(t, want[n], n)


@pytest.mark.parametrize("form,page", [("bf16", 1), ("bf16", 16), ("head", 24), (16, 16), (32, 96), (64, 64),
                                       (128, 128)])
def test_evict(form, page):
    r = np.random.default_rng(5)
    for lens, budget, sink, recent in (([500, 90, 0, 200], 100, 4, 16), ([300, 301], 150, 0, 150),
                                       ([77], 1, 0, 0), ([77], 1, 1, 0), ([400], 333, 16, 0), ([20], 64, 4, 4)):
        c = ref.Cache(lens, 2, form, page, seed=4, spread=1.0)
        w = r.random((len(lens), 2, max(lens) + 3)).astype(np.float32) ** 4
        w[:, :, ::5] = 0.125                              # ties
        run_evict(c, w, budget, sink, recent)


@pytest.mark.parametrize("kind", ["equal", "zero", "nan", "inf", "signs", "close"])
def test_evict_order(kind):
    """Equal weights, zeros of both signs, NaN and infinities, and weights a bit apart; more tokens than a
    workgroup's threads take at a time."""
    L = 9000
    r = np.random.default_rng(6)
    w = r.random((1, 2, L)).astype(np.float32)
    if kind == "equal":
        w[:] = 0.5
    elif kind == "zero":
        w[:] = np.where(r.random(w.shape) < 0.5, 0.0, -0.0)
        w[0, 0, 100:120] = 1e-40
    elif kind == "nan":
        w[r.random(w.shape) < 0.6] = np.nan
    elif kind == "inf":
        w[r.random(w.shape) < 0.3] = np.inf
        w[r.random(w.shape) < 0.3] = -np.inf
    elif kind == "signs":
        w -= 0.5
    else:
        w = np.nextafter(np.float32(1), np.float32(2)) * np.ones_like(w)
        w[0, :, ::3] = 1.0
    run_evict(ref.Cache([L], 2, 64, 64, seed=5), w, 4501, 3, 700)


@pytest.mark.parametrize("batch,max_kv", [(0, 100), (2, 0)])
def test_calls_without_tokens(batch, max_kv):
    p = fp2.make_cache_params(batch=batch, num_q_heads=4, num_kv_heads=2, max_seq_len=0, max_kv_len=max_kv, page_size=16,
                              max_pages_per_seq=7)
    cache = fp2.alloc_cache(p, 2)
    cu, table = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros((2, 7), dtype=torch.int32, device="cuda")
    q, lse = torch.zeros((0, 4, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((0, 4), device="cuda")
    w = torch.full((2, 2, 100), 3.0, device="cuda")
    fp2.cache_append(p, q[:, :2].contiguous(), q[:, :2].contiguous(), cache, cu, cu, table)
    assert fp2.cache_attend(p, q, cache, cu, cu, table)[0].shape == q.shape
    got = fp2.cache_weights(p, q, lse, cache, cu, cu, table, weights_in=w)
    assert got.shape[0] == batch and bool((got == 3).all())
    assert bool((fp2.cache_weights(p, q, lse, cache, cu, cu, table) == 0).all())
    kept, cu2, w2 = fp2.cache_evict(p, cache, w, cu, table, table.clone(), budget=20)
    assert bool((kept == -1).all()) and cu2.tolist() == [0] * (batch + 1) and bool((w2 == 0).all())


@pytest.mark.parametrize("form", ["bf16", 64])
def test_more_sequences_than_lanes(form):
    """More sequences than a wave looks at at once, some without new tokens or without any."""
    r = np.random.default_rng(21)
    lens = [int(n) for n in r.integers(0, 60, 150)]
    new = [min(n, int(m)) for n, m in zip(lens, r.integers(0, 3, 150))]
    lens[70], new[70] = 2500, 2                        # the call's bound: sequences are cut
    run_attend(ref.Cache(lens, 2, form, 64, seed=22), 8, new)
    run_attend(ref.Cache(lens, 3, form, 64, seed=23), 3, new, window=40, sink=3)


@pytest.mark.parametrize("form,page", [("bf16", 1), ("bf16", 64), ("head", 24), (16, 64)])
def test_slots_past_32_bits(form, page):
    """The same calls on a small pool and at the end of one whose rows lie past 4 GiB."""
    hkv, hq = 8, 16
    row = hkv * 128 * (2 if form == "bf16" else 1)
    c = ref.Cache([300, 41], hkv, form, page, room=80, seed=24)
    spare = ref.Cache([100] * 2, hkv, form, page, seed=25)
    small = on_gpu(c)
    for n in ("k", "v") + (("ks", "vs") if c.sb else ()):
        name = {"ks": "k_scale", "vs": "v_scale"}.get(n, n)
        setattr(small, name, torch.cat([getattr(small, name), dev(getattr(spare, n))]))
    skip = -(-((1 << 32) + (1 << 30)) // row // page) * page        # slots before the copy
    pools = {}
    for n in ("k", "v"):
        t = getattr(small, n)
        pools[n] = torch.empty((skip + t.shape[0],) + t.shape[1:], dtype=t.dtype, device="cuda")
        pools[n][skip:] = t
    scales = [small.k_scale, small.v_scale]
    if c.sb:
        scales = [torch.cat([torch.full((skip // c.sb, hkv), 255, dtype=torch.uint8, device="cuda"), t]) for t in scales]
    large = fp2.KVCache(pools["k"], pools["v"], *scales)
    g = torch.Generator().manual_seed(8)
    w_shape = (2, hkv, 400)

    def run(cache, shift):
        g.manual_seed(8)
        got, w = [], torch.zeros(w_shape, device="cuda")
        lens = list(c.lens)
        table = np.where(c.table < 2 ** 30, c.table + shift, 0).astype(np.int32)
        for new in ([70, 3], [1, 1]):
            lens = [a + b for a, b in zip(lens, new)]
            p = params(c, hq, new, max_kv=max(lens))
            q, k, v = (torch.randn((sum(new), h, 128), generator=g).bfloat16().cuda() for h in (hq, hkv, hkv))
            args = (dev(cu_of(new)), dev(cu_of(lens)), dev(table))
            fp2.cache_append(p, k, v, cache, *args)
            out, lse = fp2.cache_attend(p, q, cache, *args, want_lse=True)
            fp2.cache_weights(p, q, lse, cache, *args, weights=w, weights_in=w)
            got += [out, lse]
        target = (spare.table + c.pages + shift).astype(np.int32)
        got += fp2.cache_evict(p, cache, w, args[1], args[2], dev(target), budget=100, recent_tokens=20)
        p = params(c, hq, [1, 1], max_kv=100)
        p.max_pages_per_seq = target.shape[1]
        got.append(fp2.cache_attend(p, q, cache, args[0], dev(cu_of([100, 45])), dev(target))[0])
        torch.cuda.synchronize()
        return got + [w]

    for a, b in zip(run(small, 0), run(large, skip // page)):
        same(b, a.cpu(), "results")
    same(large.k[skip:], small.k.cpu(), "k")
    same(large.v[skip:], small.v.cpu(), "v")


def test_two_calls_at_once():
    """Calls on two streams, each with a workspace of its own, against the same calls one after the other."""
    c = ref.Cache([3000, 2000], 2, 64, 64, seed=26)
    cache, table, cuk = on_gpu(c), dev(c.table), dev(cu_of(c.lens))
    g = torch.Generator().manual_seed(9)
    calls = []
    for new in ([1, 1], [100, 70]):
        p = params(c, 8, new)
        calls.append((p, torch.randn((sum(new), 8, 128), generator=g).bfloat16().cuda(), dev(cu_of(new)),
                      fp2.alloc_cache_workspace(p)))
    torch.cuda.synchronize()
    want = [fp2.cache_attend(p, q, cache, cu, cuk, table, workspace=ws, want_lse=True) for p, q, cu, ws in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(3):
        got = [fp2.cache_attend(p, q, cache, cu, cuk, table, workspace=ws, want_lse=True, stream=s)
               for (p, q, cu, ws), s in zip(calls, streams)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ---- together

@pytest.mark.parametrize("form", ["bf16", "head", 16])
def test_captured_steps(form):
    """Decode steps captured once and replayed while the lengths grow on the device: append, attention and
    weights of each replay against the eager calls."""
    lens, steps = [70, 500, 3], 4
    base = ref.Cache(lens, 2, form, 16, room=steps, seed=14)
    g = torch.Generator().manual_seed(3)
    q = torch.randn((steps, 3, 8, 128), generator=g).bfloat16().cuda()
    kv = torch.randn((2, steps, 3, 2, 128), generator=g).bfloat16().cuda()
    p = params(base, 8, [1], max_kv=max(lens) + steps)
    table, cu = dev(base.table), dev(cu_of([1] * 3))
    ws = fp2.alloc_cache_workspace(p)

    def step(cache, qs, ks, vs, cuk, w):
        fp2.cache_append(p, ks, vs, cache, cu, cuk, table)
        out, lse = fp2.cache_attend(p, qs, cache, cu, cuk, table, want_lse=True, workspace=ws)
        fp2.cache_weights(p, qs, lse, cache, cu, cuk, table, weights=w, weights_in=w)
        return out

    def cuk_at(t):
        return dev(cu_of([n + t + 1 for n in lens]))

    w_shape = (3, 2, max(lens) + steps)
    eager, ew, want = on_gpu(base), torch.zeros(w_shape, device="cuda"), []
    for t in range(steps):
        want.append(step(eager, q[t], kv[0, t], kv[1, t], cuk_at(t), ew).clone())
    cache, w = on_gpu(base), torch.zeros(w_shape, device="cuda")
    sq, sk, sv, scu = q[0].clone(), kv[0, 0].clone(), kv[1, 0].clone(), cuk_at(0)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = step(cache, sq, sk, sv, scu, w)
    for t in range(steps):
        sq.copy_(q[t]), sk.copy_(kv[0, t]), sv.copy_(kv[1, t]), scu.copy_(cuk_at(t))
        graph.replay()
        float(torch.randn(1 << 18, device="cuda").sum())
        torch.cuda.synchronize()
        assert torch.equal(got, want[t]), "step %d" % t
    assert torch.equal(w, ew)
    same(cache.k, eager.k.cpu(), "k")


def test_other_stream():
    c = ref.Cache([400, 90], 2, 64, 64, seed=15)
    q = torch.randn((2, 8, 128), generator=torch.Generator().manual_seed(1)).bfloat16()
    p = params(c, 8, [1, 1])
    cache, args = on_gpu(c), (dev(cu_of([1, 1])), dev(cu_of(c.lens)), dev(c.table))
    qd = dev(q)
    want, _ = fp2.cache_attend(p, qd, cache, *args)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    out = torch.zeros_like(want)
    torch.cuda.synchronize()
    fp2.cache_attend(p, qd, cache, *args, out=out, stream=s)
    s.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("form,window", [("bf16", 0), (16, 200), (64, 0)])
def test_a_request_from_prompt_to_eviction(form, window):
    """Prompts are appended, attended and weighed, the caches cut, and the sequences go on decoding; each
    step against the definition on the cache as it is."""
    hkv, hq, page, budget, sink, recent = 2, 8, 64, 128, 4, 32
    new = [260, 71]
    lens = [0, 0]
    c = ref.Cache(lens, hkv, form, page, room=400, seed=16)
    spare = ref.Cache([budget + 20] * 2, hkv, form, page, seed=17)
    target = spare.table + c.pages
    c.k, c.v = torch.cat([c.k, spare.k]), torch.cat([c.v, spare.v])
    if c.sb:
        c.ks, c.vs = torch.cat([c.ks, spare.ks]), torch.cat([c.vs, spare.vs])
    cache = on_gpu(c)
    g = torch.Generator().manual_seed(5)
    stride = 512
    weights = torch.zeros((2, hkv, stride), device="cuda")

    def forward(new):
        x = [torch.randn((sum(new), h, 128), generator=g).bfloat16() for h in (hq, hkv, hkv)]
        c.lens = [a + b for a, b in zip(c.lens, new)]
        p = params(c, hq, new, window, sink, max_kv=stride if c.width * page >= stride else c.width * page)
        args = (dev(cu_of(new)), dev(cu_of(c.lens)), dev(c.table))
        fp2.cache_append(p, dev(x[1]), dev(x[2]), cache, *args)
        out, lse = fp2.cache_attend(p, dev(x[0]), cache, *args, want_lse=True)
        fp2.cache_weights(p, dev(x[0]), lse, cache, *args, weights=weights, weights_in=weights)
        torch.cuda.synchronize()
        c.k, c.v = cache.k.cpu(), cache.v.cpu()
        if c.sb:
            c.ks, c.vs = cache.k_scale.cpu(), cache.v_scale.cpu()
        o, tol, z, ztol, w = ref.attend(c, x[0], new, window, sink, lse_in=lse.double().cpu().numpy())
        close(out, o, tol, "out")
        return w

    total = [np.zeros((2, hkv, stride)) for _ in new]
    for step in (new, [1, 1], [2, 1]):
        for b, w in enumerate(forward(step)):
            total[b][:, :, :w.shape[2]] += w
    for b in range(2):
        close(weights[b], total[b][0], total[b][1] + 4 * ref.U32 * total[b][0] + 1e-30, "weights")
    p = params(c, hq, [1], window, sink)
    kept, cu, weights = fp2.cache_evict(p, cache, weights, dev(cu_of(c.lens)), dev(c.table), dev(target),
                                        budget=budget, recent_tokens=recent)
    _, _, pools = ref.evict(c, weights_that_keep(kept, total, c, budget, sink, recent), target, budget, sink, recent)
    same(cache.k, pools["k"], "k")
    c.table, c.width = target, target.shape[1]
    c.lens = [min(n, budget) for n in c.lens]
    assert cu.cpu().tolist() == cu_of(c.lens).tolist()
    c.k, c.v = cache.k.cpu(), cache.v.cpu()
    for step in ([1, 1], [3, 1]):
        forward(step)


def weights_that_keep(kept, total, c, budget, sink, recent):
    """Weights that lead to `kept`: one for what was kept, zero for the rest. A token with clearly more
    weight than another was not dropped for it."""
    k = kept.cpu().numpy()
    w = np.zeros((len(c.lens), c.hkv, total[0].shape[2]), np.float32)
    for b, n in enumerate(c.lens):
        for h in range(c.hkv):
            w[b, h, k[b, h][k[b, h] >= 0]] = 1
            ranked = np.arange(sink, n - recent)
            stay, go = ranked[w[b, h, ranked] > 0], ranked[w[b, h, ranked] == 0]
            if n > budget and len(go):
                x, tol = total[b][0, h], total[b][1, h] + 4 * ref.U32 * total[b][0, h]
                assert (x[go] - tol[go]).max() <= (x[stay] + tol[stay]).min()
    return w

"""Rotary positions on the GPU against their definition in 64 bits (tests/positions_ref.py):
queries and keys by themselves, on the way into the cache, read back, and moved."""
import numpy as np
import pytest
import torch

import paper_2608_19758_amd as fp2
from tests import cache_ref as ref
from tests import positions_ref as pos_ref
from tests.test_gpu_cache import cu_of, dev, on_gpu, params, same

pytestmark = pytest.mark.gpu

FORMS = ["bf16", "head", 16, 64]
KINDS = [(128, False), (128, True), (64, False), (96, True), (100, False), (2, False), (2, True), (126, True), (16, False),
         (126, False), (20, False)]


def rotary_of(dim, interleaved, scaling="none", factor=1.0, **kw):
    r = fp2.make_rotary(dim, interleaved=interleaved, scaling=scaling, factor=factor, original_len=4096, **kw)
    f, a = fp2.rotary_frequencies(dim, scaling=scaling, factor=factor, original_len=4096)
    return r, f, a


def rows(n, heads, seed=0, spread=1.0):
    g = np.random.default_rng(seed)
    x = g.standard_normal((n, heads, 128)) * np.exp(spread * g.standard_normal((n, heads, 1)))
    return torch.from_numpy(x).bfloat16()


def packed(q, k, v, extra=8):
    """Views of one matrix [tokens, (Hq + 2 Hkv) 128 + extra] that holds them."""
    n = q.shape[0]
    m = torch.cat([q.reshape(n, -1), k.reshape(n, -1), v.reshape(n, -1), torch.zeros(n, extra, dtype=q.dtype)], 1).cuda()
    at = np.cumsum([0, q.shape[1] * 128, k.shape[1] * 128, v.shape[1] * 128])
    return [m[:, a:z].view(n, -1, 128) for a, z in zip(at[:-1], at[1:])]


@pytest.mark.parametrize("dim,interleaved", KINDS)
@pytest.mark.parametrize("tokens", [1, 7, 65, 300])
def test_rotary(dim, interleaved, tokens):
    print("rotary dim %d interleaved %s tokens %d" % (dim, interleaved, tokens), flush=True)
    r, f, a = rotary_of(dim, interleaved, "ramp" if dim > 16 else "none", 8.0 if dim > 16 else 1.0)
    q, k, v = rows(tokens, 6, 1), rows(tokens, 2, 2), rows(tokens, 2, 3)
    at = np.random.default_rng(4).integers(0, 2 ** 20, tokens).astype(np.int32)
    at[0] = 0
    pq, pk, _ = packed(q, k, v)
    for x, y in ((dev(q), dev(k)), (pq, pk)):
        qo, ko = fp2.rotary(r, x, dev(at), y)
        want, err = pos_ref.turn(q.double().numpy(), np.repeat(at[:, None], 6, 1), f, interleaved, a)
        pos_ref.check_bf16(qo, want, err, "q")
        want, err = pos_ref.turn(k.double().numpy(), np.repeat(at[:, None], 2, 1), f, interleaved, a)
        pos_ref.check_bf16(ko, want, err, "k")
    same(fp2.rotary(r, dev(q), dev(at)), qo.cpu(), "q alone")
    # in place, in a part of a wider matrix; what lies beside it stays
    beside = pk.clone()
    assert fp2.rotary(r, pq, dev(at), out=pq) is pq
    same(pq, qo.cpu(), "in place")
    same(pk, beside.cpu(), "beside")
    # into rows that are longer and more
    wide = torch.full((tokens + 2, 9, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    fp2.rotary(r, dev(q), dev(at), out=wide[:, 1:7])
    same(wide[:tokens, 1:7], qo.cpu(), "wide")
    assert bool((wide[tokens:] == 7).all()) and bool((wide[:, 0] == 7).all()) and bool((wide[:, 7:] == 7).all())


@pytest.mark.parametrize("dim,interleaved", KINDS)
def test_rotary_codes_and_inverse(dim, interleaved):
    r, f, a = rotary_of(dim, interleaved, scale=1.25)
    a = 1.25
    q = rows(77, 4, 5)
    at = np.arange(1000, 1077).astype(np.int32)
    every = np.repeat(at[:, None], 4, 1)
    scale = (q.double().abs().amax((0, 2)) * 1.3 / 448).float()      # some turned values are past 448
    codes = fp2.rotary(r, dev(q), dev(at), q_scale=dev(scale))
    assert codes.dtype == torch.uint8
    want, err = pos_ref.turn(q.double().numpy(), every, f, interleaved, a)
    by = scale.double().numpy()[None, :, None]
    pos_ref.check_codes(codes, want / by, err / by + np.abs(want / by) * pos_ref.U, "codes")
    y = fp2.rotary(r, dev(q), dev(at))
    back = fp2.rotary(r, y, dev(at), inverse=True)
    want, err = pos_ref.turn(y.double().cpu().numpy(), every, f, interleaved, a, back=True)
    pos_ref.check_bf16(back, want, err, "back")


def test_far_positions():
    """Angles are exact at any position: the ends of 32 bits, negative ones."""
    for interleaved in (False, True):
        r, f, _ = rotary_of(128, interleaved)
        at = np.array([0, 1, -1, 2 ** 20, -2 ** 20, 2 ** 31 - 1, -2 ** 31, 123456789], np.int32)
        q = rows(len(at), 2, 6)
        want, err = pos_ref.turn(q.double().numpy(), np.repeat(at[:, None].astype(np.int64), 2, 1), f, interleaved)
        pos_ref.check_bf16(fp2.rotary(r, dev(q), dev(at)), want, err, "far")


@pytest.mark.parametrize("dim,interleaved", [(64, False), (64, True), (100, False)])
def test_odd_values_stay_in_their_pair(dim, interleaved):
    r, f, _ = rotary_of(dim, interleaved)
    q = rows(9, 2, 7)
    q[0, 0, 3], q[1, 1, dim - 1], q[2, 0, 127], q[3, 1, dim] = float("inf"), float("nan"), float("-inf"), float("nan")
    at = np.arange(1, 10, dtype=np.int32)
    want, err = pos_ref.turn(q.double().numpy(), np.repeat(at[:, None], 2, 1), f, interleaved)
    pos_ref.check_bf16(fp2.rotary(r, dev(q), dev(at)), want, np.nan_to_num(err, nan=0.0, posinf=0.0), "odd values")
    assert np.isnan(want).sum() + np.isinf(want).sum() == 6


def test_no_tokens_and_one_head():
    r, f, _ = rotary_of(128, False)
    empty = torch.empty((0, 4, 128), dtype=torch.bfloat16, device="cuda")
    assert fp2.rotary(r, empty, torch.empty(0, dtype=torch.int32, device="cuda")).shape == (0, 4, 128)
    q = rows(5, 1, 8)
    at = np.arange(5, dtype=np.int32)
    want, err = pos_ref.turn(q.double().numpy(), at[:, None], f, False)
    pos_ref.check_bf16(fp2.rotary(r, dev(q), dev(at)), want, err, "one head")


# ---- on the way into the cache

def run_append(lens, new, form, page, dim=128, interleaved=False, hq=4, hkv=2, at=None, codes=False, seed=1, part=True,
               spread=1.0):
    print("append_rotary lens %s new %s %s page %d dim %d interleaved %s" % (lens, new, form, page, dim, interleaved),
          flush=True)
    r, f, a = rotary_of(dim, interleaved, "ramp" if dim > 16 else "none", 4.0 if dim > 16 else 1.0)
    c = ref.Cache(lens, hkv, form, page, seed=seed, spread=spread)
    n = sum(new)
    q, k, v = rows(n, hq, seed + 1), rows(n, hkv, seed + 2), rows(n, hkv, seed + 3)
    index = np.concatenate([np.arange(L - m, L) for m, L in zip(new, lens)]).astype(np.int32)
    where = index if at is None else (index + at).astype(np.int32)
    pad = 3
    grow = lambda x: torch.cat([x, rows(pad, x.shape[1], 99)])      # noqa: E731
    pq, pk, pv = packed(grow(q), grow(k), grow(v)) if part else (dev(grow(q)), dev(grow(k)), dev(grow(v)))
    p = params(c, hq, new)
    cu, cuk = cu_of(new), cu_of(lens)
    cache = on_gpu(c)
    scale = (q.double().abs().amax((0, 2)) * a * 1.5 / 448).float() if codes else None
    out = torch.full((n + pad, hq, 128), 7, dtype=torch.uint8 if codes else torch.bfloat16, device="cuda")
    positions = None if at is None else torch.cat([torch.from_numpy(where), torch.zeros(pad, dtype=torch.int32)]).cuda()
    got = fp2.cache_append_rotary(p, r, pq, pk, pv, cache, dev(cu), dev(cuk), dev(c.table), positions=positions,
                                  out=out, q_scale=dev(scale), cu_seqlens_host=cu, cu_seqlens_k_host=cuk)
    assert got is out and bool((out[n:] == 7).all())
    # queries: as by themselves
    same(out[:n], fp2.rotary(r, dev(q), dev(where), q_scale=dev(scale)).cpu(), "q")
    # values: as the append without positions leaves them
    plain = ref.append(c, k, v, new)
    same(cache.v, plain["v"], "v")
    if plain["vs"] is not None:
        same(cache.v_scale, plain["vs"], "v scales")
    # keys
    want, err = pos_ref.turn(k.double().numpy(), np.repeat(where[:, None], hkv, 1), f, interleaved, a)
    left = cache.k.cpu().clone()
    row = 0
    for b, (m, L) in enumerate(zip(new, lens)):
        slots = c.slots(b, np.arange(L - m, L))
        if form == "bf16":
            pos_ref.check_bf16(cache.k[slots], want[row:row + m], err[row:row + m], "k of %d" % b)
        elif form == "head":
            by = c.ks.double().numpy()[None, :, None]
            w, e = want[row:row + m] / by, err[row:row + m] / by
            pos_ref.check_codes(cache.k[slots], w, e + np.abs(w) * pos_ref.U, "k of %d" % b)
        else:
            for t0 in range((L - m) // c.sb * c.sb, L, c.sb) if m else ():
                first, last = max(t0, L - m), min(t0 + c.sb, L)
                sl = slice(row + first - (L - m), row + last - (L - m))
                to, old = c.slots(b, np.arange(first, last)), c.slots(b, np.arange(t0, first))
                for h in range(hkv):
                    byte = int(cache.k_scale[to[0] // c.sb, h])
                    was = int(c.ks[to[0] // c.sb, h]) - 127 if t0 < L - m else -100
                    pos_ref.check_block(cache.k[to, h], byte, want[sl, h], err[sl, h], "k of %d at %d" % (b, t0), least=was)
                    if t0 < L - m and byte - 127 == was:
                        assert torch.equal(cache.k[old, h].cpu(), c.k[old, h])
                    elif t0 < L - m:
                        x = ref.VALUES[c.k[old, h].numpy()] * 2.0 ** (was - (byte - 127))
                        same(cache.k[old, h], torch.from_numpy(ref.to_codes(x)), "old codes")
                left[old] = c.k[old]
        left[slots] = c.k[slots]
        row += m
    same(left, c.k, "slots of no new token")
    return c, cache, out


@pytest.mark.parametrize("form", FORMS + [32, 128])
@pytest.mark.parametrize("dim,interleaved", [(128, False), (128, True), (64, False), (100, False), (20, False), (126, False)])
def test_append(form, dim, interleaved):
    page = 128 if form == 128 else 64
    run_append([1, 63, 200, 5, 300, 4], [1, 40, 200, 0, 129, 3], form, page, dim, interleaved)
    run_append([1, 64, 65, 200, 9, 7], [1, 1, 2, 16, 9, 0], form, page, dim, interleaved, seed=5)


@pytest.mark.parametrize("form", FORMS + [32, 128])
@pytest.mark.parametrize("dim,interleaved", [(128, True), (64, False), (100, False)])
def test_append_some_tokens(form, dim, interleaved):
    """As many new tokens as a wave may take alone, in up to three blocks, and one more."""
    page = 128 if form == 128 else 64
    run_append([32, 70, 127, 25, 400, 30], [32, 31, 17, 20, 32, 1], form, page, dim, interleaved, seed=6)
    run_append([41, 33, 150], [32, 33, 22], form, page, dim, interleaved, seed=7)


@pytest.mark.parametrize("form", FORMS + [32, 128])
@pytest.mark.parametrize("dim,interleaved", [(128, True), (128, False), (64, False), (100, False), (2, False)])
def test_append_one_token(form, dim, interleaved):
    """A decode step: blocks that the token starts, blocks whose scale it raises and others, idle sequences."""
    page = 128 if form == 128 else 64
    lens, new = [1, 16, 17, 64, 65, 200, 128, 9, 30, 127], [1, 1, 1, 1, 1, 1, 1, 0, 1, 1]
    run_append(lens, new, form, page, dim, interleaved, seed=8)
    run_append(lens, new, form, page, dim, interleaved, hq=36, hkv=9, seed=9, codes=True, part=False, spread=2.0)
    run_append(lens, new, form, page, dim, interleaved, hq=8, hkv=8, seed=10, at=70000, spread=0.1)


@pytest.mark.parametrize("form", FORMS + [32, 128])
@pytest.mark.parametrize("most", [2, 3, 4, 5, 8])
def test_append_drafted_tokens(form, most):
    """Up to two, four and eight new tokens: in one block, in two, behind codes that are held and not."""
    page = 128 if form == 128 else 64
    new = [most, most, 1, most, most - 1, 0, most, most, 2, most]
    lens = [most, 16 + most, 17, 64 + most // 2, 130, 20, 128, 66, 2, 48 + most - 1]
    for dim, interleaved in ((128, False), (96, True), (100, False)):
        run_append(lens, new, form, page, dim, interleaved, hq=12, hkv=3, seed=20 + most)
        run_append(lens, new, form, page, dim, interleaved, hq=8, hkv=8, seed=30 + most, codes=True, part=False, spread=2.5)


@pytest.mark.parametrize("sb", [16, 64])
def test_append_one_token_after_the_other(sb):
    """40 steps of one token: each block's codes have been rounded to its scale at most once for each growth, and
    infinities and NaN of a head stay with their pairs and move no scale."""
    r, f, _ = rotary_of(128, False)
    heads, n, start = 3, 40, 50
    c = ref.Cache([start + n], heads, sb, 64, seed=14)
    k, v = rows(n, heads, 15), rows(n, heads, 16)
    k *= torch.linspace(0.25, 4.0, n)[:, None, None].bfloat16()
    k[5, 0, 3], k[6, 1, 70], k[7, 2, 0] = float("inf"), float("nan"), float("-inf")
    one, many = on_gpu(c), on_gpu(c)
    was, roundings = one.k_scale.cpu(), 2
    for i in range(n):
        cuk = cu_of([start + i + 1])
        fp2.cache_append_rotary(params(c, heads, [1]), r, None, dev(k[i:i + 1]), dev(v[i:i + 1]), one, dev(cu_of([1])), dev(cuk),
                                dev(c.table))
        now = one.k_scale.cpu()
        roundings, was = roundings + (now != was).numpy(), now
    fp2.cache_append_rotary(params(c, heads, [n]), r, None, dev(k), dev(v), many, dev(cu_of([n])), dev(cu_of(c.lens)), dev(c.table))
    same(one.k_scale, many.k_scale.cpu(), "k scales")
    same(one.v_scale, many.v_scale.cpu(), "v scales")
    at = c.slots(0, np.arange(start, start + n))
    scale = many.k_scale.cpu().numpy()[at // sb].astype(np.float64)
    a, b = (ref.VALUES[x.k.cpu().numpy()[at]] * 2.0 ** (scale - 127)[..., None] for x in (one, many))
    assert np.array_equal(np.isnan(a), np.isnan(b)) and np.isnan(a).sum() == 6
    # both round once, and each growth what is there once more, by at most half a step: 2^-4 of it, or 2^-10 scales
    x, y = np.nan_to_num(a), np.nan_to_num(b)
    bound = roundings[at // sb][..., None] * (np.abs(y) * 2.0 ** -4 + 2.0 ** -10 * 2.0 ** (scale - 127)[..., None])
    assert (np.abs(x - y) <= bound).all()


@pytest.mark.parametrize("form", FORMS)
def test_append_positions_codes_and_plain_rows(form):
    run_append([400, 37], [150, 37], form, 64, at=100000, codes=True, part=False)
    run_append([400, 37], [1, 3], form, 64, at=-50, codes=True, part=False)


@pytest.mark.parametrize("form,page", [("bf16", 1), ("head", 5), ("bf16", 24), (16, 48), (64, 192)])
def test_append_pages(form, page):
    run_append([333, 97], [200, 97], form, page)
    run_append([333, 97], [2, 16], form, page)


def test_append_without_queries_matches_both_calls():
    """Keys without queries, and that a bf16 cache holds what rotary and append leave one after the other."""
    r, _, _ = rotary_of(128, False)
    c = ref.Cache([150, 20], 2, "bf16", 16, seed=9)
    new = [100, 20]
    k, v = rows(120, 2, 10), rows(120, 2, 11)
    cu, cuk = cu_of(new), cu_of(c.lens)
    p, one, two = params(c, 4, new), on_gpu(c), on_gpu(c)
    args = (dev(cu), dev(cuk), dev(c.table))
    assert fp2.cache_append_rotary(p, r, None, dev(k), dev(v), one, *args) is None
    at = np.concatenate([np.arange(50, 150), np.arange(20)]).astype(np.int32)
    fp2.cache_append(p, fp2.rotary(r, dev(k), dev(at)), dev(v), two, *args)
    same(one.k, two.k.cpu(), "k")
    same(one.v, two.v.cpu(), "v")


def test_append_odd_values():
    """Infinities and NaN become the NaN code, with their pair, and do not move the block's scale."""
    r, f, _ = rotary_of(128, False)
    for new in ([40], [3]):
        c = ref.Cache([40], 1, 16, 16, seed=12)
        n = new[0]
        k, v = rows(n, 1, 13), rows(n, 1, 14)
        k[1, 0, 5], k[2, 0, 70] = float("inf"), float("nan")
        cu, cuk = cu_of(new), cu_of(c.lens)
        cache = on_gpu(c)
        fp2.cache_append_rotary(params(c, 1, new), r, None, dev(k), dev(v), cache, dev(cu), dev(cuk), dev(c.table))
        want, err = pos_ref.turn(k.double().numpy()[:, 0], np.arange(40 - n, 40), f, False)
        err = np.nan_to_num(err, nan=0.0, posinf=0.0)
        for t0 in range((40 - n) // 16 * 16, 40, 16):
            a, z = max(t0, 40 - n), min(t0 + 16, 40)
            at = c.slots(0, np.arange(a, z))
            was = int(c.ks[at[0] // 16, 0]) - 127 if t0 < 40 - n else -100
            pos_ref.check_block(cache.k[at, 0], cache.k_scale[at[0] // 16, 0], want[a - 40 + n:z - 40 + n],
                                err[a - 40 + n:z - 40 + n], "k", least=was)


# ---- read back

@pytest.mark.parametrize("form,page", [("bf16", 16), ("bf16", 1), ("head", 24), (16, 48), (64, 64), (128, 256), (32, 32)])
def test_read(form, page):
    c = ref.Cache([1, 33, 200, 64, 7], 3, form, page, seed=15, spread=1.0)
    new = [1, 33, 77, 0, 5]
    print("read %s page %d" % (form, page), flush=True)
    cu, cuk = cu_of(new), cu_of(c.lens)
    p, cache, n = params(c, 3, new), on_gpu(c), sum(new)
    args = (dev(cu), dev(cuk), dev(c.table))
    k, v = fp2.cache_read(p, cache, *args, cu_seqlens_host=cu, cu_seqlens_k_host=cuk)
    slots = np.concatenate([c.slots(b, np.arange(L - m, L)) for b, (m, L) in enumerate(zip(new, c.lens))])
    index = np.concatenate([np.arange(L - m, L) for m, L in zip(new, c.lens)]).astype(np.int32)
    wk, wv = (np.stack([c.values(x, slots, h) for h in range(3)], 1) for x in "kv")
    # codes times an fp32 scale: the product rounded to fp32, then to bf16
    pos_ref.check_bf16(k, wk, np.abs(wk) * pos_ref.U, "k")
    pos_ref.check_bf16(v, wv, np.abs(wv) * pos_ref.U, "v")
    if form != "head":
        same(v, torch.from_numpy(wv).bfloat16(), "v exactly")
    for dim, interleaved in KINDS:
        r, f, a = rotary_of(dim, interleaved, "ramp" if dim > 16 else "none", 4.0 if dim > 16 else 1.0)
        for at in (None, index - 1000):
            out = torch.full((n + 2, 3, 128), 7.0, dtype=torch.bfloat16, device="cuda")
            pos = None if at is None else torch.cat([torch.from_numpy(at), torch.zeros(2, dtype=torch.int32)]).cuda()
            got, none = fp2.cache_read(p, cache, *args, rotary=r, positions=pos, values=False, k_out=out)
            assert none is None and got is out and bool((out[n:] == 7).all())
            where = index if at is None else at
            want, err = pos_ref.turn(wk, np.repeat(where[:, None], 3, 1), f, interleaved, a, back=True)
            # the scale's product is off by U of each, before the turn
            pos_ref.check_bf16(got[:n], want, err * 1.2, "k turned back")
    none, only = fp2.cache_read(p, cache, *args, keys=False, rows=n)
    assert none is None
    same(only, v.cpu(), "values alone")


# ---- move

def run_move(form, page, kind, dim=128, interleaved=False, in_place=False, seed=16, lens=(1, 33, 130, 0, 64)):
    print("move %s page %d %s dim %d interleaved %s in place %s" % (form, page, kind, dim, interleaved, in_place), flush=True)
    lens, hkv = list(lens), 2
    c = ref.Cache(lens, hkv, form, page, seed=seed, spread=1.0)
    g = np.random.default_rng(seed)
    r, f, _ = rotary_of(dim, interleaved, "ramp" if dim > 16 else "none", 4.0 if dim > 16 else 1.0)
    most = max(lens)
    if kind == "copy":
        moves = None
    elif kind == "one":
        moves = g.integers(-5000, 5000, len(lens)).astype(np.int32)
    elif kind == "heads":
        moves = g.integers(-5000, 5000, (len(lens), hkv, 1)).astype(np.int32)
    elif kind == "tokens":
        moves = g.integers(-5000, 5000, (1, 1, most)).astype(np.int32)
    else:
        moves = g.integers(-100, 100000, (len(lens), hkv, most + 3)).astype(np.int32)
    # a pool twice as large: the targets are its second half's pages
    cache = on_gpu(c)
    grow = lambda x: None if x is None or x.dim() == 1 else torch.cat([x, x.new_full(x.shape, 0x7f if x.dtype == torch.uint8 else float("nan"))])     # noqa: E731
    cache = fp2.KVCache(*(grow(x) if n < 2 or c.sb else x for n, x in enumerate((cache.k, cache.v, cache.k_scale, cache.v_scale))))
    before = [None if x is None else x.cpu().clone() for x in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    target = c.table if in_place else np.where(c.table == 2 ** 30, 2 ** 30, c.pages + c.table[:, :]).astype(np.int32)
    p, cuk = params(c, 2, [1] * len(lens), max_new=1), cu_of(lens)
    fp2.cache_move(p, cache, dev(cuk), dev(c.table), None if in_place else dev(target), rotary=None if moves is None else r,
                   moves=dev(moves), cu_seqlens_k_host=cuk)
    after = [None if x is None else x.cpu() for x in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    left = [None if x is None else x.clone() for x in after]
    for b, L in enumerate(lens):
        src, to = c.slots(b, np.arange(L)), c.slots(b, np.arange(L), target)
        blocks = np.unique(to // c.sb) if c.sb else None
        by = None
        if moves is not None:
            m = moves[:, None, None] if moves.ndim == 1 else moves
            by = np.broadcast_to(m[b % m.shape[0]][..., :L] if m.shape[2] > 1 else m[b % m.shape[0]], (hkv, L))
        for h in range(hkv):
            if not in_place:
                assert torch.equal(after[1][to, h].view(torch.uint8 if c.form != "bf16" else torch.int16),
                                   before[1][src, h].view(torch.uint8 if c.form != "bf16" else torch.int16)), "v"
                if c.sb:
                    assert torch.equal(after[3][to // c.sb, h], before[3][src // c.sb, h]), "v scales"
            if by is None:
                assert torch.equal(after[0][to, h].view(torch.uint8 if c.form != "bf16" else torch.int16),
                                   before[0][src, h].view(torch.uint8 if c.form != "bf16" else torch.int16)), "k"
                if c.sb:
                    assert torch.equal(after[2][to // c.sb, h], before[2][src // c.sb, h]), "k scales"
                continue
            x = ref.VALUES[before[0][src, h].numpy()] if c.form == "head" else c.values("k", src, h)
            want, err = pos_ref.turn(x, by[h], f, interleaved)
            if c.form == "bf16":
                pos_ref.check_bf16(after[0][to, h], want, err, "k")
            elif c.form == "head":
                pos_ref.check_codes(after[0][to, h], want, err, "k")
            else:
                for t0 in range(0, L, c.sb):
                    sl = slice(t0, min(t0 + c.sb, L))
                    pos_ref.check_block(after[0][to[sl], h], after[2][to[t0] // c.sb, h], want[sl], err[sl], "k at %d" % t0)
        for i in (0, 1):
            left[i][to] = before[i][to]
        if c.sb and L:
            for i in (2, 3):
                left[i][blocks] = before[i][blocks]
    for i, name in enumerate(("k", "v", "k scales", "v scales")):
        if left[i] is not None and left[i].dim() > 1:
            same(left[i], before[i], name + " of other slots")
    if in_place:
        same(after[1], before[1], "v in place")


@pytest.mark.parametrize("form,page", [("bf16", 16), ("head", 24), (16, 48), (32, 32), (64, 64), (128, 128)])
@pytest.mark.parametrize("kind", ["copy", "one", "heads", "tokens", "each"])
def test_move(form, page, kind):
    run_move(form, page, kind)
    if kind != "copy":
        run_move(form, page, kind, in_place=True)


@pytest.mark.parametrize("dim,interleaved", KINDS[1:])
@pytest.mark.parametrize("form", ["bf16", "head", 16])
def test_move_dims(dim, interleaved, form):
    run_move(form, 16, "each", dim, interleaved, in_place=True)
    run_move(form, 16, "one", dim, interleaved)


def test_move_of_nothing_changes_nothing():
    """Turned by 0 positions: rows, codes and the scales that their values need stay."""
    for form in FORMS:
        c = ref.Cache([100], 2, form, 64, seed=17)
        r, _, _ = rotary_of(128, False)
        cache = on_gpu(c)
        before = cache.k.cpu().clone()
        fp2.cache_move(params(c, 2, [1]), cache, dev(cu_of(c.lens)), dev(c.table), rotary=r,
                       moves=torch.zeros(1, dtype=torch.int32, device="cuda"))
        if c.sb:     # (scales may shrink to what the values need, exactly)
            want = np.stack([c.values("k", c.slots(0, np.arange(100)), h) for h in range(2)], 1)
            s = cache.k_scale.cpu().double().numpy()
            got = ref.VALUES[cache.k.cpu()[c.slots(0, np.arange(100))].numpy()] * \
                2.0 ** (s[c.slots(0, np.arange(100)) // c.sb][:, :, None] - 127)
            assert np.array_equal(got, want)
        else:
            same(cache.k, before, form)

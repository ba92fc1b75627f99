"""The operators of the paged KV cache whose speed is measured: appending to it,
attention over it, the attention weight its tokens received, and eviction.

Every case is one layer's call as a serving engine makes it between two
matrix products of a model, on a paged pool of keys and values in bf16, in
e4m3 codes with one fp32 scale per head, or in e4m3 codes with one
power-of-two scale per block of ``scale`` tokens and head.

* append:  the new tokens' keys and values go into the pages, in its type. A
  block's scale is 2^e, e = ceil(log2(amax / 448)) of its tokens; it never
  falls, and codes that were there are rounded again where it grows.
* attend:  O = softmax(scale * Q K^T) V of the last tokens of each sequence,
  causal, over the first ``sink`` tokens and the last ``window`` ones (all
  where window is 0).
* weights: what each cached token received of the queries' probabilities,
  summed over the queries and over the heads that share its keys.
* evict:   the ``budget`` tokens of each sequence and KV head that stay: the
  first ``sink``, the last ``recent`` and the heaviest of the others. Their
  keys, values and weights are laid out one after the other in other pages.

``own`` chooses between the plain form and the framework's calls.
"""
import math

import numpy as np
import torch

own = False

D = 128


def _case(name, op, new, prefix, **kw):
    c = dict(name=name, op=op, new=new, prefix=prefix, hq=32, hkv=8, cache="fp8", scale=64, page=64,
             window=0, sink=0, lse=False, budget=0, recent=0)
    c.update(kw)
    return c


def _spread(seed, n, lo, hi):
    """n lengths spread over the logarithm of [lo, hi], as texts."""
    r = np.random.default_rng(seed)
    return ",".join(str(int(x)) for x in np.exp(r.uniform(math.log(lo), math.log(hi), n)))


def _ones(n):
    return ",".join(["1"] * n)


def listed():
    return [
        # a decode step of a small batch: one token each, blocks partly filled; latency counts
        _case("append_step_8", "append", _ones(8), _spread(1, 8, 100, 8000), scale=16, page=16),
        # a long prompt written into an empty cache
        _case("append_prompt_32k", "append", "32768", "0"),
        # the smallest attention: one sequence of a few hundred tokens, small pages, bf16
        _case("decode_1_short", "attend", "1", "616", cache="bf16", scale=0, page=16),
        # a continuous batch at one decode step, 1K to 128K tokens behind each
        _case("decode_32_ragged", "attend", _ones(32), _spread(2, 32, 1000, 131000)),
        # one request with a long context: the keys are split over the whole chip
        _case("decode_1_128k", "attend", "1", "131071", scale=0, lse=True),
        # endless streams: four first tokens and a window of 4096 over long caches
        _case("decode_64_window", "attend", _ones(64), _spread(3, 64, 500, 60000), window=4096, sink=4),
        # drafted tokens checked in one call, 64 query heads: 64 rows per KV head
        _case("verify_8x8", "attend", ",".join(["8"] * 8), _spread(4, 8, 4000, 40000), hq=64, scale=32,
              page=32),
        # a long prompt through the window: the matrix products count
        _case("prompt_32k_window", "attend", "32768", "0", window=4096, sink=4, lse=True),
        # what a decode step of sixteen long sequences adds to the weights
        _case("weights_16_step", "weights", _ones(16), _spread(5, 16, 8000, 60000)),
        # the weights that a whole prompt leaves behind
        _case("weights_prompt_8k", "weights", "8101", "0", cache="bf16", scale=0),
        # a short cache cut to half, small blocks
        _case("evict_1_2k", "evict", "0", "2000", scale=16, page=16, budget=1000, recent=64, sink=4),
        # sixteen long caches cut to 4096 tokens
        _case("evict_16_4k", "evict", ",".join(["0"] * 16), _spread(6, 16, 5000, 60000), budget=4096,
              recent=512, sink=4),
    ]


def _lens(text):
    return [int(x) for x in text.split(",")]


def _shape(case):
    """New tokens, tokens before them and tokens after the call of each sequence."""
    new, pre = _lens(case["new"]), _lens(case["prefix"])
    return new, pre, [a + b for a, b in zip(new, pre)]


def _esz(case):
    return 2 if case["cache"] == "bf16" else 1


def _seen(case):
    """Visible (query, key) pairs of all sequences, and the distinct keys of them."""
    new, pre, kv = _shape(case)
    w, s = case["window"], case["sink"]
    pairs = keys = 0
    for n, p, t in zip(new, pre, kv):
        if n == 0:
            continue
        if w == 0:
            pairs, keys = pairs + n * p + n * (n + 1) // 2, keys + t
            continue
        pos = np.arange(p, t, dtype=np.int64)
        first = np.maximum(0, pos - w + 1)
        pairs += int(np.sum(pos - first + 1 + np.minimum(first, s)))
        keys += t - int(first[0]) + min(int(first[0]), s)
    return pairs, keys


def work(case):
    new, pre, kv = _shape(case)
    hq, hkv, sb = case["hq"], case["hkv"], case["scale"]
    row = hkv * D * _esz(case)          # a token's keys, or values, of all heads
    bytes_, flops = 0.0, 0.0
    if case["op"] == "append":
        bytes_ = 2 * sum(new) * (hkv * D * 2 + row)
        if sb:                          # scales of the blocks that are touched
            bytes_ += 2 * hkv * sum(-(-t // sb) - p // sb for p, t in zip(pre, kv))
        flops = 2.0 * 2 * sum(new) * hkv * D
    elif case["op"] in ("attend", "weights"):
        pairs, keys = _seen(case)
        both = 2 if case["op"] == "attend" else 1
        bytes_ = both * keys * (row + (hkv / sb if sb else 0)) + sum(new) * hq * D * 2
        if case["op"] == "attend":
            bytes_ += sum(new) * hq * (D * 2 + (4 if case["lse"] else 0))
        else:
            bytes_ += sum(new) * hq * 4 + 2 * keys * hkv * 4
        flops = 2.0 * both * D * hq * pairs
    else:
        stay = sum(min(t, case["budget"]) for t in kv)
        bytes_ = 2 * 2 * stay * (row + (hkv / sb if sb else 0)) + hkv * 4 * (sum(kv) + 2 * stay)
        flops = 2.0 * stay * hkv * D + hkv * sum(kv)
    return {"bytes": float(bytes_), "flops": flops}


def _cost(case):
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / 5e14


def draw(rng):
    """One more case of the ranges above."""
    most = 0.5 * max(_cost(c) for c in listed())

    def between(lo, hi):
        n = int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))
        return max(lo, n // 64 * 64) if rng.random() < 0.3 else min(n, hi)

    while True:
        op = rng.choices(["append", "attend", "weights", "evict"], [2, 6, 2, 2])[0]
        hq, hkv = rng.choice([(32, 8), (32, 8), (64, 8), (32, 4), (16, 8), (8, 8), (4, 1)])
        cache = rng.choice(["fp8", "fp8", "fp8", "bf16"])
        page = rng.choice([16, 32, 64, 64, 128, 192])
        scale = rng.choice([s for s in (16, 32, 64, 64, 128) if page % s == 0] + [0]) if cache == "fp8" else 0
        if not scale and rng.random() < 0.3:
            page = rng.choice([1, 24, 80])
        kw = dict(hq=hq, hkv=hkv, cache=cache, scale=scale, page=page)
        batch = between(1, 64)
        if op == "evict":
            new, pre = [0] * batch, [between(64, 65536) for _ in range(batch)]
            budget = between(32, 8192)
            kw.update(budget=budget, sink=rng.choice([0, 1, 4, 16]), recent=rng.randrange(0, budget // 2 + 1))
        else:
            if rng.random() < 0.6:      # decode and verify steps
                new = [rng.choice([1, 1, 1, 2, 4])] * batch
                pre = [between(1, 131000) for _ in range(batch)]
            else:                       # prompts and chunks of them
                batch = min(batch, rng.choice([1, 1, 2, 6]))
                new = [between(9, 16384) for _ in range(batch)]
                pre = [rng.choice([0, between(1, 32768)]) for _ in range(batch)]
            if op != "append" and rng.random() < 0.4:
                kw.update(window=between(128, 8192), sink=rng.choice([0, 1, 4, 128]))
            if op == "attend":
                kw.update(lse=rng.random() < 0.5)
        c = _case("drawn", op, ",".join(map(str, new)), ",".join(map(str, pre)), **kw)
        del c["name"]
        if _cost(c) > most or sum(_shape(c)[2]) > 1200000:
            continue
        if op in ("attend", "weights"):     # scores and keys that the plain form holds at a time
            rows, keys = _plan_size(c)
            if rows * keys * c["hq"] * _block(c) > 5.5e9 or rows * keys * c["hkv"] * D > 8e9:
                continue
        return c


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _block(case):
    """Queries of a sequence that the plain form takes together."""
    return min(512, max(_lens(case["new"])))


def _blocks(case):
    """(sequence, first query, queries, first and last key of the window part) of the plain form's blocks."""
    new, pre, _ = _shape(case)
    c, w = _block(case), case["window"]
    s = case["sink"] if w else 0
    found = [(b, i, min(c, n - i)) for b, n in enumerate(new) for i in range(0, n, c)]
    return s, [(b, i, m, max(s, pre[b] + i - w + 1) if w else 0, pre[b] + i + m - 1) for b, i, m in found]


def _plan_size(case):
    s, blocks = _blocks(case)
    return len(blocks), s + max(max(0, hi - lo + 1) for _, _, _, lo, hi in blocks)


def _inputs(case, seed):
    """Queries, the tokens' keys and values, and where they lie in the pool."""
    new, pre, kv = _shape(case)
    hq, hkv, page = case["hq"], case["hkv"], case["page"]
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(11 + 2 * seed)
    tokens = sum(kv)

    def draws(*shape):
        return torch.randn(shape, generator=g, device=dev)

    # keys and values whose size changes from run to run of tokens and from head
    # to head, first tokens that attract every query, and a few heavy tokens
    u = draws(hkv, D)
    u /= u.norm(dim=1, keepdim=True)
    size = torch.exp(0.4 * draws(tokens // 16 + 1, hkv, 1)).repeat_interleave(16, dim=0)[:tokens]
    k = draws(tokens, hkv, D) * size
    heavy = (torch.rand((tokens, hkv, 1), generator=g, device=dev) < 0.01).float()
    first = torch.cat([torch.arange(t, device=dev) for t in kv])[:, None, None]
    k += (12.0 * heavy * size + 16.0 * (first < 4)) * u
    v = draws(tokens, hkv, D) * torch.exp(0.4 * draws(tokens // 16 + 1, hkv, 1)).repeat_interleave(16, dim=0)[:tokens]
    q = (draws(sum(new), hq, D) + 1.2 * u.repeat_interleave(hq // hkv, dim=0)).bfloat16()
    # pages in any order, and some of other sequences between them
    need = [-(-t // page) for t in kv]
    evicted = [-(-min(t, case["budget"]) // page) for t in kv] if case["op"] == "evict" else [0] * len(kv)
    total = sum(need) + sum(evicted) + 3
    order = torch.randperm(total, generator=torch.Generator().manual_seed(7 + seed)).int()
    ends = np.cumsum([0] + need + evicted)
    rows = [order[a:b] for a, b in zip(ends[:-1], ends[1:])]
    lay = lambda part: torch.nn.utils.rnn.pad_sequence(part, batch_first=True).to(dev)     # noqa: E731
    table, target = lay(rows[:len(kv)]), lay(rows[len(kv):])
    slots = torch.cat([table[b].long().repeat_interleave(page)[:t] * page + torch.arange(t, device=dev) % page
                       for b, t in enumerate(kv)])
    return dict(q=q, k=k, v=v, slots=slots, table=table.contiguous(), target=target.contiguous(), pages=total)


def _exponent(amax):
    """e = ceil(log2(amax / 448)) within [-100, 118], of numbers held exactly; -100 where amax is 0."""
    m, e = torch.frexp(amax)                       # amax = m 2^e, 0.5 <= m < 1; 448 = 0.875 * 2^9
    e = e - 9 + (m > 0.875).to(e.dtype)
    return torch.where(amax > 0, e, torch.full_like(e, -100)).clamp(-100, 118)


def _power(e):
    """2^e exactly, -126 <= e <= 127, from its bits."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _codes(x):
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


def _values(codes):
    return codes.view(torch.float8_e4m3fn).float()


def _stored(case, x, slots, total):
    """The pool of one tensor in the cache's type, with its scales."""
    hkv, sb = case["hkv"], case["scale"]
    if case["cache"] == "bf16":
        pool = torch.zeros((total, hkv, D), dtype=torch.bfloat16, device=x.device)
        return pool.index_copy_(0, slots, x.bfloat16()), None
    pool = torch.zeros((total, hkv, D), dtype=torch.uint8, device=x.device)
    x = x.bfloat16().float()
    if not sb:
        scale = (x.abs().amax(dim=(0, 2)) / 448.0).clamp_min(1e-6)
        return pool.index_copy_(0, slots, _codes(x / scale[None, :, None])), scale.contiguous()
    at = (slots // sb)[:, None].expand(-1, hkv)
    amax = torch.zeros((total // sb, hkv), device=x.device).scatter_reduce_(0, at, x.abs().amax(2), "amax")
    e = _exponent(amax)
    pool.index_copy_(0, slots, _codes(x * _power(-e)[slots // sb][:, :, None]))
    return pool, (e + 127).to(torch.uint8)


def prepare(case, seed):
    """An engine's state before the call."""
    new, pre, kv = _shape(case)
    x = _inputs(case, seed)
    page, sb, hkv = case["page"], case["scale"], case["hkv"]
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(3 + 2 * seed)
    whole = lambda a: torch.tensor(a, device=dev)       # noqa: E731
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    cu_k = np.concatenate([[0], np.cumsum(kv)]).astype(np.int32)
    slots, total = x["slots"], x["pages"] * page
    st = dict(case=case, table=x["table"], q=x["q"], cu=torch.from_numpy(cu).to(dev),
              cu_k=torch.from_numpy(cu_k).to(dev), cu_host=cu, cu_k_host=cu_k)
    fresh = None
    if case["op"] == "append":          # the cache holds the tokens before the new ones
        is_new = torch.cat([torch.arange(t, device=dev) >= p for p, t in zip(pre, kv)])
        fresh = torch.nonzero(is_new).reshape(-1)
        st["k_new"], st["v_new"] = x["k"][fresh].bfloat16(), x["v"][fresh].bfloat16()
        old = torch.nonzero(~is_new).reshape(-1)
        st["k"], st["k_scale"] = _stored(case, x["k"][old], slots[old], total)
        st["v"], st["v_scale"] = _stored(case, x["v"][old], slots[old], total)
        st["new_slots"] = slots[fresh]
        # the pool's blocks that the call touches, which block each new token lies in, and what is old in a first block
        if sb:
            hit, st["block_of"] = torch.unique(slots[fresh] // sb, return_inverse=True)
            part = [(c, p // sb * sb, p) for c, p, n in zip(cu_k, pre, new) if n and p % sb]
            st["hit"] = hit
            st["part"] = slots[whole([c + j for c, a, p in part for j in range(a, p)]).long()] if part else None
    else:
        st["k"], st["k_scale"] = _stored(case, x["k"], slots, total)
        st["v"], st["v_scale"] = _stored(case, x["v"], slots, total)
    if case["op"] in ("attend", "weights"):
        s, blocks = _blocks(case)
        c = _block(case)
        st["sinks"], st["columns"] = s, _plan_size(case)[1]
        st["of"], st["q0"], _, st["lo"], st["hi"] = (whole([b[i] for b in blocks]).long() for i in range(5))
        st["pre"] = whole(pre).long()
        st["rows"] = whole([i * c + j for i, b in enumerate(blocks) for j in range(b[2])]).long()
        st["q_at"] = whole([[min(cu[b] + i + j, cu[b + 1] - 1) for j in range(c)] for b, i, _, _, _ in blocks]).long()
    if case["op"] == "weights":
        st["lse"] = _attention(st, False)[1]
        st["before"] = torch.rand((len(kv), hkv, max(kv)), generator=g, device=dev)
    if case["op"] == "evict":
        st["target"] = x["target"]
        st["lens"] = whole(kv).long()
        st["weights"] = torch.rand((len(kv), hkv, max(kv)), generator=g, device=dev) ** 8
        st["weights"][:, :, ::7] = 0.25            # ties
    if own:
        import paper_2608_19758_amd as fp2
        st["p"] = fp2.make_cache_params(
            batch=len(kv), num_q_heads=case["hq"], num_kv_heads=hkv, max_seq_len=max(new), max_kv_len=max(kv),
            page_size=page, max_pages_per_seq=x["table"].shape[1], dtype=case["cache"], scale_tokens=sb,
            sink_tokens=case["sink"], window_tokens=case["window"])
        st["cache"] = fp2.KVCache(st["k"], st["v"], st["k_scale"], st["v_scale"])
        st["workspace"] = fp2.alloc_cache_workspace(st["p"])
    return st


# ---------------------------------------------------------------------------
# The operators
# ---------------------------------------------------------------------------

def _at(case, pool, scale, slot):
    """Values of the pool's tokens at `slot` [..., tokens] -> [..., tokens, hkv, D], in 32 bits."""
    if case["cache"] == "bf16":
        return pool[slot].float()
    x = _values(pool[slot])
    if not case["scale"]:
        return x * scale[:, None]
    return x * _power(scale[slot // case["scale"]].int() - 127)[..., None]


def _scores(st):
    """Scaled scores [blocks, hkv, queries x group, columns] with -inf where a query does not see the
    key, the keys' indexes [blocks, columns] and their slots in the pool."""
    case = st["case"]
    hq, hkv, page, s, w = case["hq"], case["hkv"], case["page"], st["sinks"], case["window"]
    col = torch.arange(st["columns"], device=st["q"].device)
    key = torch.where(col < s, col, st["lo"][:, None] + col - s)
    there = key <= st["hi"][:, None]
    at = torch.where(there, key, 0)
    slot = st["table"][st["of"][:, None], at // page].long() * page + at % page
    k = _at(case, st["k"], st["k_scale"], slot).permute(0, 2, 3, 1).contiguous()
    nb, c = st["q_at"].shape
    q = st["q"][st["q_at"]].float().view(nb, c, hkv, hq // hkv, D).transpose(1, 2).reshape(nb, hkv, -1, D)
    x = torch.matmul(q, k).mul_(1.0 / math.sqrt(D)).view(nb, hkv, c, hq // hkv, -1)
    pos = (st["pre"][st["of"]] + st["q0"])[:, None] + torch.arange(c, device=key.device)
    seen = there[:, None] & (key[:, None] <= pos[..., None])
    if w:
        seen &= (col < s) | (pos[..., None] - key[:, None] < w)
    x.masked_fill_(~seen[:, None, :, None], -math.inf)
    return x.view(nb, hkv, -1, x.shape[-1]), key, slot


def _rows(st, x):
    """[blocks, hkv, queries x group, ...] -> [queries of the batch, hq, ...]."""
    nb, c = st["q_at"].shape
    hkv, tail = st["case"]["hkv"], x.shape[3:]
    x = x.view(nb, hkv, c, -1, *tail).transpose(1, 2)
    return x.reshape(nb * c, st["case"]["hq"], *tail)[st["rows"]]


def _attention(st, values=True):
    x, _, slot = _scores(st)
    top = x.amax(-1, keepdim=True)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = _rows(st, (top + total.log()).squeeze(-1))
    if not values:
        return None, lse
    v = _at(st["case"], st["v"], st["v_scale"], slot).transpose(1, 2).contiguous()
    return _rows(st, torch.matmul(p, v).div_(total)).bfloat16(), lse


def _weights(st):
    case = st["case"]
    x, key, slot = _scores(st)
    nb, c = st["q_at"].shape
    lse = st["lse"][st["q_at"]].view(nb, c, case["hkv"], -1).transpose(1, 2).reshape(nb, case["hkv"], -1, 1)
    valid = torch.zeros(nb * c, dtype=torch.bool, device=x.device)
    valid[st["rows"]] = True
    group = case["hq"] // case["hkv"]
    p = x.sub_(lse).exp_().mul_(valid.view(nb, 1, c).repeat_interleave(group, dim=2)[..., None])
    got = p.sum(2, dtype=torch.float64)                                            # [blocks, hkv, columns]
    out = st["before"].double()
    hi = out.shape[2]
    at = (st["of"][:, None] * case["hkv"] + torch.arange(case["hkv"], device=x.device))[..., None] * hi
    at = at + torch.where(key <= st["hi"][:, None], key, 0)[:, None]
    return out.view(-1).index_add_(0, at.reshape(-1), got.reshape(-1)).view_as(out).float()


def _append_one(st, name):
    case, sb = st["case"], st["case"]["scale"]
    pool, scale, x = st[name], st[name + "_scale"], st[name + "_new"].float()
    if case["cache"] == "bf16":
        pool.index_copy_(0, st["new_slots"], st[name + "_new"])
        return
    if not sb:
        pool.index_copy_(0, st["new_slots"], _codes(x / scale[:, None]))
        return
    hit, of = st["hit"], st["block_of"]
    amax = torch.zeros((hit.numel(), case["hkv"]), device=x.device).scatter_reduce_(
        0, of[:, None].expand(-1, case["hkv"]), x.abs().amax(2), "amax")
    e = _exponent(amax)
    if st["part"] is not None:      # blocks that hold tokens keep a scale that is larger
        block = st["part"] // sb
        place = torch.searchsorted(hit, block)
        before = scale[block].int() - 127
        e[place] = torch.maximum(e[place], before)
        moved = _values(pool[st["part"]]) * _power(before - e[place])[..., None]
        pool.index_copy_(0, st["part"], _codes(moved))
    pool.index_copy_(0, st["new_slots"], _codes(x * _power(-e)[of][:, :, None]))
    scale.index_copy_(0, hit, (e + 127).to(torch.uint8))


def _evict(st):
    case, lens, w = st["case"], st["lens"], st["weights"]
    budget, page, sb, hkv = case["budget"], case["page"], case["scale"], case["hkv"]
    b, _, most = w.shape
    dev = w.device
    t = torch.arange(most, device=dev)
    end = lens[:, None, None]
    rank = torch.where((t < case["sink"]) | (t >= end - case["recent"]), torch.full_like(w, math.inf), w)
    rank = torch.where(t < end, rank, torch.full_like(w, -math.inf))
    n = min(budget, most)
    kept = torch.sort(rank, dim=2, descending=True, stable=True).indices[:, :, :n]
    kept = torch.where(kept < end, kept, most)
    kept = torch.nn.functional.pad(torch.sort(kept, dim=2).values, (0, budget - n), value=most)
    stays = kept < end
    at = torch.where(stays, kept, 0)
    heads = torch.arange(hkv, device=dev)[None, :, None]
    seqs = torch.arange(b, device=dev)[:, None, None]
    left = torch.where(stays, w.gather(2, at.clamp(max=most - 1)), torch.zeros((), device=dev))
    weights = torch.nn.functional.pad(left, (0, max(0, most - budget)))[:, :, :most].contiguous()
    src = st["table"][seqs, at // page].long() * page + at % page
    i = torch.arange(budget, device=dev)
    inside = torch.clamp(i // page, max=st["target"].shape[1] - 1)
    dst = (st["target"][:, inside].long() * page + i % page)[:, None].expand(-1, hkv, -1)
    spot = torch.where(stays, dst, st["k"].shape[0])            # one row behind the pool takes what does not stay
    for_all = (spot.reshape(-1), heads.expand(b, -1, budget).reshape(-1))

    def move(name):
        pool, scale = st[name], st[name + "_scale"]
        rows = pool[src, heads]
        if sb:
            power = _power(scale[src // sb, heads].int() - 127)[..., None]
            x = torch.where(stays[..., None], _values(rows) * power, torch.zeros((), device=dev))
            full = torch.nn.functional.pad(x, (0, 0, 0, -budget % sb)).view(b, hkv, -1, sb, D)
            e = _exponent(full.abs().amax((3, 4)))
            rows = _codes(x * _power(-e).repeat_interleave(sb, dim=2)[:, :, :budget, None])
            where = torch.where(stays[:, :, ::sb], dst[:, :, ::sb] // sb, scale.shape[0])
            wide = torch.cat([scale, scale[:1]])
            wide[where, heads] = (e + 127).to(torch.uint8)
            scale.copy_(wide[:-1])
        wide = torch.cat([pool, pool[:1]])
        wide[for_all] = rows.reshape(-1, D)
        pool.copy_(wide[:-1])

    move("k")
    move("v")
    cu = torch.zeros(b + 1, dtype=torch.int32, device=dev)
    cu[1:] = torch.cumsum(torch.clamp(lens, max=budget), 0)
    return {"kept": torch.where(stays, kept, -1).int(), "cu_k": cu, "weights": weights}


def _pools(st):
    """The cache with its scales; 8-bit codes as the numbers that they are."""
    look = (lambda x: x) if st["case"]["cache"] == "bf16" else (lambda x: x.view(torch.float8_e4m3fn))
    got = {"k": look(st["k"]), "v": look(st["v"])}
    if st["case"]["scale"]:
        got.update(k_scale=st["k_scale"], v_scale=st["v_scale"])
    return got


def run(state):
    """One layer's call."""
    st, case = state, state["case"]
    if own:
        import paper_2608_19758_amd as fp2
        lens = dict(cu_seqlens_k_host=st["cu_k_host"])
        if case["op"] == "append":
            fp2.cache_append(st["p"], st["k_new"], st["v_new"], st["cache"], st["cu"], st["cu_k"], st["table"],
                             cu_seqlens_host=st["cu_host"], **lens)
            return _pools(st)
        if case["op"] == "attend":
            out, lse = fp2.cache_attend(st["p"], st["q"], st["cache"], st["cu"], st["cu_k"], st["table"],
                                        want_lse=case["lse"], workspace=st["workspace"],
                                        cu_seqlens_host=st["cu_host"], **lens)
            return {"out": out, "lse": lse}
        if case["op"] == "weights":
            return {"weights": fp2.cache_weights(st["p"], st["q"], st["lse"], st["cache"], st["cu"], st["cu_k"],
                                                 st["table"], weights_in=st["before"],
                                                 cu_seqlens_host=st["cu_host"], **lens)}
        kept, cu, left = fp2.cache_evict(st["p"], st["cache"], st["weights"], st["cu_k"], st["table"],
                                         st["target"], budget=case["budget"], recent_tokens=case["recent"], **lens)
        return {"kept": kept, "cu_k": cu, "weights": left, **_pools(st)}
    if case["op"] == "append":
        _append_one(st, "k")
        _append_one(st, "v")
        return _pools(st)
    if case["op"] == "attend":
        out, lse = _attention(st)
        return {"out": out, "lse": lse if case["lse"] else None}
    if case["op"] == "weights":
        return {"weights": _weights(st)}
    return {**_evict(st), **_pools(st)}


# ---------------------------------------------------------------------------
# The same from the definitions, in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    new, pre, kv = _shape(case)
    hq, hkv, page, sb = case["hq"], case["hkv"], case["page"], case["scale"]
    g, dev = hq // hkv, st["q"].device
    table = st["table"].long()

    def times_power(x, e):
        return x * ((e.long() + 1023) << 52).view(torch.float64)

    def stands_for(name, slot, h):
        x = st[name][slot, h]
        if case["cache"] == "bf16":
            return x.double()
        x = x.view(torch.float8_e4m3fn).double()
        if not sb:
            return x * st[name + "_scale"][h].double()
        return times_power(x, st[name + "_scale"][slot // sb, h].int()[:, None] - 127)

    def slots_of(b, keys, of=table):
        return of[b][keys // page] * page + keys % page

    def nearest(x):
        """x rounded to e4m3's numbers, ties to even, and held within +-448."""
        x = x.clamp(-448, 448)
        bits = 4 - torch.frexp(x.abs().clamp_min(2.0 ** -6)).exponent     # steps of 2^-bits
        return times_power(torch.round(times_power(x, bits)), -bits)

    def scale_for(most):
        """The smallest 2^e >= most / 448."""
        e = -100
        if most > 0:
            m, e = math.frexp(most / 448.0)
            e = e - 1 if m == 0.5 else e
        return min(118, max(-100, e))

    if case["op"] in ("attend", "weights"):
        if _cost(case) > 0.02 and case["window"] == 0:
            return None
        out = torch.zeros((sum(new), hq, D), dtype=torch.float64, device=dev)
        lse = torch.zeros((sum(new), hq), dtype=torch.float64, device=dev)
        weights = st["before"].double() if case["op"] == "weights" else None
        row = 0
        for b, (n, p, t) in enumerate(zip(new, pre, kv)):
            for i in range(0, n, 1024):
                m = min(1024, n - i)
                lo = max(0, p + i - case["window"] + 1) if case["window"] else 0
                keys = torch.arange(lo, p + i + m, device=dev)
                if case["window"]:
                    keys = torch.cat([torch.arange(min(lo, case["sink"]), device=dev), keys])
                pos = p + i + torch.arange(m, device=dev)
                dist = pos[:, None] - keys[None, :]
                see = dist >= 0
                if case["window"]:
                    see &= (dist < case["window"]) | (keys < case["sink"])[None, :]
                slot = slots_of(b, keys)
                for h in range(hkv):
                    k, v = stands_for("k", slot, h), stands_for("v", slot, h)
                    for a in range(h * g, h * g + g):
                        x = (st["q"][row + i:row + i + m, a].double() @ k.t()) / math.sqrt(D)
                        x = x.masked_fill(~see, -math.inf)
                        if case["op"] == "weights":
                            x = torch.exp(x - st["lse"][row + i:row + i + m, a].double()[:, None])
                            weights[b, h].index_add_(0, keys, x.sum(0))
                            continue
                        z = torch.logsumexp(x, dim=1)
                        out[row + i:row + i + m, a] = torch.exp(x - z[:, None]) @ v
                        lse[row + i:row + i + m, a] = z
            row += n
        if case["op"] == "weights":
            return {"weights": weights}
        return {"out": out, "lse": lse if case["lse"] else None}

    if sum(kv) * hkv > 4000000:
        return None
    got = {}
    if case["op"] == "append":
        for name in ("k", "v"):
            x = st[name + "_new"].double()
            if case["cache"] == "bf16":
                got[name] = st[name].double()
                got[name][st["new_slots"]] = x
                continue
            codes = st[name].view(torch.float8_e4m3fn).double()
            if not sb:
                codes[st["new_slots"]] = nearest(x / st[name + "_scale"].double()[:, None])
                got[name] = codes
                continue
            scales = st[name + "_scale"].clone()
            row = 0
            for b, (n, p, t) in enumerate(zip(new, pre, kv)):
                for a in range(p // sb * sb, t, sb) if n else ():
                    old = slots_of(b, torch.arange(a, max(a, p), device=dev)) if a < p else None
                    z = min(t, a + sb)
                    here = slots_of(b, torch.arange(max(a, p), z, device=dev))
                    part = x[row + max(a, p) - p:row + z - p]
                    tops = part.abs().amax((0, 2)).tolist()
                    for h in range(hkv):
                        e, was = scale_for(tops[h]), int(scales[here[0] // sb, h]) - 127
                        if old is not None:
                            e = max(e, was)
                            codes[old, h] = nearest(codes[old, h] * 2.0 ** (was - e))
                        codes[here, h] = nearest(part[:, h] * 2.0 ** -e)
                        scales[here[0] // sb, h] = e + 127
                row += n
                if n > 4096:
                    return None
            got[name], got[name + "_scale"] = codes, scales
        return got

    budget = case["budget"]
    kept = torch.full((len(kv), hkv, budget), -1, dtype=torch.int32, device=dev)
    weights = torch.zeros(st["weights"].shape, dtype=torch.float64, device=dev)
    if sum(min(t, budget) for t in kv) * hkv > 20000:
        return None
    pools = {n: (st[n].double() if case["cache"] == "bf16" else st[n].view(torch.float8_e4m3fn).double())
             for n in ("k", "v")}
    scales = {n: st[n + "_scale"].clone() if sb else None for n in ("k", "v")}
    for b, t in enumerate(kv):
        for h in range(hkv):
            w = st["weights"][b, h, :t].double().cpu().numpy()
            fixed = [j for j in range(t) if j < case["sink"] or j >= t - case["recent"]]
            others = sorted((j for j in range(t) if case["sink"] <= j < t - case["recent"]), key=lambda j: (-w[j], j))
            stay = sorted((fixed + others)[:budget]) if t > budget else list(range(t))
            at = torch.tensor(stay, device=dev)
            kept[b, h, :len(stay)] = at.int()
            weights[b, h, :len(stay)] = torch.from_numpy(w[stay]).to(dev)
            to = slots_of(b, torch.arange(len(stay), device=dev), st["target"].long())
            for name in ("k", "v"):
                if not sb:
                    pools[name][to, h] = pools[name][slots_of(b, at), h]
                    continue
                x = stands_for(name, slots_of(b, at), h)
                for a in range(0, len(stay), sb):
                    e = scale_for(float(x[a:a + sb].abs().max()))
                    pools[name][to[a:a + sb], h] = nearest(x[a:a + sb] * 2.0 ** -e)
                    scales[name][to[a] // sb, h] = e + 127
    cu = torch.tensor([0] + list(np.cumsum([min(t, budget) for t in kv])), dtype=torch.int32, device=dev)
    got = {"kept": kept, "cu_k": cu, "weights": weights, "k": pools["k"], "v": pools["v"]}
    if sb:
        got.update(k_scale=scales["k"], v_scale=scales["v"])
    return got

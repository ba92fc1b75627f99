"""The operators around positions in the paged KV cache, and attention to states of another
length, whose speed is measured: rotary positions, appending with them, reading a cache back,
moving its tokens to other positions, and cross attention.

Every case is one layer's call as a serving engine makes it, on a paged pool of keys and values
in bf16, in e4m3 codes with one fp32 scale per head, or in e4m3 codes with one power-of-two
scale per block of ``scale`` tokens and head.

* rotary: queries and keys turned by their positions. With angles t_i = f_i * position, f_i =
  base^(-2i/dim) after the scaling, the pair (x, y) of dimensions (i, i + dim/2), or (2i, 2i + 1)
  where ``pairs``, becomes a (x cos - y sin, x sin + y cos); dimensions from ``dim`` on stay.
* append: the same on the way into the cache: new keys are turned and written in its type,
  values written, queries returned turned. A block's scale is 2^e, e = ceil(log2(amax / 448)) of
  its tokens; it never falls, and codes that were there are rounded again where it grows.
* read:   the last tokens of each sequence as bf16 rows, the keys' turn taken back if ``undo``.
* move:   the tokens of each sequence to other pages, the keys turned by a number of positions.
* cross:  O = softmax(scale * Q K^T) V over all keys of each sequence.

``own`` chooses between the plain form and the framework's calls.
"""
import math

import numpy as np
import torch

own = False

D = 128


def _case(name, op, new, prefix, **kw):
    c = dict(name=name, op=op, new=new, prefix=prefix, hq=32, hkv=8, cache="fp8", scale=64, page=64,
             dim=128, pairs=False, base=10000.0, scaling="none", factor=1.0, start=0, qtype="bf16",
             packed=True, undo=False, each=False, lse=False)
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
        # queries and keys of a small decode step; latency counts
        _case("rotary_step_8", "rotary", _ones(8), _spread(1, 8, 100, 8000)),
        # a chunk far inside a long context, frequencies scaled for it, queries as the codes of a sparse prefill
        _case("rotary_chunk_16k", "rotary", "16384", "114688", scaling="ramp", factor=4.0, base=500000.0, qtype="fp8"),
        # a decode step of 32 sequences: blocks partly filled
        _case("append_step_32", "append", _ones(32), _spread(2, 32, 100, 60000), scale=16, page=16),
        # a long prompt written into an empty cache
        _case("append_prompt_32k", "append", "32768", "0"),
        # chunks of several requests, odd lengths, half of the head turned, bf16
        _case("append_ragged_bf16", "append", _spread(3, 9, 50, 5000), _spread(4, 9, 1, 30000), cache="bf16", scale=0,
              dim=64, pairs=True, page=16),
        # a short cached prefix read back
        _case("read_1_2k", "read", "2001", "0", cache="bf16", scale=0, page=16),
        # sixteen long sequences handed to another server, positions taken out
        _case("read_16_undo", "read", _spread(5, 16, 5000, 60000), ",".join(["0"] * 16), undo=True),
        # a short sequence after an eviction: every head kept other tokens
        _case("move_1_1k", "move", "0", "1000", scale=16, page=16, each=True),
        # cached documents taken over at other offsets
        _case("move_16_docs", "move", ",".join(["0"] * 16), _spread(6, 16, 2000, 30000), start=1),
        # a decode step over an encoder's states, which are ragged
        _case("cross_step_32", "cross", _ones(32), _spread(7, 32, 300, 4000), cache="bf16", scale=0, page=16),
        # decoder prompts of a few hundred tokens over an encoder's states
        _case("cross_prompts_8", "cross", _spread(8, 8, 100, 800), _spread(9, 8, 900, 4000), scale=32, page=32, lse=True),
        # thousands of queries over long states: the matrix products count
        _case("cross_4k_30k", "cross", "4096", "30001"),
    ]


def _lens(text):
    return [int(x) for x in text.split(",")]


def _shape(case):
    """New tokens (queries), tokens before them, and tokens in the cache of each sequence. The cache of a
    cross attention holds `prefix` tokens."""
    new, pre = _lens(case["new"]), _lens(case["prefix"])
    if case["op"] == "cross":
        return new, pre, pre
    return new, pre, [a + b for a, b in zip(new, pre)]


def _esz(case):
    return 2 if case["cache"] == "bf16" else 1


def work(case):
    new, pre, kv = _shape(case)
    hq, hkv, sb, op = case["hq"], case["hkv"], case["scale"], case["op"]
    row = hkv * D * _esz(case) + (hkv / sb if sb else 0)      # a token's keys, or values, of all heads
    qrow = hq * D * (1 if case["qtype"] == "fp8" else 2)
    t = sum(new)
    if op == "rotary":
        return {"bytes": t * (2.0 * (hq + hkv) * D + qrow + 2 * hkv * D + 4), "flops": 3.0 * t * (hq + hkv) * case["dim"]}
    if op == "append":
        return {"bytes": t * (2.0 * (hq + 2 * hkv) * D + qrow + 2 * row),
                "flops": t * (3.0 * (hq + hkv) * case["dim"] + 4 * hkv * D)}
    if op == "read":
        return {"bytes": t * (2.0 * row + 2 * 2 * hkv * D), "flops": t * hkv * (2.0 * D + 3 * case["dim"] * case["undo"])}
    if op == "move":
        t = sum(kv)
        return {"bytes": t * (4.0 * row + 4 * (hkv if case["each"] else 0)), "flops": t * hkv * 4.0 * D}
    pairs = sum(n * p for n, p in zip(new, kv))
    seen = sum(p for n, p in zip(new, kv) if n)
    return {"bytes": 2.0 * seen * row + t * hq * (4.0 * D + (4 if case["lse"] else 0)), "flops": 4.0 * D * hq * pairs}


def _cost(case):
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / 5e14


def draw(rng):
    """One more case of the ranges above."""
    most = max(_cost(c) for c in listed())

    def between(lo, hi):
        n = int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))
        return max(lo, n // 64 * 64) if rng.random() < 0.3 else min(n, hi)

    while True:
        op = rng.choices(["rotary", "append", "read", "move", "cross"], [2, 4, 2, 2, 4])[0]
        hq, hkv = rng.choice([(32, 8), (32, 8), (64, 8), (32, 4), (16, 8), (8, 8), (4, 1)])
        cache = rng.choice(["fp8", "fp8", "fp8", "bf16"])
        page = rng.choice([16, 32, 64, 64, 128, 192])
        scale = rng.choice([s for s in (16, 32, 64, 64, 128) if page % s == 0] + [0]) if cache == "fp8" else 0
        if not scale and rng.random() < 0.3:
            page = rng.choice([1, 24, 80])
        kw = dict(hq=hq, hkv=hkv, cache=cache, scale=scale, page=page)
        kw.update(dim=rng.choice([128, 128, 128, 64, 96, 32, 80, 100, 2]), pairs=rng.random() < 0.4,
                  base=rng.choice([10000.0, 500000.0, 1000000.0]))
        if rng.random() < 0.5:
            kw.update(scaling=rng.choice(["linear", "ramp"]), factor=rng.choice([2.0, 4.0, 8.0, 32.0]))
        if kw["dim"] < 16:
            kw.update(scaling="none", factor=1.0)
        batch = between(1, 64)
        if op == "cross":
            if rng.random() < 0.5:      # decoding, drafts
                new = [rng.choice([1, 1, 1, 2, 4, 8])] * batch
                pre = [between(1, 32000) for _ in range(batch)]
            else:
                batch = min(batch, rng.choice([1, 1, 2, 8]))
                new = [between(9, 8192) for _ in range(batch)]
                pre = [between(1, 32000) for _ in range(batch)]
            if batch > 2 and rng.random() < 0.3:
                pre[rng.randrange(batch)] = 0          # a request without states
            kw.update(lse=rng.random() < 0.5)
        elif op == "move":
            new, pre = [0] * batch, [between(1, 65536) for _ in range(batch)]
            kw.update(each=rng.random() < 0.5, start=rng.choice([0, 1, 1, 2]))
        elif op == "read":
            new = [between(1, 65536) for _ in range(batch)]
            pre = [rng.choice([0, between(1, 8192)]) for _ in range(batch)]
            kw.update(undo=rng.random() < 0.5)
        else:
            if rng.random() < 0.5:
                new = [rng.choice([1, 1, 1, 2, 4])] * batch
                pre = [between(1, 131000) for _ in range(batch)]
            else:
                batch = min(batch, rng.choice([1, 1, 2, 6]))
                new = [between(9, 32768) for _ in range(batch)]
                pre = [rng.choice([0, between(1, 32768)]) for _ in range(batch)]
            kw.update(qtype=rng.choice(["bf16", "bf16", "fp8"]), packed=rng.random() < 0.7, start=rng.choice([0, 0, 1000000]))
        c = _case("drawn", op, ",".join(map(str, new)), ",".join(map(str, pre)), **kw)
        del c["name"]
        if _cost(c) > most or sum(_shape(c)[2]) > 1200000:
            continue
        if op == "cross":               # scores and keys that the plain form holds at a time
            if batch * max(new) * max(max(pre), 1) * hq > 4.2e9 or batch * max(pre) * hkv * D > 4e9:
                continue
        return c


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

ORIGINAL = 8192      # positions that a "ramp" scales from


def _frequencies(case):
    """Radians a position of each pair, and the factor of both parts, in 64 bits."""
    dim, base, by = case["dim"], case["base"], case["factor"]
    i = np.arange(dim // 2, dtype=np.float64)
    f = base ** (-2.0 * i / dim)
    if case["scaling"] == "linear":
        return f / by, 1.0
    if case["scaling"] == "ramp":        # slow pairs as with "linear", fast ones as they are
        at = lambda turns: dim * math.log(ORIGINAL / (2 * math.pi * turns)) / (2 * math.log(base))     # noqa: E731
        lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), dim - 1)
        slow = np.clip((i - lo) / max(hi - lo, 0.001), 0.0, 1.0)
        return f * (1.0 - slow) + f / by * slow, 1.0 + 0.1 * math.log(by)
    return f, 1.0


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
        # room for what a turn makes of the largest: sqrt(2) times as much, and the scaling's factor
        scale = torch.full((hkv,), 1.0 / 20.0, device=x.device)
        if x.shape[0]:
            scale = (1.5 * _frequencies(case)[1] * x.abs().amax(dim=(0, 2)) / 448.0).clamp_min(1e-6)
        return pool.index_copy_(0, slots, _codes(x / scale[None, :, None])), scale.contiguous()
    at = (slots // sb)[:, None].expand(-1, hkv)
    amax = torch.zeros((total // sb, hkv), device=x.device).scatter_reduce_(0, at, x.abs().amax(2), "amax")
    e = _exponent(amax)
    pool.index_copy_(0, slots, _codes(x * _power(-e)[slots // sb][:, :, None]))
    return pool, (e + 127).to(torch.uint8)


def prepare(case, seed):
    """An engine's state before the call."""
    new, pre, kv = _shape(case)
    op, hq, hkv, page, sb = case["op"], case["hq"], case["hkv"], case["page"], case["scale"]
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(11 + 2 * seed)
    r = np.random.default_rng(5 + seed)

    def draws(*shape):
        return torch.randn(shape, generator=g, device=dev)

    freq, amplitude = _frequencies(case)
    st = dict(case=case, freq=torch.from_numpy(freq).to(dev), amplitude=amplitude)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    cu_k = np.concatenate([[0], np.cumsum(kv)]).astype(np.int32)
    st.update(cu=torch.from_numpy(cu).to(dev), cu_k=torch.from_numpy(cu_k).to(dev), cu_host=cu, cu_k_host=cu_k)
    tokens, fresh = sum(kv), sum(new)
    # keys and queries of a head lean towards one direction, sizes change from run to run of tokens
    u = draws(hkv, D)
    u /= u.norm(dim=1, keepdim=True)

    def size(n):
        return torch.exp(0.4 * draws(n // 16 + 1, hkv, 1)).repeat_interleave(16, dim=0)[:n]

    def queries(n):
        return (draws(n, hq, D) + 1.2 * u.repeat_interleave(hq // hkv, dim=0)).bfloat16()

    def keys(n):
        s = size(n)
        heavy = (torch.rand((n, hkv, 1), generator=g, device=dev) < 0.01).float()
        return draws(n, hkv, D) * s + 12.0 * heavy * s * u

    index = np.concatenate([np.arange(p, p + n) for p, n in zip(pre, new)] + [np.zeros(0)])[:fresh]
    if op in ("rotary", "append"):
        q, k, v = queries(fresh), keys(fresh).bfloat16(), (draws(fresh, hkv, D) * size(fresh)).bfloat16()
        if case["packed"]:               # as one projection gives them
            row = torch.cat([q.view(fresh, -1), k.view(fresh, -1), v.view(fresh, -1)], dim=1)
            q, k, v = row.split([hq * D, hkv * D, hkv * D], dim=1)
            q, k, v = q.view(fresh, hq, D), k.view(fresh, hkv, D), v.view(fresh, hkv, D)
        st.update(q=q, k_new=k, v_new=v)
        st["q_scale"] = None
        if case["qtype"] == "fp8":
            st["q_scale"] = (1.5 * amplitude * q.float().abs().amax(dim=(0, 2)) / 448.0).contiguous()
    if op in ("rotary", "append", "read"):
        # positions that are not the cache's indexes: tokens before these were dropped or evicted
        st["positions"] = torch.from_numpy((index + case["start"]).astype(np.int32)).to(dev)
    if op == "rotary":
        del st["v_new"]
        if own:
            st["rotary"] = _own_rotary(case)
        return st

    # pages in any order, and some of other sequences between them
    need = [-(-t // page) for t in kv]
    target = need if op == "move" else [0] * len(kv)
    total = sum(need) + sum(target) + 3
    order = torch.from_numpy(r.permutation(total).astype(np.int32))
    ends = np.cumsum([0] + need + target)
    rows = [order[a:b] for a, b in zip(ends[:-1], ends[1:])]
    width = max(1, max(need))

    def lay(part):
        t = torch.zeros((len(part), width), dtype=torch.int32)
        for i, x in enumerate(part):
            t[i, :len(x)] = x
        return t.to(dev)

    def slots_in(table):
        return torch.cat([table[b].long().repeat_interleave(page)[:t] * page + torch.arange(t, device=dev) % page
                          for b, t in enumerate(kv)])

    st["table"] = lay(rows[:len(kv)])
    slots, total = slots_in(st["table"]), total * page
    if op == "append":                   # the cache holds the tokens before the new ones
        is_new = torch.cat([torch.arange(t, device=dev) >= p for p, t in zip(pre, kv)])
        old = torch.nonzero(~is_new).reshape(-1)
        st["k"], st["k_scale"] = _stored(case, keys(len(old)), slots[old], total)
        st["v"], st["v_scale"] = _stored(case, draws(len(old), hkv, D) * size(len(old)), slots[old], total)
        st["new_slots"] = slots[torch.nonzero(is_new).reshape(-1)]
        if sb:    # the blocks that the call touches, which one each new token lies in, and what is old in a first one
            hit, st["block_of"] = torch.unique(st["new_slots"] // sb, return_inverse=True)
            at = np.concatenate([np.arange(c + p // sb * sb, c + p) for c, p, n in zip(cu_k, pre, new) if n] + [np.zeros(0)])
            st["hit"], st["part"] = hit, slots[torch.from_numpy(at.astype(np.int64)).to(dev)] if len(at) else None
    else:
        st["k"], st["k_scale"] = _stored(case, keys(tokens), slots, total)
        st["v"], st["v_scale"] = _stored(case, draws(tokens, hkv, D) * size(tokens), slots, total)
    if op == "read":
        st["read_slots"] = slots[torch.cat([torch.arange(t, device=dev) >= p for p, t in zip(pre, kv)])]
    if op == "move":
        st["target"] = lay(rows[len(kv):])
        st["slots"], st["target_slots"] = slots, slots_in(st["target"])
        most = max(kv)
        if case["each"]:                 # from where an eviction left every head's tokens
            st["moves"] = -torch.cumsum(torch.randint(0, 5, (len(kv), hkv, most), generator=g, device=dev), 2).int()
            flat = [st["moves"][b, :, :t].t() for b, t in enumerate(kv)]
        else:
            off = r.integers(-2000, 100000, len(kv)).astype(np.int32) * (case["start"] > 0)
            st["moves"] = torch.from_numpy(off).to(dev)[:, None, None]
            flat = [st["moves"][b].expand(t, 1) for b, t in enumerate(kv)]
        st["turns"] = torch.cat(flat)    # [tokens, heads or 1]
        if sb:                           # blocks of the pages, and which one each token goes to
            st["hit"], st["block_of"] = torch.unique(st["target_slots"] // sb, return_inverse=True)
            st["source_block"] = torch.empty_like(st["hit"]).index_copy_(0, st["block_of"], slots // sb)
    if op == "cross":
        st["q"] = queries(fresh)
        n, most = max(new), max(max(kv), 1)
        at = [[min(cu[b] + i, max(cu[b + 1] - 1, cu[b])) for i in range(n)] for b in range(len(new))]
        st["q_at"] = torch.tensor(at, device=dev).clamp_max(fresh - 1)
        st["rows"] = torch.cat([torch.arange(b * n, b * n + m, device=dev) for b, m in enumerate(new)])
        st["lens"] = torch.tensor(kv, device=dev)
        st["columns"] = most
    if own:
        import paper_2608_19758_amd as fp2
        st["p"] = fp2.make_cache_params(
            batch=len(kv), num_q_heads=hq, num_kv_heads=hkv, max_seq_len=max(new), max_kv_len=max(kv), page_size=page,
            max_pages_per_seq=width, dtype=case["cache"], scale_tokens=sb)
        st["cache"] = fp2.KVCache(st["k"], st["v"], st["k_scale"], st["v_scale"])
        st["rotary"] = _own_rotary(case)
        if op == "cross":
            st["workspace"] = fp2.alloc_cross_workspace(st["p"])
    return st


def _own_rotary(case):
    import paper_2608_19758_amd as fp2
    return fp2.make_rotary(case["dim"], base=case["base"], interleaved=case["pairs"], scaling=case["scaling"],
                           factor=case["factor"], original_len=ORIGINAL)


# ---------------------------------------------------------------------------
# The operators
# ---------------------------------------------------------------------------

def _turned(st, x, positions, back=False, amplitude=True):
    """x [tokens, heads, D] of 32 bits, turned by `positions` [tokens] or [tokens, heads or 1]."""
    case, dim = st["case"], st["case"]["dim"]
    pos = positions[:, None] if positions.dim() == 1 else positions
    t = (pos.double() * (-1.0 if back else 1.0))[..., None] * st["freq"]
    a = (1.0 / st["amplitude"] if back else st["amplitude"]) if amplitude else 1.0
    c, s = (torch.cos(t) * a).float(), (torch.sin(t) * a).float()
    one, two = (slice(0, dim, 2), slice(1, dim, 2)) if case["pairs"] else (slice(0, dim // 2), slice(dim // 2, dim))
    y = x.clone()
    y[..., one] = x[..., one] * c - x[..., two] * s
    y[..., two] = x[..., one] * s + x[..., two] * c
    return y


def _queries(st):
    q = _turned(st, st["q"].float(), st["positions"])
    if st["q_scale"] is None:
        return q.bfloat16()
    return _codes(q / st["q_scale"][:, None])


def _append_one(st, name):
    case, sb = st["case"], st["case"]["scale"]
    pool, scale, x = st[name], st[name + "_scale"], st[name + "_new"].float()
    if name == "k":
        x = _turned(st, x, st["positions"])
    if case["cache"] == "bf16":
        pool.index_copy_(0, st["new_slots"], x.bfloat16())
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


def _at(case, pool, scale, slot):
    """Values of the pool's tokens at `slot` [..., tokens] -> [..., tokens, hkv, D], in 32 bits."""
    if case["cache"] == "bf16":
        return pool[slot].float()
    x = _values(pool[slot])
    if not case["scale"]:
        return x * scale[:, None]
    return x * _power(scale[slot // case["scale"]].int() - 127)[..., None]


def _read(st):
    case, slot = st["case"], st["read_slots"]
    k, v = (_at(case, st[n], st[n + "_scale"], slot) for n in ("k", "v"))
    if case["undo"]:
        k = _turned(st, k, st["positions"], back=True)
    return k.bfloat16(), v.bfloat16()


def _move(st):
    case, sb, to = st["case"], st["case"]["scale"], st["target_slots"]
    for name in ("k", "v"):
        pool, scale = st[name], st[name + "_scale"]
        if name == "v" or (not case["each"] and case["start"] == 0):     # as they are
            pool.index_copy_(0, to, pool[st["slots"]])
            if sb:
                scale.index_copy_(0, st["hit"], scale[st["source_block"]])
            continue
        if case["cache"] == "bf16":
            x = _turned(st, pool[st["slots"]].float(), st["turns"], amplitude=False)
            pool.index_copy_(0, to, x.bfloat16())
        elif not sb:                 # the scale of a head stays, and the turn is linear
            x = _turned(st, _values(pool[st["slots"]]), st["turns"], amplitude=False)
            pool.index_copy_(0, to, _codes(x))
        else:
            x = _turned(st, _at(case, pool, scale, st["slots"]), st["turns"], amplitude=False)
            amax = torch.zeros((st["hit"].numel(), case["hkv"]), device=x.device).scatter_reduce_(
                0, st["block_of"][:, None].expand(-1, case["hkv"]), x.abs().amax(2), "amax")
            e = _exponent(amax)
            pool.index_copy_(0, to, _codes(x * _power(-e)[st["block_of"]][:, :, None]))
            scale.index_copy_(0, st["hit"], (e + 127).to(torch.uint8))


def _cross(st):
    case = st["case"]
    hq, hkv, page = case["hq"], case["hkv"], case["page"]
    nb, c = st["q_at"].shape
    key = torch.arange(st["columns"], device=st["q"].device)
    there = key < st["lens"][:, None]
    at = torch.where(there, key, 0)
    slot = st["table"].long().gather(1, at // page) * page + at % page
    k = _at(case, st["k"], st["k_scale"], slot).permute(0, 2, 3, 1).contiguous()
    q = st["q"][st["q_at"]].float().view(nb, c, hkv, hq // hkv, D).transpose(1, 2).reshape(nb, hkv, -1, D)
    x = torch.matmul(q, k).mul_(1.0 / math.sqrt(D))
    x.masked_fill_(~there[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp_min(-1e30)        # a sequence without keys: no NaN
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    v = _at(case, st["v"], st["v_scale"], slot).transpose(1, 2).contiguous()
    v.masked_fill_(~there[:, None, :, None], 0.0)
    out = torch.matmul(p, v).div_(total.clamp_min(1e-30))
    lse = torch.where(total > 0, top + total.log(), total.log())

    def rows(y):
        y = y.view(nb, hkv, c, hq // hkv, -1).transpose(1, 2)
        return y.reshape(nb * c, hq, -1)[st["rows"]]

    return rows(out).bfloat16(), rows(lse).squeeze(-1) if case["lse"] else None


def _as_numbers(x):
    """8-bit codes as the numbers that they are."""
    return x.view(torch.float8_e4m3fn) if x.dtype == torch.uint8 else x


def _pools(st):
    """The cache with its scales, as numbers."""
    got = {"k": _as_numbers(st["k"]), "v": _as_numbers(st["v"])}
    if st["case"]["scale"]:
        got.update({n + "_scale": st[n + "_scale"].view(torch.float8_e8m0fnu) for n in ("k", "v")})
    return got


def run(state):
    """One layer's call."""
    st, case, op = state, state["case"], state["case"]["op"]
    if own:
        import paper_2608_19758_amd as fp2
        lens = dict(cu_seqlens_host=st["cu_host"], cu_seqlens_k_host=st["cu_k_host"])
        if op == "rotary":
            q, k = fp2.rotary(st["rotary"], st["q"], st["positions"], st["k_new"], q_scale=st["q_scale"])
            return {"q": _as_numbers(q), "k": k}
        if op == "append":
            q = fp2.cache_append_rotary(st["p"], st["rotary"], st["q"], st["k_new"], st["v_new"], st["cache"], st["cu"],
                                        st["cu_k"], st["table"], positions=st["positions"] if case["start"] else None,
                                        q_scale=st["q_scale"], **lens)
            return {"q": _as_numbers(q), **_pools(st)}
        if op == "read":
            k, v = fp2.cache_read(st["p"], st["cache"], st["cu"], st["cu_k"], st["table"],
                                  rotary=st["rotary"] if case["undo"] else None, **lens)
            return {"k": k, "v": v}
        if op == "move":
            turn = case["each"] or case["start"] > 0
            fp2.cache_move(st["p"], st["cache"], st["cu_k"], st["table"], st["target"], rotary=st["rotary"] if turn else None,
                           moves=st["moves"] if turn else None, cu_seqlens_k_host=st["cu_k_host"])
            return _pools(st)
        out, lse = fp2.cache_cross(st["p"], st["q"], st["cache"], st["cu"], st["cu_k"], st["table"], want_lse=case["lse"],
                                   workspace=st["workspace"], **lens)
        return {"out": out, "lse": lse}
    if op == "rotary":
        return {"q": _as_numbers(_queries(st)), "k": _turned(st, st["k_new"].float(), st["positions"]).bfloat16()}
    if op == "append":
        q = _queries(st)
        _append_one(st, "k")
        _append_one(st, "v")
        return {"q": _as_numbers(q), **_pools(st)}
    if op == "read":
        k, v = _read(st)
        return {"k": k, "v": v}
    if op == "move":
        _move(st)
        return _pools(st)
    out, lse = _cross(st)
    return {"out": out, "lse": lse}


# ---------------------------------------------------------------------------
# The same from the definitions, in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    new, pre, kv = _shape(case)
    op, hq, hkv, page, sb, dim = (case[n] for n in ("op", "hq", "hkv", "page", "scale", "dim"))
    dev, freq, amp = st["freq"].device, st["freq"], st["amplitude"]

    def power(e):
        """2^e of whole numbers in 64 bits."""
        return ((e.long() + 1023) << 52).view(torch.float64)

    def nearest(x):
        """x rounded to e4m3's numbers, ties to even, and held within +-448."""
        x = x.clamp(-448, 448)
        step = torch.frexp(x.abs().clamp_min(2.0 ** -6)).exponent - 4     # numbers lie 2^step apart
        return torch.round(x * power(-step)) * power(step)

    def turn(x, pos, by):
        """Complex numbers times e^(i angle): pos [tokens] or [tokens, heads]."""
        angle = pos.double().view(len(x), -1, 1) * freq
        w = torch.polar(torch.full_like(angle, by), angle)
        if case["pairs"]:
            y = torch.view_as_complex(x[..., :dim].reshape(*x.shape[:2], -1, 2).contiguous()) * w
            y = torch.view_as_real(y).reshape(*x.shape[:2], dim)
        else:
            y = torch.complex(x[..., :dim // 2].contiguous(), x[..., dim // 2:dim].contiguous()) * w
            y = torch.cat([y.real, y.imag], dim=-1)
        return torch.cat([y, x[..., dim:]], dim=-1)

    def exponents(tops):
        """The smallest e with 2^e >= tops / 448, within [-100, 118]."""
        e = torch.ceil(torch.log2((tops / 448.0).clamp_min(2.0 ** -120))).long()
        e = torch.where(power(e - 1) * 448.0 >= tops, e - 1, e)
        e = torch.where(power(e) * 448.0 < tops, e + 1, e)
        return e.clamp(-100, 118)

    def slots_of(b, first, last, table="table"):
        j = torch.arange(first, last, device=dev)
        return st[table][b].long()[j // page] * page + j % page

    def stands_for(name, slot):
        x = st[name][slot]
        if case["cache"] == "bf16":
            return x.double()
        x = x.view(torch.float8_e4m3fn).double()
        if not sb:
            return x * st[name + "_scale"].double()[:, None]
        return x * power(st[name + "_scale"][slot // sb].int() - 127)[..., None]

    def query_rows():
        q = turn(st["q"].double(), st["positions"], amp)
        return q if st["q_scale"] is None else nearest(q / st["q_scale"].double()[:, None])

    if op == "rotary":
        return {"q": query_rows(), "k": turn(st["k_new"].double(), st["positions"], amp)}
    if op == "read":
        k, v = (torch.cat([stands_for(n, slots_of(b, p, t)) for b, (p, t) in enumerate(zip(pre, kv))]) for n in ("k", "v"))
        if case["undo"]:
            k = turn(k, -st["positions"].double(), 1.0 / amp)
        return {"k": k, "v": v}
    if op == "cross":
        out = torch.zeros((sum(new), hq, D), dtype=torch.float64, device=dev)
        lse = torch.full((sum(new), hq), -math.inf, dtype=torch.float64, device=dev)
        if sum(n * t for n, t in zip(new, kv)) * hq > 6e9:
            return None
        row = 0
        for b, (n, t) in enumerate(zip(new, kv)):
            if t and n:
                k, v = stands_for("k", slots_of(b, 0, t)), stands_for("v", slots_of(b, 0, t))
                for a in range(hq):
                    h = a // (hq // hkv)
                    for i in range(0, n, 2048):
                        some = slice(row + i, row + min(i + 2048, n))
                        x = st["q"][some, a].double() @ k[:, h].t() / math.sqrt(D)
                        z = torch.logsumexp(x, dim=1)
                        out[some, a] = torch.exp(x - z[:, None]) @ v[:, h]
                        lse[some, a] = z
            row += n
        return {"out": out, "lse": lse if case["lse"] else None}

    # pools after an append or a move
    got, scales = {}, {}
    for name in ("k", "v"):
        got[name] = st[name].double() if case["cache"] == "bf16" else st[name].view(torch.float8_e4m3fn).double()
        scales[name] = None if not sb else st[name + "_scale"].long() - 127
    if op == "append":
        rows = {"k": turn(st["k_new"].double(), st["positions"], amp), "v": st["v_new"].double()}
        got["q"] = query_rows()
    elif sum(kv) * hkv > 6000000:
        return None
    row = 0
    for b, (n, p, t) in enumerate(zip(new, pre, kv)):
        for name in ("k", "v"):
            if op == "append":
                x, first, to = rows[name][row:row + n], p, slots_of(b, p, t)
            else:
                x, first, to = stands_for(name, slots_of(b, 0, t)), 0, slots_of(b, 0, t, "target")
                if name == "k" and (case["each"] or case["start"]):
                    m = st["moves"][b, :, :t].t() if case["each"] else st["moves"][b].expand(t, 1)
                    x = turn(x, m, 1.0)
                else:                    # as they are
                    got[name][to] = got[name][slots_of(b, 0, t)]
                    if sb:
                        scales[name][to // sb] = scales[name][slots_of(b, 0, t) // sb]
                    continue
            if not len(x):
                continue
            if case["cache"] == "bf16":
                got[name][to] = x
            elif not sb:
                got[name][to] = nearest(x / st[name + "_scale"].double()[:, None])
            else:
                skip = first % sb        # tokens that the first block holds already
                pad = -(skip + len(x)) % sb
                tops = torch.nn.functional.pad(x.abs().amax(2), (0, 0, skip, pad)).view(-1, sb, hkv).amax(1)
                e = exponents(tops)
                blocks = torch.nn.functional.pad(to, (skip, pad), value=-1).view(-1, sb).amax(1) // sb
                if skip:
                    old = slots_of(b, first - skip, first)
                    was = scales[name][blocks[0]]
                    e[0] = torch.maximum(e[0], was)
                    got[name][old] = nearest(got[name][old] * power(was - e[0])[:, None])
                scales[name][blocks] = e
                got[name][to] = nearest(x * power(-e).repeat_interleave(sb, dim=0)[skip:skip + len(x), :, None])
        row += n
    if sb:
        got.update({n + "_scale": power(scales[n]) for n in ("k", "v")})
    return got

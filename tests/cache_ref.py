"""The paged cache's operators in 64 bits on the CPU, from their definitions, and
inputs for their tests. Slots that no sequence owns hold NaN."""
import math

import numpy as np
import torch

D = 128
EPS16 = 2.0 ** -8          # largest relative rounding to bf16
U32 = 2.0 ** -24           # and to fp32


def e4m3_values():
    """The number of each of the 256 codes (NaN at 0x7f and 0xff)."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v[(c & 0x7f) == 0x7f] = np.nan
    return np.where(c >= 128, -v, v)


VALUES = e4m3_values()


def to_codes(x):
    """Nearest codes of numbers in +-448, ties to the even code; NaN code for what is not finite."""
    x = np.asarray(x, np.float64)
    bad = ~np.isfinite(x)
    y = np.clip(np.where(bad, 0.0, x), -448, 448)
    a = np.abs(y)
    e = np.maximum(np.frexp(np.maximum(a, 2.0 ** -6))[1] - 1, -6)
    steps = np.rint(a / 2.0 ** (e - 3.0)).astype(np.int64)          # rint: ties to even
    code = np.where(a < 2.0 ** -6, steps, ((e + 7) << 3) + steps - 8)
    code = np.where(np.signbit(y), code | 0x80, code)
    return np.where(bad, 0x7f, code).astype(np.uint8)


def exponent_for(amax):
    """e of the smallest 2^e >= amax / 448, within [-100, 118]."""
    if amax == 0:
        return -100
    e = math.ceil(math.log2(amax / 448.0))
    while 448.0 * 2.0 ** (e - 1) >= amax:
        e -= 1
    while 448.0 * 2.0 ** e < amax:
        e += 1
    return min(118, max(-100, e))


class Cache:
    """A pool with `lens` tokens of each sequence, pages in any order."""

    def __init__(self, lens, hkv, form, page, room=0, seed=0, spread=0.0):
        """form: "bf16", "head" or the tokens per scale. room: tokens that a sequence may grow by."""
        self.rng = np.random.default_rng(seed)
        r = self.rng
        self.lens, self.hkv, self.form, self.page = list(lens), hkv, form, page
        self.sb = form if isinstance(form, int) else 0
        self.width = max(1, max(-(-(n + room) // page) for n in lens))
        self.pages = len(lens) * self.width + 3
        self.table = np.full((len(lens), self.width), 2 ** 30, np.int32)    # never read past a sequence
        order = r.permutation(self.pages)
        at = 0
        for b, n in enumerate(lens):
            need = -(-(n + room) // page)
            self.table[b, :need] = order[at:at + need]
            at += need
        self.free = order[at:]
        slots = self.pages * page
        self.k, self.v, self.ks, self.vs = None, None, None, None
        for name in ("k", "v"):
            x = r.standard_normal((slots, hkv, D)) * np.exp(spread * r.standard_normal((slots // 16 + 1, hkv, 1))
                                                             ).repeat(16, axis=0)[:slots]
            if form == "bf16":
                pool = torch.from_numpy(x).bfloat16()
                scale = None
            elif form == "head":
                scale = torch.from_numpy((np.abs(x).max((0, 2)) / 448.0).astype(np.float32))
                pool = torch.from_numpy(to_codes(x / scale.numpy()[None, :, None]))
            else:
                amax = np.abs(x).reshape(-1, self.sb, hkv, D).max((1, 3))
                e = np.vectorize(exponent_for)(amax)
                scale = torch.from_numpy((e + 127).astype(np.uint8))
                pool = torch.from_numpy(to_codes(x / 2.0 ** e.repeat(self.sb, axis=0)[:, :, None].astype(np.float64)))
            own = np.zeros(slots, bool)
            for b, n in enumerate(lens):
                own[self.slots(b, np.arange(n))] = True
            if form == "bf16":
                pool[torch.from_numpy(~own)] = float("nan")
            else:
                pool[torch.from_numpy(~own)] = 0x7f
                if self.sb:
                    scale[torch.from_numpy(~own.reshape(-1, self.sb).any(1))] = 255
            setattr(self, name, pool)
            setattr(self, name + "s", scale)

    def slots(self, b, t, table=None):
        t = np.asarray(t, np.int64)
        table = self.table if table is None else table
        return table[b][t // self.page].astype(np.int64) * self.page + t % self.page

    def values(self, name, slots, h):
        """Numbers of head h at the slots, [n, D] in 64 bits."""
        pool, scale = getattr(self, name), getattr(self, name + "s")
        if self.form == "bf16":
            return pool[slots, h].double().numpy()
        x = VALUES[pool[slots, h].numpy()]
        if self.form == "head":
            return x * float(scale[h])
        return x * 2.0 ** (scale[slots // self.sb, h].numpy().astype(np.float64) - 127)[:, None]


def sees(pos, keys, window, sink):
    d = pos[:, None] - keys[None, :]
    m = d >= 0
    return m & ((d < window) | (keys[None, :] < sink)) if window else m


def attend(c, q, new, window=0, sink=0, scale=None, lse_in=None):
    """out, its tolerance, lse, its tolerance and the weights [batch][hkv][L] with theirs."""
    hq, g = q.shape[1], q.shape[1] // c.hkv
    scale = 1 / math.sqrt(D) if scale is None else scale
    qd = q.double().numpy()
    out, tol = np.zeros(qd.shape), np.zeros(qd.shape)
    lse, ltol = np.zeros(qd.shape[:2]), np.zeros(qd.shape[:2])
    weights = [np.zeros((2, c.hkv, n)) for n in c.lens]
    row = 0
    for b, (n, L) in enumerate(zip(new, c.lens)):
        pos, keys = np.arange(L - n, L), np.arange(L)
        m = sees(pos, keys, window, sink)
        for h in range(c.hkv if n else 0):
            used = m.any(0)
            k = np.where(used[:, None], c.values("k", c.slots(b, keys), h), 0.0)
            v = np.where(used[:, None], c.values("v", c.slots(b, keys), h), 0.0)
            odd = ~np.isfinite(v)
            fin = np.where(odd, 0.0, v)
            for a in range(h * g, h * g + g):
                x = qd[row:row + n, a] @ k.T * scale
                # fp32 products summed in any order, then an exponential of a number of that size
                err = (130 * U32 * scale) * (np.abs(qd[row:row + n, a]) @ np.abs(k).T) + 8 * U32 * (1 + np.abs(x))
                x = np.where(m, x, -np.inf)
                top = x.max(1, keepdims=True)
                p = np.exp(x - top)
                s = p.sum(1, keepdims=True)
                z = top[:, 0] + np.log(s[:, 0])
                p /= s
                far = np.where(m, err, 0).max(1, keepdims=True)
                size = p @ np.abs(fin)
                o = p @ fin
                # each probability rounded to bf16, then the output; scores off by `far` twice (row and sum);
                # sums of fp32 in any order
                t = EPS16 * (size + np.abs(o)) * 1.01 + (2.2 * far + (L + 64) * U32) * size + 1e-37
                for j, d in zip(*np.nonzero(odd)):
                    o[m[:, j], d] += v[j, d]
                sl = slice(row, row + n)
                out[sl, a], tol[sl, a] = o, t
                lse[sl, a] = z
                ltol[sl, a] = far[:, 0] + (L + 64) * U32 + 4 * U32 * np.abs(z)
                ref = z if lse_in is None else lse_in[sl, a]
                w = np.where(m, np.exp(x - ref[:, None]), 0.0)
                weights[b][0, h] += w.sum(0)
                weights[b][1, h] += (w * (far + 8 * U32 * (1 + np.abs(ref)[:, None]))).sum(0) * 1.1
        row += n
    for w in weights:
        w[1] += (w[0] * (len(q) * g + 64)) * U32 + 1e-37
    return out, tol, lse, ltol, weights


def append(c, k_new, v_new, new):
    """The pools and scales after the append (c.lens count the new tokens)."""
    got = {}
    for name, x in (("k", k_new), ("v", v_new)):
        pool, scale = getattr(c, name).clone(), getattr(c, name + "s")
        scale = None if scale is None else scale.clone()
        row = 0
        for b, (n, L) in enumerate(zip(new, c.lens)):
            P = L - n
            if c.form == "bf16":
                pool[c.slots(b, np.arange(P, L))] = x[row:row + n]
            elif c.form == "head" and n:
                y = x[row:row + n].float() / scale[None, :, None]          # fp32, rounded to nearest
                y = torch.where(x[row:row + n].isfinite(), y.double(), float("nan"))
                pool[c.slots(b, np.arange(P, L))] = torch.from_numpy(to_codes(y.numpy()))
            elif n:
                for t0 in range(P // c.sb * c.sb, L, c.sb):
                    a, z = max(t0, P), min(t0 + c.sb, L)
                    new_at, old_at = c.slots(b, np.arange(a, z)), c.slots(b, np.arange(t0, a))
                    blk = new_at[0] // c.sb
                    y = x[row + a - P:row + z - P].double().numpy()
                    for h in range(c.hkv):
                        f = np.abs(y[:, h])
                        e = exponent_for(np.where(np.isfinite(f), f, 0).max())
                        if t0 < P:
                            was = int(scale[blk, h]) - 127
                            e = max(e, was)
                            old = VALUES[pool[old_at, h].numpy()]
                            pool[old_at, h] = torch.from_numpy(np.where(np.isnan(old), 0x7f, to_codes(old * 2.0 ** (was - e))).astype(np.uint8)) \
                                if e > was else pool[old_at, h]
                        pool[new_at, h] = torch.from_numpy(to_codes(y[:, h] * 2.0 ** -e))
                        scale[blk, h] = e + 127
            row += n
        got[name], got[name + "s"] = pool, scale
    return got


def keep(w, L, budget, sink, recent):
    """Indexes that stay of a head with weights w[:L]."""
    if L <= budget:
        return np.arange(L)
    w = np.where(np.isnan(w[:L]), -np.inf, w[:L].astype(np.float64))
    rest = np.arange(sink, L - recent)
    heavy = rest[np.argsort(-w[rest], kind="stable")][:budget - sink - recent]
    return np.sort(np.concatenate([np.arange(sink), heavy, np.arange(L - recent, L)])).astype(np.int64)


def evict(c, weights, target, budget, sink, recent):
    """kept, weights and the pools and scales after the eviction to the pages `target`."""
    got = {n: (None if getattr(c, n) is None else getattr(c, n).clone()) for n in ("k", "v", "ks", "vs")}
    kept = np.full((len(c.lens), c.hkv, budget), -1, np.int32)
    left = np.zeros(weights.shape, np.float32)
    for b, L in enumerate(c.lens):
        for h in range(c.hkv):
            at = keep(weights[b, h], L, budget, sink, recent)
            kept[b, h, :len(at)] = at
            left[b, h, :len(at)] = weights[b, h, at]
            to = c.slots(b, np.arange(len(at)), target)
            src = c.slots(b, at)
            for n in ("k", "v"):
                if not c.sb:
                    got[n][to, h] = getattr(c, n)[src, h]
                    continue
                x = c.values(n, src, h)
                for i in range(0, len(at), c.sb):
                    y = x[i:i + c.sb]
                    e = exponent_for(np.nan_to_num(np.abs(y), nan=0.0).max())
                    got[n][to[i:i + c.sb], h] = torch.from_numpy(to_codes(y * 2.0 ** -e))
                    got[n + "s"][to[i] // c.sb, h] = e + 127
    return kept, left, got

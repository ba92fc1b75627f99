"""Rotary positions and what goes with them in 64 bits on the CPU, from the definitions, with
bounds of the kernels' errors (derived below, before any run)."""
import math

import numpy as np
import torch

from tests import cache_ref as ref

D = 128
U = 2.0 ** -24            # half a step of fp32, relative

# The kernels' sines and cosines are off by at most 2^-23.7, 1.3 U (an angle cut at 2^-32 turns, 2^-29.3, among
# it); their scale and the two products and the sum lose U each. In all below 10 U of |x| + |y| times the scale.
# Frequencies of 64 bits lose 2^-51 of the angle itself.
TURN = 10 * U


def turn(x, pos, freq, interleaved, scale=1.0, back=False):
    """x [..., D] at positions pos (of x's leading shape); the result and the bound of the fp32 error."""
    x = np.asarray(x, np.float64)
    h = len(freq)
    one = np.arange(h) * 2 if interleaved else np.arange(h)
    two = one + 1 if interleaved else one + h
    t = np.asarray(pos, np.float64)[..., None] * freq * (-1.0 if back else 1.0)
    a = 1.0 / scale if back else scale
    y, err = x.copy(), np.zeros(x.shape)
    with np.errstate(invalid="ignore"):
        y[..., one] = a * (x[..., one] * np.cos(t) - x[..., two] * np.sin(t))
        y[..., two] = a * (x[..., one] * np.sin(t) + x[..., two] * np.cos(t))
        e = a * (np.abs(x[..., one]) + np.abs(x[..., two])) * (TURN + np.abs(t) * 2.0 ** -51)
    err[..., one] = err[..., two] = e
    return y, err


def check_bf16(got, want, err, what):
    """A bf16 result of values that fp32 has `err` off."""
    got = got.double().cpu().numpy()
    fin = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what + ": NaN in other places"
    assert np.array_equal(got[~fin & ~np.isnan(want)], want[~fin & ~np.isnan(want)]), what + ": infinities"
    w, e = want[fin], err[fin]
    over = np.abs(got[fin] - w) / (2.0 ** -8 * (np.abs(w) + e) + e + 2.0 ** -134)
    print("%s: largest error %.3f of its bound" % (what, over.max() if over.size else 0), flush=True)
    assert not (over > 1).any(), what


def check_codes(codes, want, err, what):
    """Codes: each between those that want - err and want + err are rounded to."""
    got = ref.VALUES[codes.cpu().numpy()]
    fin = np.isfinite(want)
    assert np.array_equal(np.isnan(got), ~fin), what + ": NaN in other places"
    lo = ref.VALUES[ref.to_codes(np.where(fin, want - err, 0.0))]
    hi = ref.VALUES[ref.to_codes(np.where(fin, want + err, 0.0))]
    bad = fin & ~((got >= lo) & (got <= hi))
    assert not bad.any(), "%s: %d codes of %d" % (what, bad.sum(), bad.size)


def check_block(codes, byte, want, err, what, least=-100):
    """Codes [tokens, D] of one block and its scale's byte: the power of two of the largest, then each code."""
    e = int(byte) - 127
    size = np.where(np.isfinite(want), np.abs(want), 0.0)
    lo, hi = (size - err).max(initial=0.0, where=np.isfinite(want)), (size + err).max(initial=0.0, where=np.isfinite(want))
    allowed = {max(least, ref.exponent_for(max(lo, 0.0))), max(least, ref.exponent_for(hi))}
    assert e in allowed, "%s: scale 2^%d, wants %s" % (what, e, sorted(allowed))
    check_codes(codes, want * 2.0 ** -e, err * 2.0 ** -e, what)


def cross(c, q, new, scale=None):
    """Attention over all keys: out, its tolerance, lse, its tolerance (as tests/cache_ref.attend)."""
    hq, g = q.shape[1], q.shape[1] // c.hkv
    scale = 1 / math.sqrt(D) if scale is None else scale
    qd = q.double().numpy()
    out, tol = np.zeros(qd.shape), np.full(qd.shape, 1e-37)
    lse, ltol = np.full(qd.shape[:2], -np.inf), np.ones(qd.shape[:2])
    row = 0
    for b, (n, L) in enumerate(zip(new, c.lens)):
        for h in range(c.hkv if n and L else 0):
            k, v = c.values("k", c.slots(b, np.arange(L)), h), c.values("v", c.slots(b, np.arange(L)), h)
            for a in range(h * g, h * g + g):
                sl = slice(row, row + n)
                x = qd[sl, a] @ k.T * scale
                err = (130 * U * scale) * (np.abs(qd[sl, a]) @ np.abs(k).T) + 8 * U * (1 + np.abs(x))
                top = x.max(1, keepdims=True)
                p = np.exp(x - top)
                s = p.sum(1, keepdims=True)
                z = top[:, 0] + np.log(s[:, 0])
                p /= s
                far = err.max(1, keepdims=True)
                with np.errstate(invalid="ignore"):
                    size, o = p @ np.abs(v), p @ v
                # each probability rounded to bf16, then the output; scores off by `far` twice; sums of fp32
                out[sl, a], tol[sl, a] = o, ref.EPS16 * (size + np.abs(o)) * 1.01 + (2.2 * far + (L + 64) * U) * size + 1e-37
                lse[sl, a] = z
                ltol[sl, a] = far[:, 0] + (L + 64) * U + 4 * U * np.abs(z)
        row += n
    return out, tol, lse, ltol

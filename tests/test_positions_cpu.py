"""Rotary positions, reading back, moving and cross attention without a GPU: refusals before any
launch, frequencies, and the reference that the GPU tests use."""
import copy
import ctypes
import dataclasses
import math
import pickle

import numpy as np
import pytest
import torch

import paper_2608_19758_amd as fp2
from paper_2608_19758_amd import positions as fpos
from tests import cache_ref as ref
from tests import positions_ref as pos_ref
from tests.test_cache_cpu import FAKE, base, pointers

FAR = 1 << 40        # fake tensors lie this far apart


def turns(**kw):
    d = dict(turns=FAKE, dim=128, interleaved=0, scale=1.0)
    d.update(kw)
    return fpos._RotaryArgs(**d)


def rows(n=0, **kw):
    d = dict(x=FAKE + n * FAR, x_stride=32 * 128, out=FAKE + (n + 8) * FAR, out_stride=32 * 128, heads=32, out_dtype=fp2.BF16,
             out_scale=None)
    d.update(kw)
    return fpos._RotaryRows(**d)


def call(op, p=None, **over):
    a = dict(rotary=turns(), tokens=4, positions=FAKE + 20 * FAR, inverse=0, q=rows(0), k=rows(1, heads=8), k_new=FAKE + 2 * FAR,
             ks=1024, v_new=FAKE + 3 * FAR, vs=1024, cu=FAKE, cuh=None, cuk=FAKE, cukh=None, cache=pointers(), table=FAKE,
             k_out=FAKE, v_out=FAKE + FAR, moves=FAKE, strides=(1, 0, 0), target=2 * FAKE, pages=64, cq=FAKE, out=FAKE + FAR,
             lse=FAKE + 2 * FAR, ws=None, wsb=0)
    a.update(over)
    by = lambda x: None if x is None else ctypes.byref(x)      # noqa: E731
    held = [np.asarray(a[n], np.int32) if a[n] is not None else None for n in ("cuh", "cukh")]
    cuh, cukh = (None if x is None else x.ctypes.data for x in held)
    L, rot, c = fp2.lib(), by(a["rotary"]), by(a["cache"])
    if op == "rotary":
        return L.fp2_rotary(rot, a["tokens"], a["positions"], a["inverse"], by(a["q"]), by(a["k"]), None)
    if op == "append":
        return L.fp2_cache_append_rotary(by(p), rot, by(a["q"]), a["k_new"], a["ks"], a["v_new"], a["vs"], a["positions"],
                                         a["cu"], cuh, a["cuk"], cukh, c, a["table"], None)
    if op == "read":
        return L.fp2_cache_read(by(p), rot, a["positions"], a["cu"], cuh, a["cuk"], cukh, c, a["table"], a["k_out"],
                                a["v_out"], None)
    if op == "move":
        return L.fp2_cache_move(by(p), rot, a["moves"], *a["strides"], a["cuk"], cukh, c, a["table"], a["target"], a["pages"],
                                None)
    return L.fp2_cache_cross(by(p), a["cq"], a["cu"], cuh, a["cuk"], cukh, c, a["table"], a["out"], a["lse"], a["ws"],
                             a["wsb"], None)


@pytest.mark.parametrize("kw", [dict(dim=0), dict(dim=3), dict(dim=130), dict(dim=-2), dict(turns=None), dict(turns=FAKE + 4),
                                dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
                                dict(scale=1e-40)])
@pytest.mark.parametrize("op", ["rotary", "append", "read", "move"])
def test_bad_rotary(op, kw):
    assert call(op, base(), rotary=turns(**kw)) == fp2.EINVAL
    assert "rotary" in fp2.last_error()


@pytest.mark.parametrize("over", [
    dict(rotary=None), dict(q=None), dict(tokens=-1), dict(inverse=2), dict(positions=None),
    dict(q=rows(0, x=None)), dict(q=rows(0, out=None)), dict(q=rows(0, x=FAKE + 8)), dict(q=rows(0, out=FAKE + 2)),
    dict(q=rows(0, x_stride=4095)), dict(q=rows(0, x_stride=4088)), dict(q=rows(0, out_stride=128)), dict(q=rows(0, heads=0)),
    dict(q=rows(0, heads=8193, x_stride=1 << 21, out_stride=1 << 21)), dict(q=rows(0, out_dtype=2)),
    dict(q=rows(0, out_dtype=fp2.FP8_E4M3)), dict(q=rows(0, out_dtype=fp2.FP8_E4M3, out_scale=FAKE, out_stride=4104)),
    dict(k=rows(1, x=None)),
    # outputs that meet what is read
    dict(q=rows(0, out=FAKE + 256)), dict(q=rows(0, out=FAKE + 4096, x_stride=8192, out_stride=8192)),
    dict(q=rows(0, out=FAKE, out_stride=8192)), dict(q=rows(0, out=FAKE, out_dtype=fp2.FP8_E4M3, out_scale=FAKE)),
    dict(q=rows(0, out=FAKE + FAR)), dict(k=rows(1, heads=8, out=FAKE + 8 * FAR)), dict(k=rows(1, heads=8, out=FAKE + 128)),
    dict(q=rows(0, out=FAKE + 20 * FAR)),
])
def test_bad_rows(over):
    assert call("rotary", **over) == fp2.EINVAL


def test_too_many_tokens():
    assert call("rotary", tokens=1 << 31) == fp2.EUNSUPPORTED
    assert call("rotary", tokens=(1 << 31) - 1, k=None, q=rows(0, x=FAKE, out=FAKE, heads=8192, x_stride=1 << 20,
                                                               out_stride=1 << 20), positions=FAKE - (1 << 15) * 4) == fp2.EINVAL
    assert call("rotary", tokens=(1 << 31) - 1, k=None, positions=FAKE + (1 << 55),
                q=rows(0, x=FAKE, out=FAKE, heads=8192, x_stride=1 << 20, out_stride=1 << 20)) == fp2.EUNSUPPORTED
    assert "threads" in fp2.last_error()


def test_no_tokens():
    assert call("rotary", tokens=0, positions=None, q=rows(0, x=None, out=None), k=None) == fp2.OK
    for op in ("append", "read", "move", "cross"):
        assert call(op, base(batch=0), cu=None, cuk=None, cache=None, table=None) == fp2.OK, op
    for op in ("append", "read", "cross"):
        assert call(op, base(max_seq_len=0), cu=None, cuk=None, cache=None, table=None) == fp2.OK, op
    assert call("move", base(max_seq_len=0, max_kv_len=0), cuk=None, cache=None, table=None) == fp2.OK


OPS = ["append", "read", "move", "cross"]


@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), fp2.EINVAL), (dict(batch=65537), fp2.EUNSUPPORTED), (dict(num_kv_heads=0), fp2.EINVAL),
    (dict(num_q_heads=48), fp2.EUNSUPPORTED), (dict(head_dim=64), fp2.EUNSUPPORTED), (dict(page_size=0), fp2.EINVAL),
    (dict(max_pages_per_seq=63), fp2.EINVAL), (dict(max_kv_len=(1 << 20) + 1), fp2.EUNSUPPORTED), (dict(dtype=5), fp2.EINVAL),
    (dict(scale_tokens=8), fp2.EUNSUPPORTED), (dict(scale_tokens=128), fp2.EINVAL), (dict(max_seq_len=-1), fp2.EINVAL)])
@pytest.mark.parametrize("op", OPS)
def test_bad_params(op, kw, status):
    assert call(op, base(**kw)) == status
    assert fp2.lib().fp2_cache_cross_workspace_bytes(ctypes.byref(base(**kw))) == 0


@pytest.mark.parametrize("op,over", [(op, o) for op in OPS for o in (
    dict(cuk=None), dict(cache=None), dict(cache=pointers(k=None)), dict(cache=pointers(k=FAKE + 8)), dict(table=None),
    dict(cache=pointers(k_block_scale=None)), dict(cukh=[1, 2, 3]), dict(cukh=[0, 5000, 5001]), dict(cukh=[0, 9, 3]))] + [
    ("append", o) for o in (
        dict(cu=None), dict(cuh=[0, 5, 6]), dict(cuh=[0, 4, 8], cukh=[0, 3, 100]), dict(k_new=None), dict(v_new=None),
        dict(ks=1020), dict(ks=1000), dict(vs=512), dict(k_new=FAKE + 8), dict(rotary=None), dict(cache=pointers(v=None)),
        dict(q=rows(0, heads=31, x_stride=4096)), dict(q=rows(0, x=None)), dict(q=rows(0, out_dtype=fp2.FP8_E4M3)),
        dict(cuh=[0, 2, 4], q=rows(0, out=FAKE + 2 * FAR)), dict(cuh=[0, 2, 4], q=rows(0, out=FAKE + 3 * FAR + 1024)),
        dict(cuh=[0, 2, 4], q=rows(0, out=FAKE + 16)), dict(cuh=[0, 2, 4], q=rows(0, out=FAKE + 20 * FAR)))] + [
    ("read", o) for o in (
        dict(cu=None), dict(k_out=None, v_out=None), dict(k_out=FAKE + 2), dict(v_out=FAKE + FAR + 4), dict(rotary=None),
        dict(cuh=[0, 2, 4], v_out=FAKE + 4 * 2048 - 16), dict(cuh=[0, 4, 8], cukh=[0, 3, 100]), dict(cache=pointers(v=None)))] + [
    ("move", o) for o in (
        dict(moves=None), dict(rotary=None), dict(rotary=None, moves=None, target=None), dict(strides=(-1, 0, 0)),
        dict(strides=(0, 0, -4)), dict(pages=63), dict(target=FAKE), dict(cache=pointers(v=None)))] + [
    ("cross", o) for o in (
        dict(cu=None), dict(cq=None), dict(out=None), dict(out=FAKE), dict(cq=FAKE + 4), dict(cuh=[0, 2, 4], out=FAKE + 1024),
        dict(cuh=[0, 2, 4], lse=FAKE + 1024), dict(cuh=[0, 5, 6]), dict(cache=pointers(v=None)))])
def test_bad_arguments(op, over):
    assert call(op, base(), **over) == fp2.EINVAL


def test_parts_of_one_matrix_do_not_meet():
    """Rows beside each other in one matrix, in place. With so many tokens what is accepted ends at the launch's limit."""
    wide, many = 48 * 128, (1 << 31) - 1
    there = dict(tokens=many, positions=FAKE + (1 << 50), q=rows(0, x=FAKE, out=FAKE, x_stride=wide, out_stride=wide))

    def beside(at, heads=8):
        return call("rotary", **there, k=rows(1, x=FAKE + at, out=FAKE + at, x_stride=wide, out_stride=wide, heads=heads))

    assert beside(8192) == beside(2 * wide - 2048) == fp2.EUNSUPPORTED
    assert beside(8192 - 16) == beside(2 * wide - 2048 + 16) == beside(2 * wide - 16) == beside(8192, 17) == fp2.EINVAL


def test_cross_bounds_and_workspace():
    """Queries have a bound of their own; windows and more than it are refused; the workspace is asked for."""
    assert call("cross", base(window_tokens=5)) == fp2.EINVAL
    assert call("cross", base(sink_tokens=1)) == fp2.EINVAL
    assert call("cross", base(max_seq_len=(1 << 20) + 1)) == fp2.EUNSUPPORTED
    assert fp2.cross_workspace_bytes(base(window_tokens=5)) == 0
    p = base(batch=1, num_q_heads=4, num_kv_heads=1, max_seq_len=100, max_kv_len=20000)
    need = fp2.cross_workspace_bytes(p)
    assert 0 < need <= fp2.CACHE_WORKSPACE_MAX and need % 256 == 0
    for ws, size in ((None, need), (FAKE + 128, need), (FAKE, need - 1)):
        assert call("cross", p, ws=ws, wsb=size) == fp2.EWORKSPACE
    longer = base(max_seq_len=9000, max_kv_len=100)
    assert call("cross", longer, cuh=[0, 9000, 9001], cukh=[0, 0, 100], cache=None) == fp2.EINVAL   # lengths are fine, the cache is not
    assert "cache" in fp2.last_error()


@pytest.mark.parametrize("hkv,hq", [(8, 32), (1, 8), (8, 8), (4, 32)])
def test_cross_workspace_is_bounded(hkv, hq):
    """FP2_CACHE_WORKSPACE_MAX holds for every call that the library cuts by itself."""
    for batch in (1, 2, 3, 7, 16, 100, 1000):
        for new in (1, 2, 7, 8, 9, 64, 65, 300, 2000, 8192, 1 << 20):
            for kv in (0, 1, 100, 1500, 30000, 1 << 20):
                if batch * (kv + 4096) > 1 << 35:
                    continue
                p = base(batch=batch, num_q_heads=hq, num_kv_heads=hkv, max_seq_len=new, max_kv_len=kv)
                assert fp2.cross_workspace_bytes(p) <= fp2.CACHE_WORKSPACE_MAX, (batch, new, kv)


def test_launches_past_the_limit():
    """2^32 threads or more are refused before any launch."""
    big = dict(batch=65536, num_kv_heads=1024, num_q_heads=1024, max_kv_len=4096)
    assert call("append", base(**big, max_seq_len=9), q=None, ks=1 << 17, vs=1 << 17) == fp2.EUNSUPPORTED
    assert call("cross", base(batch=65536, num_kv_heads=1024, num_q_heads=1024, max_seq_len=4096, max_kv_len=64, kv_splits=1)) == fp2.EUNSUPPORTED


# ---- the binding

def cpu_rotary(dim=128, **kw):
    return fp2.make_rotary(dim, device="cpu", **kw)


def test_binding_refuses():
    r, q, at = cpu_rotary(), torch.zeros((4, 2, 128), dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    for bad in (q.float(), q[:, :, :64], q[0], q.transpose(0, 1), q[..., ::2].repeat(1, 1, 2)[:, :, ::1].transpose(1, 2), None, 3):
        with pytest.raises(ValueError):
            fp2.rotary(r, bad, at)
    for kw in (dict(positions=at.long()), dict(positions=at[:3]), dict(positions=at[::2]), dict(k=q[:3], positions=at),
               dict(out=q[:3], positions=at), dict(q_scale=torch.ones(1), positions=at), dict(q_scale=torch.ones(2).double(), positions=at),
               dict(out=q, q_scale=torch.ones(2), positions=at), dict(k=q, k_out=q.float(), positions=at)):
        with pytest.raises(ValueError):
            fp2.rotary(r, q, **kw)
    for bad in (None, dict(turns=1), r.turns):
        with pytest.raises(ValueError):
            fp2.rotary(bad, q, at)
    for bad in ((r.turns[:63], 128), (r.turns.int(), 128), (r.turns, 127), (r.turns, 130), (torch.zeros(8, dtype=torch.int64)[::2], 8), (None, 128), (r.turns, 2.0)):
        with pytest.raises(ValueError):
            fp2.Rotary(*bad)
    with pytest.raises(ValueError, match="CUDA tensor"):      # all else is right
        fp2.rotary(r, q, at)


def cpu_call():
    p = fp2.make_cache_params(batch=2, num_q_heads=4, num_kv_heads=2, max_seq_len=8, max_kv_len=32, page_size=16, dtype="fp8",
                              scale_tokens=16)
    cache = fp2.alloc_cache(p, 4, device="cpu")
    cu, cuk, table = torch.tensor([0, 3, 5], dtype=torch.int32), torch.tensor([0, 20, 30], dtype=torch.int32), torch.zeros((2, 2), dtype=torch.int32)
    return p, cache, (cu, cuk, table), dict(cu_seqlens_host=cu, cu_seqlens_k_host=cuk)


def test_cache_binding_refuses():
    p, cache, lens, host = cpu_call()
    r = cpu_rotary()
    q, k = torch.zeros((5, 4, 128), dtype=torch.bfloat16), torch.zeros((5, 2, 128), dtype=torch.bfloat16)
    ok = dict(rotary=r, moves=torch.zeros(2, dtype=torch.int32))
    target = torch.ones((2, 2), dtype=torch.int32)
    for args, kw in (((q[:4], k, k), {}), ((q, k[:4], k), {}), ((q, k, k[:4]), {}), ((q, q, k), {}), ((k, k, k), {}),
                     ((q[:4], k[:4], k[:4]), host), ((q, k, k), dict(positions=torch.zeros(4, dtype=torch.int32))),
                     ((q, k, k), dict(positions=torch.zeros(5))), ((q, k, k), dict(out=q[:, :2])), ((3, k, k), {})):
        with pytest.raises(ValueError):
            fp2.cache_append_rotary(p, r, *args, cache, *lens, **kw)
    for kw in (dict(), dict(keys=False, values=False, rows=5), dict(rows=4, **host), dict(rows=5, k_out=k[:4]),
               dict(k_out=k.float()), dict(rows=5, positions=torch.zeros(4, dtype=torch.int32), rotary=r),
               dict(rows=5, rotary=3), dict(k_out=q[:4])):
        with pytest.raises(ValueError):
            fp2.cache_read(p, cache, *lens, **kw)
    for kw in (dict(rotary=r), dict(moves=ok["moves"]), dict(ok, moves=ok["moves"].long()), dict(ok, moves=ok["moves"][:0]),
               dict(ok, moves=torch.zeros((2, 3, 1), dtype=torch.int32)), dict(ok, moves=torch.zeros((2, 2, 31), dtype=torch.int32)),
               dict(ok, moves=torch.zeros((2, 2), dtype=torch.int32)), dict(ok, target_table=target[0]), dict(ok, target_table=target.long())):
        with pytest.raises(ValueError):
            fp2.cache_move(p, cache, *lens[1:], **kw)
    for bad in (dict(q=q.float()), dict(out=q[:4]), dict(out=q), dict(lse=torch.zeros(3)), dict(cu_seqlens_host=lens[0][:2])):
        kw = dict(q=q, workspace=torch.zeros(1, dtype=torch.uint8))
        kw.update(bad)
        with pytest.raises(ValueError):
            fp2.cache_cross(p, cache=cache, cu_seqlens=lens[0], cu_seqlens_k=lens[1], block_table=lens[2], **kw)
    for go in (lambda: fp2.cache_append_rotary(p, r, q, k, k, cache, *lens, **host), lambda: fp2.cache_read(p, cache, *lens, **host),
               lambda: fp2.cache_move(p, cache, *lens[1:], target, **ok)):
        with pytest.raises(ValueError, match="CUDA tensor"):
            go()


def test_interleaved_is_0_or_1():
    for op in ("rotary", "append", "read", "move"):
        for bad in (2, -1):
            assert call(op, base(), rotary=turns(interleaved=bad)) == fp2.EINVAL
            assert "interleaved" in fp2.last_error()


def test_rotary_copies():
    """A copy's arguments are those of its own tensor."""
    r = cpu_rotary(64, interleaved=True, scale=1.5)
    for c in (copy.deepcopy(r), pickle.loads(pickle.dumps(r)), copy.copy(r), dataclasses.replace(r)):
        assert c._args.turns == c.turns.data_ptr() and torch.equal(c.turns, r.turns)
        assert (c.dim, c.interleaved, c.scale, c._args.dim, c._args.interleaved) == (64, True, 1.5, 64, 1)
    c = copy.deepcopy(r)
    assert c.turns.data_ptr() != r.turns.data_ptr() and c != r and r == r and len({r, c}) == 2


def test_append_output_overlap():
    """Queries out onto other rows of the call, without lengths on the host; parts of one matrix may be turned in place."""
    p, cache, lens, _ = cpu_call()
    r, m = cpu_rotary(), torch.zeros((6, 8, 128), dtype=torch.bfloat16)
    q, k, v = m[:5, :4], m[:5, 4:6], m[:5, 6:]
    for out in (m[:5, 1:5], m[:5, 4:8], m[1:, :4], m[1:, 2:6], m.view(-1, 4, 128)[:5]):
        with pytest.raises(ValueError, match="overlap"):
            fp2.cache_append_rotary(p, r, q, k, v, cache, *lens, out=out)
    for scale, codes in ((None, None), (torch.ones(4), m.view(torch.uint8).view(-1, 4, 128))):
        with pytest.raises(ValueError, match="CUDA tensor" if scale is None else "overlap"):
            fp2.cache_append_rotary(p, r, q, k, v, cache, *lens, out=q if scale is None else codes, q_scale=scale)
    with pytest.raises(ValueError, match="CUDA tensor"):
        fp2.cache_append_rotary(p, r, m[:5, :4], m[:5, 6:], m[:5, 6:], cache, *lens, out=m[:5, :4].clone())


# ---- frequencies

def test_frequencies():
    f, a = fp2.rotary_frequencies(128)
    assert a == 1.0 and f[0] == 1.0 and f.shape == (64,)
    np.testing.assert_allclose(f, [10000.0 ** (-2 * i / 128) for i in range(64)], rtol=1e-14)
    np.testing.assert_allclose(fp2.rotary_frequencies(64, 500000.0, scaling="linear", factor=4.0)[0],
                               [500000.0 ** (-i / 32) / 4 for i in range(32)], rtol=1e-14)
    b, a = fp2.rotary_frequencies(128, scaling="base", factor=8.0)
    assert b[0] == 1.0 and a == 1.0 and abs(b[63] / (f[63] / 8) - 1) < 1e-13         # the ends that its definition names
    n = 8192
    for scaling, low, high in (("bands", 1.0, 4.0), ("bands", 0.5, 20.0)):
        got, a = fp2.rotary_frequencies(128, 500000.0, scaling=scaling, factor=8.0, original_len=n, low=low, high=high)
        assert a == 1.0
        for i, x in enumerate(got):
            w = 500000.0 ** (-i / 64)
            t = n * w / (2 * math.pi)
            want = w if t >= high else w / 8 if t <= low else w * ((t - low) / (high - low)) + w / 8 * (1 - (t - low) / (high - low))
            assert abs(x / want - 1) < 1e-12
    got, a = fp2.rotary_frequencies(128, 10000.0, scaling="ramp", factor=4.0, original_len=n)
    assert abs(a - (0.1 * math.log(4) + 1)) < 1e-15
    lo = math.floor(64 * math.log(n / (2 * math.pi * 32)) / math.log(10000.0))
    hi = math.ceil(64 * math.log(n / (2 * math.pi * 1)) / math.log(10000.0))
    for i, x in enumerate(got):
        s = min(1.0, max(0.0, (i - lo) / (hi - lo)))
        assert abs(x / (f[i] / 4 * s + f[i] * (1 - s)) - 1) < 1e-12
    assert 0 < lo < hi < 64 and got[lo] == f[lo] and abs(got[hi] / (f[hi] / 4) - 1) < 1e-13


@pytest.mark.parametrize("kw", [dict(dim=3), dict(dim=0), dict(dim=130), dict(dim=2.0), dict(base=1.0), dict(base=float("nan")),
                                dict(factor=0.5), dict(factor=2.0), dict(scaling="other"), dict(scaling="ramp", factor=2.0),
                                dict(scaling="bands", factor=2.0, original_len=100, low=4.0), dict(dim=2, scaling="base", factor=2.0)])
def test_frequencies_refused(kw):
    kw = dict(dict(dim=128), **kw)
    with pytest.raises(ValueError):
        fp2.rotary_frequencies(kw.pop("dim"), **kw)


def test_make_rotary():
    """Fractions of a turn in fixed point: far positions come out as the frequencies say."""
    r = cpu_rotary(96, base=500000.0, interleaved=True)
    assert r.turns.shape == (48,) and r.turns.dtype == torch.int64 and r.interleaved and r.scale == 1.0
    f = fp2.rotary_frequencies(96, 500000.0)[0]
    for n in (1, -1, 1000, 2 ** 20):
        for x, t in zip(f, r.turns.tolist()):
            turn = (n * t % 2 ** 64) / 2.0 ** 64 * 2 * math.pi
            assert abs(math.cos(turn) - math.cos(n * x)) < 2e-9 and abs(math.sin(turn) - math.sin(n * x)) < 2e-9
    given = cpu_rotary(4, frequencies=torch.tensor([2 * math.pi * 1.25, -math.pi / 2], dtype=torch.float64))
    assert [t % 2 ** 64 for t in given.turns.tolist()] == [2 ** 62, 3 * 2 ** 62]
    assert cpu_rotary(128, scaling="ramp", factor=4.0, original_len=4096).scale == 1.0 + 0.1 * math.log(4.0)
    assert cpu_rotary(128, scaling="ramp", factor=4.0, original_len=4096, scale=1.0).scale == 1.0
    for kw in (dict(frequencies=[1.0] * 63), dict(frequencies=[float("inf")] * 64), dict(scale=0.0), dict(scale=float("nan")),
               dict(frequencies=[1.0] * 64, scaling="linear", factor=2.0)):
        with pytest.raises(ValueError):
            cpu_rotary(128, **kw)


def test_reference_turn():
    """The reference against complex numbers, and turns that add up."""
    g = np.random.default_rng(0)
    x, f = g.standard_normal((5, 128)), fp2.rotary_frequencies(64)[0]
    at = np.arange(5) * 7
    y, _ = pos_ref.turn(x, at, f, True, 2.0)
    z = (x[:, 0:64:2] + 1j * x[:, 1:64:2]) * np.exp(1j * at[:, None] * f) * 2.0
    np.testing.assert_allclose(y[:, 0:64:2] + 1j * y[:, 1:64:2], z, rtol=1e-13)
    assert np.array_equal(y[:, 64:], x[:, 64:])
    y, _ = pos_ref.turn(x, at, f, False)
    z = (x[:, :32] + 1j * x[:, 32:64]) * np.exp(1j * at[:, None] * f)
    np.testing.assert_allclose(y[:, :32] + 1j * y[:, 32:64], z, rtol=1e-13)
    two, _ = pos_ref.turn(y, at * 3, f, False)
    once, _ = pos_ref.turn(x, at * 4, f, False)
    np.testing.assert_allclose(two, once, atol=1e-12)
    back, _ = pos_ref.turn(pos_ref.turn(x, at, f, True, 1.7)[0], at, f, True, 1.7, back=True)
    np.testing.assert_allclose(back, x, atol=1e-12)


def test_reference_cross():
    """With one query that sees all keys it is the causal reference."""
    c = ref.Cache([50, 3], 2, 16, 16, seed=1)
    q = torch.randn((2, 4, 128)).bfloat16()
    a, b = pos_ref.cross(c, q, [1, 1]), ref.attend(c, q, [1, 1])
    np.testing.assert_allclose(a[0], b[0], rtol=1e-12)
    np.testing.assert_allclose(a[2], b[2], rtol=1e-12)


def test_plan_cross():
    """Queries and states are bounded apart from each other; windows of the config do not count."""
    from paper_2608_19758_amd import serving
    cfg = serving.CacheConfig(num_q_heads=8, num_kv_heads=2, page_size=16, max_batch=3, max_extend_len=50, max_kv_len=100,
                              window_tokens=10, sink_tokens=2)
    plan = serving.plan_cross(cfg, [50, 0, 7], [0, 100, 3])
    p = plan.params
    assert (p.batch, p.max_seq_len, p.max_kv_len, p.window_tokens, p.sink_tokens) == (3, 50, 100, 0, 0)
    assert plan.cu_q.tolist() == [0, 50, 50, 57] and plan.cu_k.tolist() == [0, 0, 100, 103] and plan.total_tokens == 57
    assert plan.cu_q.dtype == plan.cu_k.dtype == np.int32
    for new, kv in (([51], [1]), ([1], [101]), ([-1], [1]), ([1], [-1]), ([1, 1], [1]), ([1] * 4, [1] * 4)):
        with pytest.raises(ValueError):
            serving.plan_cross(cfg, new, kv)
    empty = serving.plan_cross(cfg, [], [])
    assert empty.params.batch == 0 and empty.total_tokens == 0

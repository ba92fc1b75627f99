"""The paged cache's operators without a GPU: refusals before any launch, the
workspace, and the reference that the GPU tests use."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2608_19758_amd as fp2
from paper_2608_19758_amd import cache as fc
from tests import cache_ref as ref

FAKE = 0x100000        # never dereferenced: validation fails first


def base(**kw):
    d = dict(batch=2, num_q_heads=32, num_kv_heads=8, max_seq_len=4, max_kv_len=4096, page_size=64,
             dtype="fp8", scale_tokens=64)
    d.update(kw)
    return fp2.make_cache_params(**d)


def pointers(**kw):
    d = dict(k=FAKE, v=FAKE, k_head_scale=FAKE, v_head_scale=FAKE, k_block_scale=FAKE, v_block_scale=FAKE)
    d.update(kw)
    return fc._CachePointers(**d)


def host(x):
    return None if x is None else ctypes.c_void_p(np.asarray(x, np.int32).ctypes.data)


def call(op, p, **over):
    a = dict(k_new=FAKE, v_new=FAKE, q=FAKE, cu=FAKE, cuh=None, cuk=FAKE, cukh=None, cache=pointers(), table=FAKE,
             out=4 * FAKE, lse=FAKE, ws=None, wsb=0, win=None, w=FAKE, stride=p.max_kv_len if p else 0, target=FAKE, pages=64,
             budget=100, recent=10, wout=2 * FAKE, kept=FAKE, cuo=3 * FAKE)
    a.update(over)
    held = [np.asarray(a[n], np.int32) if a[n] is not None else None for n in ("cuh", "cukh")]
    cuh, cukh = (None if x is None else x.ctypes.data for x in held)
    ref_p = ctypes.byref(p) if p else None
    c = ctypes.byref(a["cache"]) if a["cache"] else None
    L = fp2.lib()
    if op == "append":
        return L.fp2_cache_append(ref_p, a["k_new"], a["v_new"], a["cu"], cuh, a["cuk"], cukh, c, a["table"], None)
    if op == "attend":
        return L.fp2_cache_attend(ref_p, a["q"], a["cu"], cuh, a["cuk"], cukh, c, a["table"], a["out"], a["lse"],
                                  a["ws"], a["wsb"], None)
    if op == "weights":
        return L.fp2_cache_weights(ref_p, a["q"], a["lse"], a["cu"], cuh, a["cuk"], cukh, c, a["table"], a["win"],
                                   a["w"], a["stride"], a["ws"], a["wsb"], None)
    return L.fp2_cache_evict(ref_p, c, a["cuk"], cukh, a["table"], a["target"], a["pages"], a["budget"],
                             a["recent"], a["w"], a["wout"], a["stride"], a["kept"], a["cuo"], None)


OPS = ["append", "attend", "weights", "evict"]


@pytest.mark.parametrize("op", OPS)
@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), fp2.EINVAL),
    (dict(batch=65537), fp2.EUNSUPPORTED),
    (dict(batch=65536, max_kv_len=1 << 20), fp2.EUNSUPPORTED),
    (dict(num_kv_heads=0), fp2.EINVAL),
    (dict(num_kv_heads=2048, num_q_heads=2048), fp2.EUNSUPPORTED),
    (dict(num_q_heads=30), fp2.EINVAL),
    (dict(num_q_heads=24), fp2.EUNSUPPORTED),                        # g = 3
    (dict(num_q_heads=128), fp2.EUNSUPPORTED),                       # g = 16
    (dict(head_dim=64), fp2.EUNSUPPORTED),
    (dict(head_dim=0), fp2.EINVAL),
    (dict(page_size=0, max_pages_per_seq=64), fp2.EINVAL),
    (dict(max_pages_per_seq=63), fp2.EINVAL),
    (dict(max_seq_len=4097), fp2.EINVAL),                            # more new tokens than tokens
    (dict(max_seq_len=-1), fp2.EINVAL),
    (dict(max_kv_len=(1 << 20) + 1), fp2.EUNSUPPORTED),
    (dict(max_kv_len=-1, max_seq_len=-1), fp2.EINVAL),
    (dict(dtype=7), fp2.EINVAL),
    (dict(dtype="bf16"), fp2.EINVAL),                                # with scales
    (dict(scale_tokens=-16), fp2.EINVAL),
    (dict(scale_tokens=8), fp2.EUNSUPPORTED),
    (dict(scale_tokens=256, page_size=256), fp2.EUNSUPPORTED),
    (dict(scale_tokens=128), fp2.EINVAL),                            # page of 64
    (dict(sink_tokens=-1), fp2.EINVAL),
    (dict(window_tokens=-1), fp2.EINVAL),
    (dict(kv_splits=33), fp2.EINVAL),
    (dict(kv_splits=-1), fp2.EINVAL),
    (dict(softmax_scale=float("nan")), fp2.EINVAL),
])
def test_params_refused(op, kw, status):
    assert call(op, base(**kw)) == status
    assert fp2.last_error()
    assert fp2.cache_workspace_bytes(base(**kw)) == 0


@pytest.mark.parametrize("op", OPS)
def test_arguments_refused(op):
    p = base()
    assert call(op, None) == fp2.EINVAL
    need = {"append": ["k_new", "v_new", "cu", "cuk", "cache", "table"],
            "attend": ["q", "cu", "cuk", "cache", "table", "out"],
            "weights": ["q", "lse", "cu", "cuk", "cache", "table", "w"],
            "evict": ["cuk", "cache", "table", "target", "w", "wout", "kept", "cuo"]}[op]
    for name in need:
        assert call(op, p, **{name: None}) == fp2.EINVAL, name
    for name in [n for n in ("k_new", "v_new", "q", "out") if n in need]:
        assert call(op, p, **{name: FAKE + 8}) == fp2.EINVAL
        assert "aligned" in fp2.last_error()
    assert call(op, p, cache=pointers(k=FAKE + 4)) == fp2.EINVAL
    assert call(op, p, cache=pointers(k=None)) == fp2.EINVAL
    assert call(op, p, cache=pointers(k_block_scale=None)) == fp2.EINVAL
    assert call(op, base(scale_tokens=0), cache=pointers(k_head_scale=None)) == fp2.EINVAL
    # host copies of the lengths
    assert call(op, p, cukh=[1, 2, 3]) == fp2.EINVAL
    assert call(op, p, cukh=[0, 9, 3]) == fp2.EINVAL
    assert call(op, p, cukh=[0, 4097, 4098]) == fp2.EINVAL
    if op != "evict":
        assert call(op, p, cuh=[0, 5, 6]) == fp2.EINVAL             # over max_seq_len
        assert call(op, p, cuh=[0, 4, 8], cukh=[0, 100, 103]) == fp2.EINVAL
        assert "fewer cached than new" in fp2.last_error()


def test_attend_workspace():
    p = base()
    need = fp2.cache_workspace_bytes(p)
    assert need > 0 and need % 256 == 0
    assert call("attend", p) == fp2.EWORKSPACE
    assert call("attend", p, ws=FAKE, wsb=need - 1) == fp2.EWORKSPACE
    assert call("attend", p, ws=FAKE + 16, wsb=need) == fp2.EWORKSPACE
    assert "workspace" in fp2.last_error()
    p = base(max_seq_len=1000)                                       # rows of the weights are cut too
    need = fp2.cache_workspace_bytes(p)
    assert need > 0 and call("weights", p) == fp2.EWORKSPACE
    assert call("weights", p, ws=FAKE + 16, wsb=need) == fp2.EWORKSPACE


def test_workspace_bounds():
    """Nothing where no keys are cut; else bounded whatever the sizes."""
    assert fp2.cache_workspace_bytes(base(max_kv_len=400, batch=256)) == 0      # many short sequences are taken whole
    assert fp2.cache_workspace_bytes(base(kv_splits=1)) == 0
    assert fp2.cache_workspace_bytes(base(max_seq_len=2000, max_kv_len=8000, batch=64)) == 0
    for kw in (dict(batch=65536), dict(max_seq_len=8), dict(max_seq_len=17, max_kv_len=1 << 20),
               dict(num_q_heads=64, max_seq_len=8, max_kv_len=1 << 20, batch=256), dict(window_tokens=100),
               dict(num_kv_heads=772, num_q_heads=772 * 8, max_seq_len=8)):
        assert fp2.cache_workspace_bytes(base(**kw)) <= 140 << 20, kw


def test_weights_and_eviction_refusals():
    p = base(sink_tokens=4)
    assert call("weights", p, stride=4095) == fp2.EINVAL
    assert call("evict", p, stride=4095) == fp2.EINVAL
    assert call("evict", p, budget=0) == fp2.EINVAL
    assert call("evict", p, recent=-1) == fp2.EINVAL
    assert call("evict", p, budget=13, recent=10) == fp2.EINVAL
    assert call("evict", p, budget=100, pages=1) == fp2.EINVAL
    assert call("evict", p, wout=FAKE) == fp2.EINVAL                # the weights themselves
    row = 4 * 4096                                                  # bytes; 2 x 8 rows
    for w in (FAKE + 15 * row, FAKE - 15 * row, FAKE + 4):
        assert call("evict", p, wout=w) == fp2.EINVAL and "overlap" in fp2.last_error()
        assert call("weights", p, win=w) == fp2.EINVAL and "overlap" in fp2.last_error()
    for cu in (FAKE, FAKE + 8, FAKE - 8):
        assert call("evict", p, cuo=cu) == fp2.EINVAL and "cu_seqlens_k_out" in fp2.last_error()
    assert call("attend", p, out=FAKE) == fp2.EINVAL and "out must not be q" in fp2.last_error()
    assert call("evict", p, budget=(1 << 20) + 1) == fp2.EUNSUPPORTED


@pytest.mark.parametrize("op", OPS)
def test_nothing_to_do(op):
    kw = dict(cu=None, cuk=None, cache=None, table=None)
    assert call(op, base(batch=0), **kw) == fp2.OK
    assert call(op, base(max_kv_len=0, max_seq_len=0), **kw) == fp2.OK
    if op in ("append", "attend"):
        assert call(op, base(max_seq_len=0), **kw) == fp2.OK


def tensors(p, slots=640):
    hkv = p.num_kv_heads
    c = fp2.KVCache(torch.zeros(slots, hkv, 128, dtype=torch.uint8), torch.zeros(slots, hkv, 128, dtype=torch.uint8),
                    torch.zeros(slots // 64, hkv, dtype=torch.uint8), torch.zeros(slots // 64, hkv, dtype=torch.uint8))
    return dict(q=torch.zeros(6, 32, 128, dtype=torch.bfloat16), new=torch.zeros(6, hkv, 128, dtype=torch.bfloat16),
                cache=c, cu=torch.zeros(3, dtype=torch.int32), table=torch.zeros(2, 64, dtype=torch.int32),
                w=torch.zeros(2, hkv, 4096), lse=torch.zeros(6, 32))


def binding(op, p, t):
    if op == "append":
        return fp2.cache_append(p, t["new"], t["new"], t["cache"], t["cu"], t["cu"], t["table"])
    if op == "attend":
        return fp2.cache_attend(p, t["q"], t["cache"], t["cu"], t["cu"], t["table"], out=torch.zeros_like(t["q"]),
                                workspace=torch.zeros(1 << 20, dtype=torch.uint8))
    if op == "weights":
        return fp2.cache_weights(p, t["q"], t["lse"], t["cache"], t["cu"], t["cu"], t["table"], weights=t["w"])
    return fp2.cache_evict(p, t["cache"], t["w"], t["cu"], t["table"], t["table"], budget=100)


@pytest.mark.parametrize("op", OPS)
def test_binding_refuses(op):
    """Wrong types, shapes, strides and devices are refused by the binding: the library sees bare pointers."""
    p = base()
    z = torch.zeros
    with pytest.raises(ValueError, match="must be a CUDA tensor"):        # well formed, but on the host
        binding(op, p, tensors(p))
    bad = [("table", z(2, 65, dtype=torch.int32)), ("table", z(2, 64, dtype=torch.int64)),
           ("table", z(2, 128, dtype=torch.int32)[:, ::2]), ("table", z(1, 64, dtype=torch.int32)),
           ("cu", z(2, dtype=torch.int32)), ("cu", z(3, dtype=torch.int64))]
    if op == "append":
        bad += [("new", z(6, 8, 128)), ("new", z(6, 8, 256, dtype=torch.bfloat16)[:, :, ::2]),
                ("new", z(7, 127, dtype=torch.bfloat16))]
    if op in ("attend", "weights"):
        bad += [("q", z(6, 32, 128)), ("q", z(6, 32, 256, dtype=torch.bfloat16)[..., :128])]
    if op in ("weights", "evict"):
        bad += [("w", z(2, 8, 4095)), ("w", z(2, 8, 4096, dtype=torch.float64)), ("w", z(2, 8, 8192)[..., ::2])]
    if op == "weights":
        bad += [("lse", z(5, 32))]
    for name, x in bad:
        t = tensors(p)
        t[name] = x
        with pytest.raises(ValueError, match=r"^(?!.*CUDA)"):
            binding(op, p, t)
    for part, x in (("k", z(640, 8, 128, dtype=torch.bfloat16)), ("k", z(641, 8, 128, dtype=torch.uint8)),
                    ("k", z(600, 8, 128, dtype=torch.uint8)),             # pages cut off
                    ("k_scale", None), ("k_scale", z(10, 8)), ("k_scale", z(9, 8, dtype=torch.uint8)),
                    ("k_scale", z(20, 8, dtype=torch.uint8)[::2])):
        t = tensors(p)
        setattr(t["cache"], part, x)
        if part == "k" and op != "weights":
            t["cache"].v = x
        with pytest.raises(ValueError, match=r"^(?!.*CUDA)"):
            binding(op, p, t)


def test_rows_of_the_call():
    """With host lengths the binding sees that the tensors hold the new tokens."""
    p, h = base(), np.array([0, 4, 7], np.int32)
    t = tensors(p)
    with pytest.raises(ValueError, match="7 new tokens"):
        fp2.cache_append(p, t["new"], t["new"], t["cache"], t["cu"], t["cu"], t["table"], cu_seqlens_host=h)
    with pytest.raises(ValueError, match="7 new tokens"):
        fp2.cache_attend(p, t["q"], t["cache"], t["cu"], t["cu"], t["table"], cu_seqlens_host=torch.from_numpy(h))
    with pytest.raises(ValueError, match="7 new tokens"):
        fp2.cache_weights(p, t["q"], t["lse"], t["cache"], t["cu"], t["cu"], t["table"], cu_seqlens_host=h)


def test_host_lengths():
    """Strided, short and mistyped host lengths are refused; read-only ones and torch's serve."""
    p = base()
    t = tensors(p)

    def append(h, hk=None):
        with pytest.raises(ValueError) as e:
            fp2.cache_append(p, t["new"], t["new"], t["cache"], t["cu"], t["cu"], t["table"], cu_seqlens_host=h,
                             cu_seqlens_k_host=hk)
        return str(e.value)

    z = np.zeros(6, np.int32)
    for h in (z[::2], z.astype(np.int64), z.astype(np.float32), torch.zeros(6, dtype=torch.int32)[::2],
              torch.zeros(3, dtype=torch.int64)):
        assert "dense host int32" in append(h) and "dense host int32" in append(None, h)
    assert "batch + 1" in append(z[:2]) and "batch + 1" in append(None, torch.zeros(2, dtype=torch.int32))
    z.flags.writeable = False
    for h in (z, torch.zeros(3, dtype=torch.int32)):
        assert "must be a CUDA tensor" in append(h, h)       # all is well but for the device
    assert fc._Args.host("x", z, 2) == z.ctypes.data


def test_alloc_cache():
    p = base()
    c = fp2.alloc_cache(p, 10, device="cpu")
    assert c.k.shape == (640, 8, 128) and c.k.dtype == torch.uint8 and c.k_scale.shape == (10, 8)
    assert fp2.alloc_cache(base(dtype="bf16", scale_tokens=0), 3, device="cpu").k_scale is None
    with pytest.raises(ValueError):
        fp2.alloc_cache(base(scale_tokens=0), 3, device="cpu")
    with pytest.raises(ValueError):
        fp2.alloc_cache(p, 3, device="cpu", k_scale=torch.ones(8), v_scale=torch.ones(8))


# ---- the reference of the GPU tests

def test_reference_codes():
    every = torch.arange(256).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.VALUES, every, equal_nan=True)
    x = np.concatenate([np.random.default_rng(0).standard_normal(20000) * 10.0 ** np.random.default_rng(1).integers(-4, 3, 20000),
                        every[np.isfinite(every)], (every[:126] + every[1:127]) / 2])
    want = torch.from_numpy(x).clamp(-448, 448).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ref.to_codes(x.astype(np.float32)), want)


@pytest.mark.parametrize("x,e", [(0, -100), (448, 0), (448.0001, 1), (449, 1), (224, -1), (1, -8), (1.75, -8), (1.76, -7),
                                 (1e-38, -100), (3e38, 118)])
def test_reference_exponent(x, e):
    assert ref.exponent_for(x) == e


def test_reference_attention():
    """Against torch's attention in 64 bits, without a window, and a window by hand."""
    c = ref.Cache([50], 2, "bf16", 16, seed=1)
    q = torch.randn(50, 4, 128, generator=torch.Generator().manual_seed(0)).bfloat16()
    k, v = (torch.stack([torch.from_numpy(c.values(n, c.slots(0, np.arange(50)), h)) for h in (0, 0, 1, 1)]) for n in "kv")
    want = torch.nn.functional.scaled_dot_product_attention(q.double().transpose(0, 1), k, v, is_causal=True)
    out, _, lse, _, w = ref.attend(c, q, [50])
    assert np.abs(out - want.transpose(0, 1).numpy()).max() < 1e-12
    assert abs(w[0][0].sum() - 200) < 1e-9
    out, *_ = ref.attend(c, q, [50], window=3, sink=2)
    i, h = 30, 3
    keys = [0, 1, 28, 29, 30]
    x = (q[i, h].double() @ k[h][keys].T) / 128 ** 0.5
    assert np.abs(out[i, h] - (torch.softmax(x, 0) @ v[h][keys]).numpy()).max() < 1e-12


def test_reference_keeps_the_heaviest():
    w = np.array([1, 5, 5, 9, 0, 5, np.nan, 2], np.float32)
    assert ref.keep(w, 8, 5, 1, 1).tolist() == [0, 1, 2, 3, 7]
    assert ref.keep(w, 8, 8, 1, 1).tolist() == list(range(8))
    assert ref.keep(w, 8, 7, 0, 0).tolist() == [0, 1, 2, 3, 4, 5, 7]

"""Attention over all keys of another sequence on the GPU against its definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2608_19758_amd as fp2
from tests import cache_ref as ref
from tests import positions_ref as pos_ref
from tests.test_gpu_cache import close, cu_of, dev, on_gpu, params

pytestmark = pytest.mark.gpu

FORMS = ["bf16", "head", 16, 64]


def run_cross(c, hq, new, splits=0, seed=1, scale=0.0, pad=3, max_new=None, odd=()):
    print("cross lens %s new %s hkv %d hq %d %s page %d splits %d" % (c.lens, new, c.hkv, hq, c.form, c.page, splits),
          flush=True)
    g = torch.Generator().manual_seed(seed)
    n = sum(new)
    q = torch.randn((n + pad, hq, 128), generator=g).bfloat16()
    for row, head, d, x in odd:
        q[row, head, d] = x
    p = params(c, hq, new, splits=splits, scale=scale, max_new=max_new)
    cu, cuk = cu_of(new), cu_of(c.lens)
    out = torch.full((n + pad, hq, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n + pad, hq), 7.0, device="cuda")
    ws = fp2.alloc_cross_workspace(p)
    ws.fill_(0xff)                                     # what a workspace holds does not matter
    fp2.cache_cross(p, dev(q), on_gpu(c), dev(cu), dev(cuk), dev(c.table), out=out, lse=lse, workspace=ws,
                    cu_seqlens_host=cu, cu_seqlens_k_host=cuk)
    torch.cuda.synchronize()
    o, tol, z, ztol = pos_ref.cross(c, q[:n], new, scale or None)
    close(out[:n], o, tol, "out")
    close(lse[:n], z, ztol, "lse")
    assert bool((out[n:] == 7).all()) and bool((lse[n:] == 7).all())     # rows behind the last sequence
    return out, lse


@pytest.mark.parametrize("form", FORMS + [32, 128])
def test_single_queries(form):
    c = ref.Cache([1, 2, 31, 32, 33, 0, 129, 700], 2, form, 128, seed=1, spread=1.0)
    run_cross(c, 8, [1] * 8)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("g", [1, 2, 4, 8])
def test_few_queries(form, g):
    """More queries than keys among them; sequences without queries, without keys, without both."""
    c = ref.Cache([900, 1, 50, 64, 3, 0, 0], 3, form, 64, seed=2)
    run_cross(c, 3 * g, [8, 1, 0, 5, 8, 3, 0])


@pytest.mark.parametrize("form", FORMS + [128])
@pytest.mark.parametrize("g", [1, 4, 8])
def test_many_queries(form, g):
    page = 128
    c = ref.Cache([300, 1, 65, 0, 64, 127, 5], 2, form, page, seed=3)
    run_cross(c, 2 * g, [70, 300, 0, 9, 1, 33, 64])


@pytest.mark.parametrize("form,page", [("bf16", 128), ("head", 128), (16, 128), (128, 128), ("bf16", 24), ("head", 5)])
@pytest.mark.parametrize("g", [1, 4, 8])
def test_cut_sequences(form, page, g):
    """Keys so long that sequences are cut, short and empty ones between them."""
    c = ref.Cache([1, 0, 1700, 65, 0, 300, 1601, 5, 0], 2, form, page, seed=12)
    run_cross(c, 2 * g, [70, 3, 300, 0, 9, 1, 33, 64, 0])
    run_cross(c, 2 * g, [1, 3, 8, 0, 7, 1, 5, 8, 0])


@pytest.mark.parametrize("new", [[1] * 150, [3, 0, 1] * 50, [70, 0, 40] * 50])
def test_many_sequences_cut(new):
    """More sequences than a wave has lanes, some longer than those that are left whole."""
    lens = [(37 * b) % 190 for b in range(150)]
    lens[3], lens[64], lens[149] = 1900, 1750, 2000
    c = ref.Cache(lens, 1, 64, 64, seed=13)
    run_cross(c, 2, new)


@pytest.mark.parametrize("form,page", [("bf16", 1), ("bf16", 24), ("head", 5), ("head", 48), ("bf16", 4096),
                                       (16, 48), (32, 96), (64, 192)])
def test_pages(form, page):
    c = ref.Cache([333, 97, 16], 2, form, page, seed=4)
    run_cross(c, 8, [1, 4, 2])
    run_cross(c, 8, [80, 4, 300])


@pytest.mark.parametrize("splits", [1, 2, 5, 32])
@pytest.mark.parametrize("form", ["bf16", 64])
def test_splits(form, splits):
    c = ref.Cache([1500, 30, 0, 640], 1, form, 64, seed=5)
    run_cross(c, 4, [2, 1, 5, 3], splits)
    run_cross(c, 4, [200, 10, 5, 3], splits)


def test_long_and_few_units():
    """One request over long states: the keys are cut."""
    c = ref.Cache([9001], 1, 64, 64, seed=6)
    run_cross(c, 4, [1])
    run_cross(c, 4, [150])


def test_only_empty_sequences():
    for new in ([1, 2], [100, 3]):
        for splits in (0, 1, 3):
            c = ref.Cache([0, 0], 2, "bf16", 16, seed=7)
            n = sum(new)
            p = fp2.make_cache_params(batch=2, num_q_heads=4, num_kv_heads=2, max_seq_len=max(new), max_kv_len=0,
                                      page_size=16, kv_splits=splits)
            q = torch.randn((n, 4, 128)).bfloat16()
            cu = cu_of(new)
            cache = fp2.KVCache(*(torch.empty((0, 2, 128), dtype=torch.bfloat16, device="cuda") for _ in "kv"))
            out, lse = fp2.cache_cross(p, dev(q), cache, dev(cu), dev(cu_of(c.lens)),
                                       torch.empty((2, 0), dtype=torch.int32, device="cuda"), want_lse=True)
            assert not bool(out.any()) and bool((lse == -np.inf).all())


def test_scales_and_heavy_scores():
    c = ref.Cache([200, 77], 2, 16, 16, seed=8, spread=2.0)
    run_cross(c, 4, [3, 1], scale=0.5)
    run_cross(c, 4, [90, 40], scale=0.5)
    run_cross(c, 4, [90, 40], scale=1e-4)


@pytest.mark.parametrize("form", ["bf16", "head"])
def test_odd_values_reach_their_sequence(form):
    """A NaN in a query spoils its row; one in the values the dimension of every row of its sequence."""
    for new in ([2, 3], [100, 70]):
        c = ref.Cache([40, 100], 1, form, 16, seed=9)
        if form == "bf16":
            c.v[c.slots(0, [39])[0], 0, 5] = float("nan")
        else:
            c.v[c.slots(0, [39])[0], 0, 5] = 0x7f
        run_cross(c, 2, new, odd=[(sum(new) - 1, 1, 3, float("nan"))])


def test_bound_larger_than_lengths():
    """Bounds of a captured forward: fewer queries and keys than they allow."""
    c = ref.Cache([100, 7], 2, 64, 64, seed=10)
    run_cross(c, 8, [1, 2], max_new=500)
    run_cross(c, 8, [1, 2], max_new=8)


def test_one_key_of_the_encoder_alone():
    c = ref.Cache([1], 1, "bf16", 1, seed=11)
    out, lse = run_cross(c, 1, [77])
    assert torch.equal(out[:77, 0].cpu(), c.v[c.slots(0, [0])[0], 0].expand(77, 128))

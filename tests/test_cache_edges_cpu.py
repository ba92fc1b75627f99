"""Calls of the paged cache's operators at the edges of what the host can see,
refused before any launch (no GPU)."""
import numpy as np
import pytest
import torch

import paper_2608_19758_amd as fp2
from paper_2608_19758_amd import serving
from tests.test_cache_cpu import FAKE, OPS, base, binding, call, tensors

ROOM = dict(ws=FAKE, wsb=1 << 60)


@pytest.mark.parametrize("op,kw,over", [
    ("append", dict(batch=65536, num_q_heads=512, num_kv_heads=512), {}),
    ("append", dict(batch=512, max_seq_len=131072, max_kv_len=131072), {}),
    ("attend", dict(batch=65536, num_q_heads=64, num_kv_heads=64, kv_splits=32), ROOM),
    ("attend", dict(batch=65536, num_q_heads=256, num_kv_heads=64), ROOM),             # the join alone
    ("attend", dict(batch=1024, num_q_heads=64, max_seq_len=131072, max_kv_len=131072), ROOM),
    ("weights", dict(batch=65536, num_q_heads=128, num_kv_heads=128), ROOM),
    ("weights", dict(batch=1024, max_seq_len=1000, max_kv_len=524288), ROOM),
    ("weights", dict(batch=1, max_seq_len=1000), dict(ROOM, stride=1 << 29)),          # the sum alone
    ("evict", dict(batch=65536, num_q_heads=64, num_kv_heads=64), dict(wout=1 << 50)),
    ("evict", dict(batch=4096, max_kv_len=1 << 20),                                    # the rows alone
     dict(wout=1 << 50, budget=1 << 20, pages=16384)),
])
def test_more_threads_than_a_launch_takes(op, kw, over):
    """A launch takes fewer than 2^32 threads. A call in which any kernel would have more is refused as a
    whole, before the first."""
    assert call(op, base(**kw), **over) == fp2.EUNSUPPORTED
    assert "threads" in fp2.last_error()


@pytest.mark.parametrize("kw", [{}, dict(max_seq_len=100)])
def test_outputs_over_the_queries(kw):
    """Host lengths tell how many rows are read and written: none of them may be shared."""
    p, h = base(**kw), [0, 4, 7]
    q = 16 * FAKE
    row, size = 32 * 128 * 2, 7 * 32 * 128 * 2
    for out in (q + row, q - row, q + size - 16, q - size + 16):
        assert call("attend", p, q=q, out=out, cuh=h, **ROOM) == fp2.EINVAL and "overlap q" in fp2.last_error()
    for lse in (q, q + size - 4, q - 7 * 32 * 4 + 4, 2 * q, 2 * q + size - 4):
        assert call("attend", p, q=q, out=2 * q, lse=lse, cuh=h, **ROOM) == fp2.EINVAL
        assert "lse must not overlap" in fp2.last_error()
    # side by side: refused only later, for want of a workspace
    for out in (q + size, q - size):
        assert call("attend", p, q=q, out=out, lse=4 * q, cuh=h) == fp2.EWORKSPACE


def test_binding_refuses_outputs_over_the_queries():
    """The binding knows the sizes without host lengths."""
    p = base()
    t = tensors(p)
    both = torch.zeros(13, 32, 128, dtype=torch.bfloat16)
    ws = torch.zeros(1, dtype=torch.uint8)

    def attend(q, out, lse=None):
        with pytest.raises(ValueError) as e:
            fp2.cache_attend(p, q, t["cache"], t["cu"], t["cu"], t["table"], out=out, lse=lse, workspace=ws)
        return str(e.value)

    for q, out in ((both[:6], both[:6]), (both[:6], both[5:11]), (both[5:11], both[:6])):
        assert "out must not overlap q" in attend(q, out)
    assert "CUDA" in attend(both[:6], both[6:12])                        # side by side
    flat = both.view(torch.float32).view(-1)                            # 2048 to a row
    for at in (100, 2048 * 6 - 1, 2048 * 6, 2048 * 12 - 1):
        assert "lse must not overlap" in attend(both[:6], both[6:12], flat[at:at + 192].view(6, 32))
    assert "CUDA" in attend(both[:6], both[6:12], flat[2048 * 12:2048 * 12 + 192].view(6, 32))


@pytest.mark.parametrize("op", OPS)
@pytest.mark.parametrize("x", [None, [1.0, 2.0], np.zeros((6, 8, 128), np.float32)])
def test_binding_refuses_what_is_no_tensor(op, x):
    """With the binding's own error, as for every other argument."""
    p = base()
    for name in {"append": ["new", "table"], "attend": ["q", "table"], "weights": ["q", "w", "table"],
                 "evict": ["w", "table"]}[op]:
        if name == "w" and op == "weights" and x is None:
            continue                                                  # the result is allocated then
        t = tensors(p)
        t[name] = x
        if name == "q" and op == "attend":
            with pytest.raises(ValueError, match="q must be"):
                fp2.cache_attend(p, x, t["cache"], t["cu"], t["cu"], t["table"])
            continue
        with pytest.raises(ValueError, match="must be"):
            binding(op, p, t)
    t = tensors(p)
    t["cache"].k = x
    with pytest.raises(ValueError, match="cache.k must be"):
        binding(op, p, t)
    t["cache"] = None
    with pytest.raises(ValueError, match="cache must be"):
        binding(op, p, t)


def test_host_lengths_that_are_no_arrays():
    p, t = base(), tensors(base())
    for h in ([0, 1, 2], (0, 1, 2), 3, "012"):
        for kw in (dict(cu_seqlens_host=h), dict(cu_seqlens_k_host=h)):
            with pytest.raises(ValueError, match="dense host int32"):
                fp2.cache_append(p, t["new"], t["new"], t["cache"], t["cu"], t["cu"], t["table"], **kw)
            if "cu_seqlens_k_host" in kw:
                with pytest.raises(ValueError, match="dense host int32"):
                    fp2.cache_evict(p, t["cache"], t["w"], t["cu"], t["table"], t["table"], budget=100, **kw)


def test_updates_over_the_captured_rows():
    """A forward captured with four rows goes on reading those: more new tokens are refused, though each
    sequence stays within its bound."""
    cfg = serving.CacheConfig(num_q_heads=8, num_kv_heads=2, page_size=16, max_batch=2, max_extend_len=40,
                              max_kv_len=256)
    be = serving.CacheBackend(cfg, device="cpu")
    lengths, table = torch.zeros(6, dtype=torch.int32), torch.zeros((2, 16), dtype=torch.int32)
    meta = serving.CacheMetadata(serving.plan_forward(cfg, [1, 3], [30, 10]), lengths, table, replayed=True)
    meta.rows = 4
    for new in ([3, 2], [3, 3]):
        with pytest.raises(ValueError, match="5 new tokens.*4 rows|6 new tokens.*4 rows"):
            be.update_forward_metadata(meta, new, [30, 10], None)
    with pytest.raises(ValueError, match="block_table"):                  # fits
        be.update_forward_metadata(meta, [3, 1], [30, 10], None)


def test_a_refused_update_changes_nothing():
    cfg = serving.CacheConfig(num_q_heads=8, num_kv_heads=2, page_size=16, max_batch=2, max_extend_len=40,
                              max_kv_len=256)
    be = serving.CacheBackend(cfg, device="cpu")
    lengths, table = torch.full((6,), 7, dtype=torch.int32), torch.full((2, 16), 7, dtype=torch.int32)
    plan = serving.plan_forward(cfg, [1, 3], [30, 10])
    meta = serving.CacheMetadata(plan, lengths, table, replayed=True)
    for bad in (None, table, table[:1]):                                  # (on the host)
        with pytest.raises(ValueError, match="block_table"):
            be.update_forward_metadata(meta, [3, 1], [30, 10], bad)
    assert bool((lengths == 7).all()) and bool((table == 7).all()) and meta.plan is plan


def test_indexes_of_another_budget():
    """The indexes that stay lie `budget` apart: a tensor of another last size would be misread."""
    p, t = base(), tensors(base())
    for shape, says in (((2, 8, 101), "kept must be"), ((2, 8, 200), "kept must be"), ((2, 16, 100), "kept must be"),
                        ((1, 8, 100), "kept holds"), ((2, 8, 100), "CUDA"), ((5, 8, 100), "CUDA"), ((1600,), "CUDA")):
        with pytest.raises(ValueError, match=says):
            fp2.cache_evict(p, t["cache"], t["w"], t["cu"], t["table"], t["table"], budget=100,
                            kept=torch.zeros(shape, dtype=torch.int32))

"""Host side of the cache backend (no GPU): refused configurations, the workspace
bound that every forward fits, and forwards outside the bounds."""
import numpy as np
import pytest

import paper_2608_19758_amd as fp2
from paper_2608_19758_amd import serving


def config(**kw):
    d = dict(num_q_heads=32, num_kv_heads=8, page_size=64, max_batch=4, max_extend_len=8192,
             max_kv_len=65536, dtype="fp8", scale_tokens=64)
    d.update(kw)
    return serving.CacheConfig(**d)


@pytest.mark.parametrize("kw,msg", [
    (dict(num_kv_heads=7), "num_q_heads"), (dict(num_q_heads=24), "group size"),
    (dict(scale_tokens=48), "scale_tokens"), (dict(page_size=24), "multiple"),
    (dict(dtype="bf16"), "bf16"), (dict(max_batch=-1), "batch"), (dict(max_batch=70000), "batch"),
    (dict(max_kv_len=1 << 21), "max_kv_len"), (dict(max_extend_len=65537), "max_extend_len"),
    (dict(max_extend_len=-1), "max_extend_len"), (dict(window_tokens=-1), "window_tokens"),
    (dict(max_batch=65536, max_kv_len=1 << 20), "max_kv_len"),
    (dict(softmax_scale=float("nan")), "softmax_scale"),
])
def test_configurations_refused(kw, msg):
    with pytest.raises(ValueError, match=msg):
        serving.CacheBackend(config(**kw), device="cpu")


def test_workspace_fits_every_forward():
    rng = np.random.default_rng(0)
    for cfg in (config(), config(num_q_heads=64, max_batch=16), config(dtype="bf16", scale_tokens=0),
                config(num_q_heads=8, num_kv_heads=1), config(num_kv_heads=32, window_tokens=4096)):
        be = serving.CacheBackend(cfg, device="cpu")
        assert be.workspace.numel() == fp2.CACHE_WORKSPACE_MAX == 140 << 20
        for _ in range(200):
            b = int(rng.integers(1, cfg.max_batch + 1))
            ext = np.exp(rng.uniform(0, np.log(cfg.max_extend_len), b)).astype(int)
            pre = rng.integers(0, cfg.max_kv_len - ext + 1)
            plan = serving.plan_forward(cfg, ext.tolist(), pre.tolist())
            assert isinstance(plan.params, fp2.CacheParams)
            assert fp2.cache_workspace_bytes(plan.params) <= be.workspace.numel()


@pytest.mark.parametrize("ext,pre,msg", [
    ([9000], [0], "max_extend_len"), ([8192], [65536 - 4096], "max_kv_len"), ([1] * 5, None, "max_batch"),
    ([1, 2], [0], "differ"), ([-1], None, "negative"),
])
def test_forwards_refused(ext, pre, msg):
    be = serving.CacheBackend(config(), device="cpu")
    with pytest.raises(ValueError, match=msg):
        be.init_forward_metadata(ext, pre, None)


def test_table_refused():
    import torch
    be = serving.CacheBackend(config(), device="cpu")
    with pytest.raises(ValueError, match="block_table"):
        be.init_forward_metadata([1], None, torch.zeros((1, 1024), dtype=torch.int32))


def test_caches_and_lengths():
    be = serving.CacheBackend(config(), device="cpu")
    c = be.alloc_cache(3)
    assert tuple(c.k.shape) == (192, 8, 128) and tuple(c.v_scale.shape) == (3, 8)
    assert tuple(be.alloc_weights().shape) == (4, 8, 65536)
    plan = serving.plan_forward(be.cfg, [3, 1, 100], [0, 700, 0])
    meta = serving.CacheMetadata(plan, None, None)
    assert serving.evicted_lens(meta, 64) == [3, 64, 64]

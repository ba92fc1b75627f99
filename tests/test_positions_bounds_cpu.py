"""Bounds of the cache backend's positions, reading back and cross attention without a GPU."""
import numpy as np
import pytest
import torch

import paper_2608_19758_amd as fp2
from paper_2608_19758_amd import serving
from tests.test_cache_cpu import FAKE, base
from tests.test_positions_cpu import FAR, call, cpu_call, cpu_rotary


def config(**kw):
    d = dict(num_q_heads=8, num_kv_heads=2, page_size=16, max_batch=3, max_extend_len=50, max_kv_len=1000)
    d.update(kw)
    return serving.CacheConfig(**d)


# ---- reading back

def test_plan_read():
    """Whole sequences, longer than a forward's chunk, and the last tokens of others."""
    cfg = config()
    plan = serving.plan_read(cfg, [1000, 0, 51])
    p = plan.params
    assert (p.batch, p.max_seq_len, p.max_kv_len) == (3, 1000, 1000)
    assert plan.cu_q.tolist() == plan.cu_k.tolist() == [0, 1000, 1000, 1051] and plan.total_tokens == 1051
    assert plan.cu_q.dtype == plan.cu_k.dtype == np.int32
    plan = serving.plan_read(cfg, [60, 3], [900, 0])
    assert plan.cu_q.tolist() == [0, 60, 63] and plan.cu_k.tolist() == [0, 960, 963]
    assert (plan.params.max_seq_len, plan.params.max_kv_len) == (60, 960)
    assert serving.plan_read(cfg, []).total_tokens == 0
    assert serving.plan_read(cfg, (n for n in (60, 3))).total_tokens == 63
    for lens, pre in (([1001], None), ([1000], [1]), ([-1], None), ([1], [-1]), ([1], [1, 1]), ([1] * 4, None)):
        with pytest.raises(ValueError):
            serving.plan_read(cfg, lens, pre)
    with pytest.raises(ValueError, match="max_kv_len"):
        serving.plan_read(cfg, [1001])
    with pytest.raises(ValueError, match="max_extend_len"):       # a forward's chunk is as long as it was
        serving.plan_forward(cfg, [51])


def test_metadata_of_a_read_is_no_forwards():
    be = serving.CacheBackend(config(), device="cpu")
    with pytest.raises(ValueError, match="block_table"):          # the lengths are right
        be.init_read_metadata([1000, 0, 51], None, None)
    with pytest.raises(ValueError, match="max_kv_len"):
        be.init_read_metadata([1001], None, None)
    meta = serving.CacheMetadata(serving.plan_read(be.cfg, [1000]), None, None, read=True)
    for go in (lambda: be.forward(None, None, None, None, meta), lambda: be.append(None, None, None, meta)):
        with pytest.raises(ValueError, match="metadata of a read"):
            go()
    with pytest.raises(ValueError, match="metadata of a read"):
        be.forward_cross(None, None, meta)


# ---- cross attention

def test_plan_cross_of_more_queries_than_states():
    cfg = config(max_kv_len=100, max_query_len=5000)
    plan = serving.plan_cross(cfg, [5000, 1, 0], [100, 0, 3])
    p = plan.params
    assert (p.batch, p.max_seq_len, p.max_kv_len) == (3, 5000, 100)
    assert plan.cu_q.tolist() == [0, 5000, 5001, 5001] and plan.cu_k.tolist() == [0, 100, 100, 103]
    for cfg, new in ((cfg, 5001), (config(max_query_len=20), 21), (config(), 51)):
        with pytest.raises(ValueError, match="%d queries" % new):
            serving.plan_cross(cfg, [new], [100])
    with pytest.raises(ValueError, match="max_extend_len"):       # what is appended keeps its own bound
        serving.plan_forward(config(max_query_len=5000), [51])


@pytest.mark.parametrize("n", [-1, (1 << 20) + 1])
def test_query_bounds_refused(n):
    with pytest.raises(ValueError, match="max_seq_len"):
        serving.CacheBackend(config(max_query_len=n), device="cpu")


def test_workspace_fits_every_cross_attention():
    rng = np.random.default_rng(1)
    for kw in (dict(), dict(num_q_heads=64, num_kv_heads=8, max_batch=16), dict(num_kv_heads=8), dict(num_kv_heads=1)):
        cfg = config(max_kv_len=70000, max_query_len=1 << 20, **kw)
        be = serving.CacheBackend(cfg, device="cpu")
        for _ in range(200):
            b = int(rng.integers(1, cfg.max_batch + 1))
            new = np.exp(rng.uniform(0, np.log(cfg.max_query_len), b)).astype(int)
            kv = np.exp(rng.uniform(0, np.log(cfg.max_kv_len), b)).astype(int)
            plan = serving.plan_cross(cfg, new.tolist(), kv.tolist())
            assert fp2.cross_workspace_bytes(plan.params) <= be.workspace.numel()


# ---- outputs of a read that meet other tensors of the call

ROWS = FAKE + 64 * FAR


@pytest.mark.parametrize("over", [
    dict(positions=ROWS, k_out=ROWS), dict(positions=ROWS, v_out=ROWS), dict(positions=ROWS + 4 * 2048 - 4, k_out=ROWS),
    dict(positions=ROWS + 4 * 2048 - 4, v_out=ROWS, k_out=None), dict(positions=ROWS + 12, k_out=ROWS + 16)])
def test_read_over_its_positions(over):
    """8 heads: rows of 2048 bytes, four of them."""
    assert call("read", base(), cuh=[0, 2, 4], **over) == fp2.EINVAL
    assert "positions" in fp2.last_error()


def test_read_binding_refuses_outputs_that_meet():
    """Without lengths on the host, as with them."""
    p, cache, lens, host = cpu_call()
    r = cpu_rotary()
    m = torch.zeros((12, 2, 128), dtype=torch.bfloat16)
    at = m.view(-1)[:10].view(torch.int32)
    far = torch.zeros((5, 2, 128), dtype=torch.bfloat16)
    for kw in (dict(k_out=m[:5], v_out=m[4:9]), dict(k_out=m[2:7], v_out=m[:5]), dict(k_out=m[:5], v_out=m[:5]),
               dict(k_out=m[:5], values=False, rotary=r, positions=at), dict(v_out=m[:5], k_out=far, rotary=r, positions=at)):
        with pytest.raises(ValueError, match="overlap"):
            fp2.cache_read(p, cache, *lens, **kw)
    # outputs side by side are right: what is refused is the device
    with pytest.raises(ValueError, match="CUDA tensor"):
        fp2.cache_read(p, cache, *lens, k_out=m[:5], v_out=m[5:10])
    with pytest.raises(ValueError, match="CUDA tensor"):
        fp2.cache_read(p, cache, *lens, k_out=m[1:6], v_out=m[6:11], rotary=r, positions=at[:5])


def test_append_binding_refuses_queries_over_positions():
    """Without lengths on the host, as with them."""
    p, cache, lens, host = cpu_call()
    r, m = cpu_rotary(), torch.zeros((6, 8, 128), dtype=torch.bfloat16)
    q, k, v = m[:5, :4], m[:5, 4:6], m[:5, 6:]
    out = torch.zeros((12, 4, 128), dtype=torch.bfloat16)
    ints = out.view(-1).view(torch.int32)
    codes = dict(out=out.view(torch.uint8).view(-1, 4, 128)[:5], q_scale=torch.ones(4))
    # rows of 256 integers' bytes, and of 128 where they are codes
    for kw, at in ((dict(out=out[:5]), 0), (dict(out=out[:5]), 700), (dict(out=out[:5]), 5 * 256 - 1), (codes, 0), (codes, 5 * 128 - 1)):
        with pytest.raises(ValueError, match="positions"):
            fp2.cache_append_rotary(p, r, q, k, v, cache, *lens, positions=ints[at:at + 5], **kw)
    with pytest.raises(ValueError, match="CUDA tensor"):          # beside them: right
        fp2.cache_append_rotary(p, r, q, k, v, cache, *lens, positions=ints[5 * 256:][:5], out=out[:5])


def test_no_cross_kernels_that_no_call_reaches():
    """Scales of blocks of 16 tokens and more imply pages of a multiple of 8."""
    from paper_2608_19758_amd import build
    with open(build.LIB, "rb") as f:
        names = f.read()
    for kernel in (b"cross_kernel", b"split_kernel"):
        for form, grouped in ((0, 0), (0, 1), (1, 0), (1, 1), (2, 1)):
            assert kernel + b"ILi%dELb%dE" % (form, grouped) in names
        assert kernel + b"ILi2ELb0E" not in names

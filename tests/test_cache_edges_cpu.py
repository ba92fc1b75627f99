"""Calls of the paged cache's operators at the edges of what the host can see,
refused before any launch (no GPU)."""
import pytest

import paper_2608_19758_amd as fp2
from tests.test_cache_cpu import FAKE, base, call

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

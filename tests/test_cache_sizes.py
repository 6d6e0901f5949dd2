"""Sizes that the cache operators refuse, by every way that a caller asks for them, without a GPU."""
import ctypes as C

import pytest

from paper_1811_03115_amd import binding
from test_cache_ops import F32, attend, blocks, cache


@pytest.mark.parametrize("kw,args,block", [
    (dict(capacity=1 << 16), (5, 3, 4), 0), (dict(max_batch=1, capacity=1 << 16), (2, 1, 2), 64), (dict(capacity=1 << 16), (2, 3, 130), 0), (dict(n_kv_heads=1, capacity=1 << 17), (1, 1, 65), 32), (dict(capacity=32 * 4097), (2, 3, 4), 32),
    (dict(capacity=128 * 4097), (1, 1, 2), 128), (dict(dtype=F32, head_dim=16, capacity=64 * 4097 + 5), (1, 1, 2), 64)], ids=str)
def test_workspace_of_refused_sizes(kw, args, block):
    L = binding.lib()
    c = cache(**kw)
    b, t, heads = args
    assert attend(c=c, b=b, t=t, heads=heads, blocks=blocks(block=block) if block else None) in (-1, -3)
    assert L.bpd_attention_workspace_bytes(C.byref(c), b, t, heads, block) == 0


@pytest.mark.parametrize("block", [32, 64, 128])
def test_summaries_of_refused_sizes(block):
    L = binding.lib()
    assert L.bpd_summaries_bytes(C.byref(cache(capacity=block * 4096)), block) == 4 * 2 * 64 * 2 * 64 * 64 * 2
    assert L.bpd_summaries_bytes(C.byref(cache(capacity=block * 4097)), block) == 0
    assert L.bpd_attention_workspace_bytes(C.byref(cache(capacity=block * 4096)), 4, 64, 128, block) > 0

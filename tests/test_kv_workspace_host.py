"""What the operators that bound a cache take as their workspace."""
import ctypes

import pytest
import torch

from paper_2504_11320_amd import binding as B
from paper_2504_11320_amd import kv
from test_kv_more_host import batch, cache, eviction

MOST = 256 << 20


def evict_bytes(n_seq, kv_heads, bound, page=16, **kw):
    n = ctypes.c_size_t()
    cols = 1 << 16
    rc = kv._lib().wait_kv_evict_workspace_bytes(
        cache(kv_heads=kv_heads), eviction(n_seq=n_seq, table_cols=cols, table_stride=cols, max_kv_len=bound, **kw),
        ctypes.byref(n))
    assert rc == B.WS_OK
    return n.value


def test_eviction_has_a_limit():
    """The counts of 4096 keys of a request and head, and their numbers, while
    both fit 256 MB; never more than that."""
    each, counts = 4 * 256 * 4 + 16 + 4096 * 4, 4 * 256 * 4 + 16
    assert evict_bytes(1, 8, 131072) == 8 * 32 * each
    assert evict_bytes(128, 8, 8192) == 128 * 8 * 2 * each
    assert evict_bytes(128, 32, 8192) == 128 * 32 * 2 * each
    assert evict_bytes(128, 32, 16384) == 128 * 32 * 4 * counts
    assert evict_bytes(128, 32, 131072) == 128 * 32 * 15 * counts     # of 32 parts
    assert evict_bytes(1024, 32, 131072) == 1024 * 32 * counts
    assert evict_bytes(2048, 32, 131072) == 0
    for n_seq in (1, 7, 100, 1000, 2040, 30000):
        for heads in (1, 8, 32):
            for bound in (2048, 2049, 5000, 131072, 1 << 20):
                n = evict_bytes(n_seq, heads, bound)
                assert n <= MOST and (n == 0) == (bound == 2048 or n_seq * heads * counts > MOST)
    assert evict_bytes(1000, 32, 1 << 20, keep=20, recent=20) == 0
    c = kv.Cache.empty(64, 16, 32, 64, device="cpu")
    pages, lens = torch.zeros(128, 8192, dtype=torch.int32), torch.zeros(128, dtype=torch.int32)
    assert kv.evict_workspace_bytes(c, pages, lens, keep=5) == 128 * 32 * 15 * counts

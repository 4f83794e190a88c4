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


def weigh_bytes(heads=4, kv_heads=1, dim=64, bound=1000, **kw):
    n = ctypes.c_size_t()
    b = dict(heads=heads, table_cols=1 << 16, table_stride=1 << 16, max_kv_len=bound)
    rc = kv._lib().wait_kv_weigh_workspace_bytes(cache(kv_heads=kv_heads, dim=dim), batch(**{**b, **kw}),
                                                 ctypes.byref(n))
    assert rc == B.WS_OK
    return n.value


def test_weighing_has_a_limit():
    """Room for the parts of the rows of all requests, over as many keys as the
    bound allows: none for single tokens, at most 64 MB."""
    for heads, kv_heads in ((4, 1), (16, 1), (32, 8)):
        assert weigh_bytes(heads, kv_heads, n_seq=128, n_tokens=128, max_q_len=1) == 0
    # 512 tokens of one request, 4 rows each: parts of two blocks of 64 rows, and one for
    # the request, over tiles of 256 keys
    one = dict(n_seq=1, n_tokens=512, max_q_len=512)
    assert weigh_bytes(bound=1000, **one) == (2048 // 128 + 1) * 1024 * 4
    assert weigh_bytes(bound=1025, **one) == (2048 // 128 + 1) * 1280 * 4
    assert weigh_bytes(bound=1000, dim=256, **one) == (2048 // 64 + 1) * 1024 * 4
    assert weigh_bytes(bound=1000, **{**one, "n_seq": 7}) == (2048 // 128 + 7) * 1024 * 4
    assert weigh_bytes(bound=1000, **{**one, "max_q_len": 20}) == 0   # 80 rows: less than a part
    for n_seq in (1, 50, 3000):
        for n_tokens in (64, 8192, 200000):
            for bound in (1, 3000, 131072):
                for heads, kv_heads in ((16, 1), (64, 8), (32, 32)):
                    n = weigh_bytes(heads, kv_heads, bound=bound, n_seq=n_seq, n_tokens=n_tokens,
                                    max_q_len=min(n_tokens, 8192))
                    assert n <= 64 << 20 and n % 4 == 0


def test_a_workspace_that_is_too_small():
    """The sizes are what the calls take."""
    at = 1 << 44
    b = dict(table=at, starts=at + 4096, kv_lens=at + 8192, n_seq=1, n_tokens=512, max_q_len=512, table_cols=64,
             table_stride=64, max_kv_len=1000)
    c = cache(k=at << 1, v=at << 2, kv_heads=1)
    n = weigh_bytes(**{k: v for k, v in b.items() if k != "max_kv_len"})
    assert n > 0

    def weigh(ws, size):
        return kv._lib().wait_kv_weigh(c, batch(heads=4, **b), kv.ROWS.pack(at * 3, 256, 64, kv.BF16), at * 5,
                                       at * 6, 1, ws, size, None)

    assert weigh(at * 7, n - 4) == B.WS_EWORKSPACE and weigh(None, n) == B.WS_EWORKSPACE
    assert weigh(at * 7 + 2, n) == B.WS_EINVAL


def test_more_requests_and_heads_than_a_launch_has():
    """Refused before sizes are multiplied that 64 bits do not hold."""
    n = ctypes.c_size_t(7)
    for n_seq, heads in ((1 << 24, 1), (1 << 19, 32), ((1 << 31) - 1, 1 << 30)):
        rc = kv._lib().wait_kv_evict_workspace_bytes(cache(kv_heads=heads, pages=1, page_size=1),
                                                     eviction(n_seq=n_seq, table_cols=1 << 17, max_kv_len=1 << 17),
                                                     ctypes.byref(n))
        assert rc == B.WS_EUNSUPPORTED and n.value == 7
    assert evict_bytes((1 << 24) - 1, 1, 1 << 17) == 0

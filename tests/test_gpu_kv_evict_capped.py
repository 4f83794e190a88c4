"""Eviction where the counts of all keys would take more workspace than there is
for them: without the numbers kept, in fewer and longer parts, by a workgroup for
each request and head."""
import pytest
import torch

from paper_2504_11320_amd import kv
from test_gpu_kv_evict import check

pytestmark = pytest.mark.gpu


def lengths(n, long):
    g = torch.Generator().manual_seed(n)
    lens = torch.randint(0, 50, (n,), generator=g).tolist()
    for i, m in long:
        lens[i] = m
    return lens


@pytest.mark.parametrize("to", [False, True])
@pytest.mark.parametrize("n,long,bound", [(52, [(3, 20000), (51, 2049)], 16384),   # numbers not kept
                                          (52, [(0, 20000), (50, 4097)], 131072)],  # and fewer parts
                         ids=["numbers", "parts"])
def test_capped(n, long, bound, to):
    check(lengths(n, long), 16, 64, 64, torch.int8, keep=33, recent=9, to=to, max_kv_len=bound, kind="few")


def test_capped_at_none():
    check(lengths(1021, [(7, 5000), (1020, 2100)]), 16, 64, 64, torch.int8, keep=33, recent=9, to=False,
          max_kv_len=8192, kind="few")


def test_the_same_keys_whatever_the_bound():
    """Kept keys and rows do not depend on how they are counted."""
    for bound in (2048, 2049, 70000):
        check([3000, 9000, 40], 16, 2, 64, torch.bfloat16, keep=700, recent=50, to=False, max_kv_len=bound,
              kind="near")


def test_what_a_table_wider_than_the_requests_takes():
    """128 requests of 32 heads under a table for 131,072 keys, no bound given."""
    c = kv.Cache.empty(64, 16, 32, 64)
    pages = torch.zeros(128, 8192, dtype=torch.int32).cuda()
    lens = torch.full((128,), 3, dtype=torch.int32).cuda()
    assert kv.evict_workspace_bytes(c, pages, lens, keep=5) <= 256 << 20

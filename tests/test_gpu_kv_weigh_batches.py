"""Accumulated weights of batches as a server has them: many requests and KV heads,
whose waves are dealt out over the dies, and prompts anywhere among more than 64
requests, whose rows are split."""
import pytest
import torch

from paper_2504_11320_amd import kv
from test_gpu_kv_weigh import batch, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache_dtype", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("dim,heads,kv_heads", [(128, 5, 5), (64, 15, 5), (256, 3, 3)])
@pytest.mark.parametrize("prompt", [0, 40])
def test_many_requests_and_heads(cache_dtype, dim, heads, kv_heads, prompt):
    """Numbers of requests times KV heads that are no multiple of 32."""
    g = torch.Generator().manual_seed(3)
    kl = torch.randint(1, 70, (37,), generator=g).tolist()
    ql = [1] * 37
    if prompt:
        ql[20], kl[20] = prompt, prompt + 13
    run(ql, kl, 16, heads, kv_heads, dim, cache_dtype, max_q_len=max(ql), max_kv_len=max(kl))


@pytest.mark.parametrize("n", [1, 31, 32, 33, 64, 95])
def test_pairs_about_a_multiple_of_32(n):
    run([1] * n, [5 + 3 * i % 40 for i in range(n)], 8, 1, 1, 64, torch.float16, max_q_len=1)


@pytest.mark.parametrize("accumulate", [True, False])
@pytest.mark.parametrize("window", [0, 50])
def test_parts_of_more_than_64_requests(accumulate, window):
    """Prompts before, at and behind the 64th and the 128th request, requests
    without tokens between, single tokens everywhere else."""
    ql, kl = [1] * 140, [9 + 7 * i % 60 for i in range(140)]
    for i in (5, 61, 65, 100, 126, 129):
        ql[i] = 0
    for i, (n, m) in {3: (150, 150), 62: (20, 90), 63: (300, 310), 64: (90, 200), 66: (17, 17),
                      127: (64, 64), 128: (130, 150), 139: (200, 200)}.items():
        ql[i], kl[i] = n, m
    q, pages, starts, lens, n = batch(ql, kl, 16, 4, 64, torch.bfloat16, 1)
    c = kv.Cache.empty(n, 16, 1, 64)
    assert kv.weigh_workspace_bytes(q.cuda(), c, pages.cuda(), starts.cuda(), lens.cuda(), max_q_len=300,
                                    max_kv_len=310, window=window) > 0
    run(ql, kl, 16, 4, 1, 64, torch.bfloat16, accumulate=accumulate, window=window, max_q_len=300, max_kv_len=310)

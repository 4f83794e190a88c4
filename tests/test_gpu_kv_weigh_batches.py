"""Accumulated weights of batches as a server has them: many requests and KV heads,
whose waves are dealt out over the dies."""
import pytest
import torch

from test_gpu_kv_weigh import run

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

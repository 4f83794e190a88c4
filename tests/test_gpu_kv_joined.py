"""Attention over 8-bit caches where requests are split over their keys, held to
bounds that tell a wrong joining of the parts."""
import pytest
import torch

from kv_bounds import attend_codes, says_something
from kv_util import within
from test_gpu_kv_attention import make

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float16
E4, I8 = torch.float8_e4m3fn, torch.int8


@pytest.fixture(scope="module")
def kv():
    from paper_2504_11320_amd import kv
    return kv


def held(kv, s, what, hints=({},), **kw):
    o, tol = attend_codes(s["q"], s["cache"], s["pages"], s["starts"], s["kv_lens"], **kw)
    assert says_something(o, tol)
    for h in hints:
        got = kv.attention(s["q"], s["cache"], s["pages"], s["starts"], s["kv_lens"], **kw, **h)
        within(got, o, tol, f"{what} {h}")


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("ctype", [E4, I8])
def test_single_token_in_many_parts(kv, ctype, dim):
    s = make(kv, [1, 1], [70000, 3000], 2, 1, dim, 64, ctype, FP)
    held(kv, s, f"70000 keys {ctype} {dim}", (dict(max_q_len=1), {}, dict(max_kv_len=5000)))


@pytest.mark.parametrize("group", [1, 8])
@pytest.mark.parametrize("ctype,qtype", [(E4, FP), (I8, FP), (I8, BF)])
def test_one_request_in_parts(kv, ctype, qtype, group):
    hints = [dict(max_q_len=1, max_kv_len=n) for n in (5003, 100, None)]
    s = make(kv, [1], [5003], 2 * group, 2, 128, 16, ctype, qtype)
    held(kv, s, "5003 keys", hints)
    held(kv, s, "5003 keys, window", hints, window=3000)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("ctype", [E4, I8])
def test_prompts_in_parts(kv, ctype, dim):
    """Many rows in parts beside few rows in parts; the same laid out for single
    tokens."""
    s = make(kv, [40, 1, 3], [2600, 4100, 1900], 10, 2, dim, 16, ctype, FP)
    held(kv, s, f"prompts {ctype} {dim}", ({}, dict(max_q_len=1), dict(max_kv_len=700)))
    held(kv, s, f"prompts {ctype} {dim}, not causal", causal=False)


@pytest.mark.parametrize("group", [1, 4])
@pytest.mark.parametrize("ctype", [E4, I8])
def test_requests_longer_than_laid_out(kv, ctype, group):
    """Rows that have room for parts beside rows that have none, in a workspace
    of exactly the bytes asked for."""
    s = make(kv, [1, 2, 4, 1, 3], [3000, 2900, 4100, 1800, 2600], 2 * group, 2, 128, 16, ctype, FP)
    args = s["q"], s["cache"], s["pages"], s["starts"], s["kv_lens"]
    o, tol = attend_codes(*args)
    assert says_something(o, tol)
    for n in (1, 2, 3, 4, 9, None):
        size = kv.attention_workspace_bytes(*args, max_q_len=n)
        space = torch.full((size + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        got = kv.attention(*args, max_q_len=n, workspace=space[:size])
        within(got, o, tol, f"laid out for {n}")
        assert size > 0 and bool((space[size:] == 0xA5).all())

"""KV-path operators at sizes where the work is laid out differently: rows for
more threads than the card holds at once, requests in many parts."""
import pytest
import torch

from kv_util import TOP, codes
from test_gpu_kv_attention import check, make

pytestmark = pytest.mark.gpu

BF, FP, F32 = torch.bfloat16, torch.float16, torch.float32
E4, I8 = torch.float8_e4m3fn, torch.int8


@pytest.fixture(scope="module")
def kv():
    from paper_2504_11320_amd import kv
    return kv


@pytest.mark.parametrize("T,heads,dim,part", [(4100, 9, 128, None), (4100, 9, 128, 128),
                                              (4103, 9, 128, 48), (7300, 9, 64, 64),
                                              (1900, 9, 256, 128), (33000, 1, 128, 128)])
@pytest.mark.parametrize("dtype,ctype", [(BF, E4), (FP, I8), (F32, BF)])
def test_append_of_many_rows(kv, T, heads, dim, part, dtype, ctype):
    """As by calls of few rows each, bit for bit, the last head of an odd number
    among them; some tokens have no slot or no position."""
    assert T * heads * dim // 8 > 256 * 2048
    g = torch.Generator().manual_seed(T + dim)
    page = 16
    pages = -(-T // page)
    slots = torch.randperm(pages * page, generator=g)[:T]
    slots[::97] = -1
    k, v = (torch.randn(T, heads, dim, generator=g).to(dtype) for _ in range(2))
    how = {}
    if part:
        pos = torch.randint(0, 500, (T,), generator=g)
        pos[5::501] = 500  # behind the table
        how = dict(positions=pos.cuda(), table=kv.rotary_table(500, part, device="cuda"))
    one, other = (kv.Cache.empty(pages, page, heads, dim, ctype) for _ in range(2))
    at, ck, cv = slots.cuda(), k.cuda(), v.cuda()
    kv.append(one, ck, cv, at, **how)
    for i in range(0, T, 1000):
        j = slice(i, i + 1000)
        kv.append(other, ck[j], cv[j], at[j],
                  **({**how, "positions": how["positions"][j]} if how else {}))
    for name in ("k", "v", "k_scale", "v_scale"):
        x, y = getattr(one, name), getattr(other, name)
        if x is not None:
            assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))
    here = slots >= 0
    if part:
        here &= pos < 500
        k = kv.rotary(ck.float(), **how).cpu()
    s = slots[here]
    for name, x in (("k", k.float()[here]), ("v", v.float()[here])):
        held = getattr(one, name).cpu().view(torch.uint8)[s // page, :, s % page].view(ctype).float()
        assert torch.equal(held, codes(x, ctype)[0] if ctype in TOP else x.to(ctype).float())


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("ctype", [BF, I8])
def test_single_token_in_many_parts(kv, ctype, dim):
    s = make(kv, [1, 1], [70000, 3000], 2, 1, dim, 64, ctype, BF)
    check(kv, s, f"70000 keys {ctype} {dim}", max_q_len=1)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("ctype", [BF, E4])
def test_prompt_in_many_parts(kv, ctype, dim):
    """Rows with more parts than are joined at once, heads that do not fill a
    wave, beside a request in one part."""
    s = make(kv, [40, 20], [2600, 20], 5, 1, dim, 16, ctype, BF)
    check(kv, s, f"a prompt over 2600 keys {ctype} {dim}")

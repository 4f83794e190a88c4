"""The C++ side of the KV-path operators' Python calls without a GPU: structs,
errors and their types."""
import ctypes as C

import pytest
import torch

from paper_2504_11320_amd import binding as B
from paper_2504_11320_amd import build as Bd
from paper_2504_11320_amd import kv


def small(dtype=torch.bfloat16, heads=2, pages=4):
    return kv.Cache.empty(pages, 16, heads, 64, dtype, device="cpu")


def batch(heads=4, cols=2, tokens=3):
    q = torch.zeros(tokens, heads, 64, dtype=torch.bfloat16)
    return (q, torch.zeros(1, cols, dtype=torch.int32), torch.tensor([0, tokens], dtype=torch.int32),
            torch.tensor([9], dtype=torch.int32))


@pytest.mark.parametrize("dtype,code", [(torch.bfloat16, kv.BF16), (torch.float16, kv.FP16),
                                        (torch.float8_e4m3fn, kv.FP8), (torch.int8, kv.INT8)])
def test_cache_struct(dtype, code):
    """The bytes are those of the packed struct."""
    c = small(dtype)
    scales = [0 if t is None else t.data_ptr() for t in (c.k_scale, c.v_scale)]
    fields = [c.k.data_ptr(), c.v.data_ptr(), *scales, 4, 16, 2, 64, code]
    assert c._c == kv.CACHE.pack(*fields)
    assert (c.pages, c.page_size, c.kv_heads, c.dim) == (4, 16, 2, 64)


def test_missing_module_is_an_error(monkeypatch):
    assert kv.BINDING == Bd.BINDING
    monkeypatch.setattr(kv, "_kv", None)
    monkeypatch.setattr(kv, "BINDING", kv.BINDING + ".none")
    with pytest.raises(RuntimeError, match="missing"):
        small()


def test_types_of_errors():
    c = small()
    q, pages, starts, lens = batch()
    for call in (lambda: kv.rotary([1.0], pages, q), lambda: kv.append(c, None, q, starts),
                 lambda: kv.read(c, 3), lambda: kv.Cache(1, q),
                 lambda: kv.attention(None, c, pages, starts, lens),
                 lambda: kv.attention(q, c, pages, starts, [9]),
                 lambda: kv.attention(q, c, pages, starts, lens, max_q_len="3"),
                 lambda: kv.attention(q, c, pages, starts, lens, scale="one")):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        kv.read(c, torch.zeros(3, dtype=torch.int64), dtype=3)
    native = kv._native()
    for bad in (b"", c._c[:-1], None, 3):
        with pytest.raises(ValueError):
            native.read(bad, 0, torch.zeros(3, dtype=torch.int64), torch.bfloat16, None, None)
    with pytest.raises(TypeError):
        native.read(c._c)


def test_empty_dimensions():
    """A cache without heads or pages is refused, not divided by."""
    q, pages, starts, lens = batch()
    for c in (small(heads=0), small(pages=0)):
        with pytest.raises((ValueError, B.WaitSimError)):
            kv.attention_workspace_bytes(q, c, pages, starts, lens)
    with pytest.raises(ValueError):
        kv.attention_workspace_bytes(q[:, :0], small(), pages, starts, lens)


def test_workspace_is_the_librarys():
    """The same bytes as the C ABI's for the same batch, bounds clamped to the
    shapes; the library's refusals come as its error."""
    c = small(pages=4096)
    q, pages, starts, lens = batch(cols=4096)
    for max_q, max_kv, window in ((None, None, 0), (3, 65536, 0), (1, 4096, 0), (1 << 40, 1 << 40, 7),
                                  (3, 65536, 1 << 40)):
        b = kv.BATCH.pack(pages.data_ptr(), 4096, 4096, starts.data_ptr(), lens.data_ptr(), 1, 3, 4,
                          0.125, 1, min(window, 2**31 - 1), min(3 if max_q is None else max_q, 3),
                          min(65536 if max_kv is None else max_kv, 65536))
        n = C.c_size_t()
        assert kv._lib().wait_kv_attention_workspace_bytes(c._c, b, n) == B.WS_OK
        assert n.value == kv.attention_workspace_bytes(q, c, pages, starts, lens, max_q_len=max_q,
                                                       max_kv_len=max_kv, window=window)
    assert n.value > 0
    for bad in (dict(window=-1), dict(window=-(1 << 40)), dict(max_q_len=-1), dict(max_kv_len=-5)):
        with pytest.raises(B.WaitSimError) as e:
            kv.attention_workspace_bytes(q, c, pages, starts, lens, **bad)
        assert e.value.code == B.WS_EINVAL
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises((ValueError, B.WaitSimError)):
            kv.attention(q, c, pages, starts, lens, scale=scale)

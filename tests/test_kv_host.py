"""The KV-path operators without a GPU: exports, argument checks of the C ABI
and of the Python side, angles of the rotation, workspace sizes."""
import ctypes as C
import math
import os
import re

import pytest
import torch

from paper_2504_11320_amd import binding as B
from paper_2504_11320_amd import kv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 40   # never dereferenced: the checks come first


def test_library_exports_header_symbols():
    src = open(os.path.join(ROOT, "include", "wait_kv.h")).read()
    names = sorted(set(re.findall(r"^int (wait_kv_\w+)\s*\(", src, re.M)))
    assert names == ["wait_kv_append", "wait_kv_attention", "wait_kv_attention_workspace_bytes",
                     "wait_kv_read", "wait_kv_rotary"]
    for n in names:
        assert hasattr(B.lib(), n), n


def cache(**kw):
    d = dict(k=FAKE, v=FAKE, k_scale=None, v_scale=None, pages=4, page_size=16, kv_heads=2, dim=64,
             type=kv.BF16)
    d.update(kw)
    return kv.CACHE.pack(*[d[n] or 0 for n in ("k", "v", "k_scale", "v_scale", "pages", "page_size",
                                               "kv_heads", "dim", "type")])


def rows(data=FAKE, token=128, head=64, type=kv.BF16):
    return kv.ROWS.pack(data or 0, token, head, type)


def turn(**kw):
    d = dict(table=FAKE, positions=FAKE, positions_32=0, n_table=10, part=32, interleaved=0)
    d.update(kw)
    return kv.TURN.pack(*[d[n] or 0 for n in ("table", "positions", "positions_32", "n_table",
                                              "part", "interleaved")])


def batch(**kw):
    d = dict(table=FAKE, table_stride=8, table_cols=8, starts=FAKE, kv_lens=FAKE, n_seq=2,
             n_tokens=4, heads=4, scale=1.0, causal=1, window=0, max_q_len=2, max_kv_len=100)
    d.update(kw)
    return kv.BATCH.pack(*[d[n] or 0 for n in ("table", "table_stride", "table_cols", "starts",
                                               "kv_lens", "n_seq", "n_tokens", "heads", "scale",
                                               "causal", "window", "max_q_len", "max_kv_len")])


def test_rotary_refusals():
    L = kv._lib()

    def call(x=None, out=None, n=3, heads=2, dim=64, t=None):
        return L.wait_kv_rotary(x or rows(), out or rows(), n, heads, dim, t or turn(), 0, None)

    assert call(n=-1) == call(heads=0) == call(dim=1) == B.WS_EINVAL
    assert call(n=1 << 31) == B.WS_EUNSUPPORTED
    assert call(x=rows(data=None)) == call(out=rows(data=None)) == B.WS_EINVAL
    assert call(x=rows(type=kv.FP8)) == call(x=rows(type=9)) == B.WS_EINVAL
    assert call(x=rows(type=kv.FP16)) == B.WS_EINVAL                    # two types
    assert call(x=rows(data=FAKE + 1)) == B.WS_EINVAL                   # not aligned
    assert call(out=rows(token=256)) == B.WS_EINVAL                     # in place, other strides
    for t in (turn(part=0), turn(part=31), turn(part=66), turn(table=None), turn(positions=None),
              turn(n_table=-1), turn(table=FAKE + 2), turn(positions=FAKE + 4)):
        assert call(t=t) == B.WS_EINVAL
    assert L.wait_kv_rotary(None, rows(), 3, 2, 64, turn(), 0, None) == B.WS_EINVAL
    assert L.wait_kv_rotary(rows(), rows(), 3, 2, 64, None, 0, None) == B.WS_EINVAL
    assert b"positions" in L.wait_sim_last_error()
    assert call(n=0, x=rows(data=None), out=rows(data=None)) == B.WS_OK
    assert L.wait_sim_last_error() == b""


BAD_CACHES = [(dict(k=None), B.WS_EINVAL), (dict(dim=96), B.WS_EUNSUPPORTED),
              (dict(page_size=24), B.WS_EINVAL), (dict(page_size=0), B.WS_EINVAL),
              (dict(page_size=2048), B.WS_EINVAL), (dict(pages=0), B.WS_EINVAL),
              (dict(kv_heads=0), B.WS_EINVAL), (dict(type=kv.FP32), B.WS_EINVAL),
              (dict(type=7), B.WS_EINVAL), (dict(k=FAKE + 8), B.WS_EINVAL),
              (dict(pages=1 << 28), B.WS_EUNSUPPORTED), (dict(k_scale=FAKE), B.WS_EINVAL),
              (dict(type=kv.FP8), B.WS_EINVAL), (dict(type=kv.INT8, k_scale=FAKE), B.WS_EINVAL),
              (dict(type=kv.FP8, k_scale=FAKE, v_scale=FAKE + 2), B.WS_EINVAL)]


@pytest.mark.parametrize("bad,code", BAD_CACHES)
def test_cache_refusals(bad, code):
    L = kv._lib()
    c = cache(**bad)
    assert L.wait_kv_append(c, rows(), rows(), FAKE, 3, None, None) == code
    assert L.wait_kv_read(c, FAKE, 3, rows(), rows(), None) == code
    size = C.c_size_t()
    assert L.wait_kv_attention_workspace_bytes(c, batch(), size) == code
    assert L.wait_kv_attention(c, batch(), rows(), rows(), None, None, 0, None) == code


def test_append_and_read_refusals():
    L = kv._lib()
    for call in (lambda k, v, s, n: L.wait_kv_append(cache(), k, v, s, n, None, None),
                 lambda k, v, s, n: L.wait_kv_read(cache(), s, n, k, v, None)):
        assert call(rows(), rows(), FAKE, -1) == B.WS_EINVAL
        assert call(rows(), rows(), FAKE, 1 << 30) == B.WS_EUNSUPPORTED
        assert call(rows(data=None), rows(), FAKE, 3) == B.WS_EINVAL
        assert call(rows(), rows(type=kv.FP32), FAKE, 3) == B.WS_EINVAL
        assert call(rows(), rows(), None, 3) == B.WS_EINVAL
        assert call(rows(), rows(), FAKE + 4, 3) == B.WS_EINVAL
        assert call(rows(data=None), rows(data=None), None, 0) == B.WS_OK
    assert L.wait_kv_append(cache(), rows(), rows(), FAKE, 3, turn(part=66), None) == B.WS_EINVAL


def test_attention_refusals():
    L = kv._lib()

    def call(c=None, b=None, q=None, out=None, lse=None, ws=None, size=0):
        return L.wait_kv_attention(c or cache(), b or batch(), q or rows(), out or rows(), lse, ws,
                                   size, None)

    for bad in (dict(n_seq=-1), dict(n_tokens=-1), dict(heads=0), dict(heads=3),
                dict(table_cols=-1), dict(table_stride=-1), dict(scale=0.0), dict(scale=-1.0),
                dict(scale=math.nan), dict(scale=math.inf), dict(window=-1), dict(max_q_len=-1),
                dict(max_kv_len=-1), dict(table=None), dict(starts=None), dict(kv_lens=None),
                dict(table=FAKE + 2), dict(starts=FAKE + 1)):
        assert call(b=batch(**bad)) == B.WS_EINVAL, bad
    assert call(b=batch(n_tokens=1 << 30)) == B.WS_EUNSUPPORTED
    assert call(b=batch(table_cols=1 << 27)) == B.WS_EUNSUPPORTED
    assert call(q=rows(type=kv.FP32), out=rows(type=kv.FP32)) == B.WS_EINVAL
    assert call(q=rows(type=kv.FP16), out=rows(type=kv.FP16)) == B.WS_EINVAL  # the cache is bf16
    assert call(out=rows(type=kv.FP16)) == B.WS_EINVAL
    assert call(q=rows(data=None)) == call(lse=FAKE + 1) == B.WS_EINVAL
    long = batch(table_cols=1 << 12, max_kv_len=1 << 16)
    size = C.c_size_t()
    assert L.wait_kv_attention_workspace_bytes(cache(), long, size) == B.WS_OK and size.value > 0
    assert L.wait_kv_attention_workspace_bytes(cache(), long, None) == B.WS_EINVAL
    assert call(b=long, ws=FAKE, size=size.value - 1) == B.WS_EWORKSPACE
    assert call(b=long) == B.WS_EWORKSPACE
    assert call(b=long, ws=FAKE + 8, size=size.value) == B.WS_EINVAL
    assert call(b=batch(n_seq=0)) == B.WS_OK
    assert call(b=batch(n_tokens=0), q=rows(data=None), out=rows(data=None)) == B.WS_OK


def test_workspace_stays_small():
    """Parts are for few rows and long requests; a batch that fills the card
    has none, and prompts take none for the rows that they have."""
    L = kv._lib()

    def size(c, **kw):
        n = C.c_size_t()
        assert L.wait_kv_attention_workspace_bytes(c, batch(**kw), n) == B.WS_OK
        return n.value

    wide = cache(kv_heads=32, dim=128, pages=1 << 13)
    assert size(wide, n_seq=128, n_tokens=128, heads=32, max_q_len=1, max_kv_len=1512,
                table_cols=95) == 0
    one = size(cache(kv_heads=8, dim=128), n_seq=1, n_tokens=1, heads=64, max_q_len=1,
               max_kv_len=131072, table_cols=8192)
    assert 0 < one < 64 << 20
    assert size(wide, n_seq=2, n_tokens=16384, heads=32, max_q_len=8192, max_kv_len=8192,
                table_cols=512) < 64 << 20


def test_rotary_angles():
    f, by = kv.rotary_frequencies(8, base=100.0)
    assert by == 1.0
    assert torch.allclose(f, torch.tensor([1.0, 100 ** -0.25, 0.1, 100 ** -0.75],
                                          dtype=torch.float64), rtol=1e-15)
    lin, _ = kv.rotary_frequencies(8, scaling="linear", factor=4.0)
    assert torch.equal(lin * 4, kv.rotary_frequencies(8)[0])
    # the fastest pair as before, the slowest `factor` times slower
    ntk, _ = kv.rotary_frequencies(128, scaling="ntk", factor=8.0)
    plain = kv.rotary_frequencies(128)[0]
    assert float(ntk[0]) == 1.0 and abs(float(plain[-1] / ntk[-1]) - 8.0) < 1e-12
    yarn, by = kv.rotary_frequencies(128, scaling="yarn", factor=8.0, original=4096)
    turns = 4096 * plain / (2 * math.pi)
    assert torch.equal(yarn[turns >= 32], plain[turns >= 32])
    assert torch.allclose(yarn[turns <= 1], plain[turns <= 1] / 8, rtol=1e-15)
    between = (turns > 1) & (turns < 32)
    assert bool(((yarn < plain) & (yarn > plain / 8))[between].all())
    assert abs(by - (0.1 * math.log(8.0) + 1)) < 1e-15
    t = kv.rotary_table(50, 8, device="cpu", scaling="yarn", factor=2.0)
    f, by = kv.rotary_frequencies(8, scaling="yarn", factor=2.0)
    a = torch.arange(50, dtype=torch.float64)[:, None] * f
    assert t.shape == (50, 8) and t.dtype == torch.float32
    assert torch.equal(t, torch.cat([a.cos() * by, a.sin() * by], 1).float())
    for bad in (dict(part=7), dict(part=0), dict(part=8, scaling="other"),
                dict(part=8, factor=0.5), dict(part=8, base=0.0)):
        with pytest.raises(ValueError):
            kv.rotary_frequencies(**bad)


def test_python_refusals():
    """Wrong shapes, types, devices and layouts raise before any call."""
    x = torch.zeros(3, 2, 64)
    pos = torch.zeros(3, dtype=torch.int64)
    table = torch.zeros(10, 64)
    for args, kw in (((x[0], pos, table), {}), ((x.double(), pos, table), {}),
                     ((x, pos[:2], table), {}), ((x, pos.float(), table), {}),
                     ((x, pos, table.double()), {}), ((x, pos, torch.zeros(10, 66)), {}),
                     ((x, pos, torch.zeros(10, 31)), {}), ((x, pos, table[:, ::2]), {}),
                     ((x.transpose(1, 2), pos, table), {}),
                     ((x, pos, table), dict(out=x.half())),
                     ((x, pos, table), dict(out=torch.zeros(1, 2, 64).expand(3, 2, 64))),
                     ((x, pos, table), {})):            # the last: not on the GPU
        with pytest.raises(ValueError):
            kv.rotary(*args, **kw)
    c = kv.Cache.empty(2, 16, 2, 64, torch.int8, device="cpu")
    slots = torch.zeros(3, dtype=torch.int64)
    for args, kw in (((c, x, x.half(), slots), {}), ((c, x[:2], x[:2], slots), {}),
                     ((c, x[:, :1], x[:, :1], slots), {}), ((c, x, x, slots.int()), {}),
                     ((c, x, x, slots), dict(positions=pos)), ((c, x, x, slots), dict(table=table)),
                     ((c, x, x, slots), {})):
        with pytest.raises(ValueError):
            kv.append(*args, **kw)
    for args, kw in (((c, slots[None]), {}), ((c, slots, torch.int8), {}),
                     ((c, slots), dict(out=(x, x[:2]))), ((c, slots), {})):
        with pytest.raises(ValueError):
            kv.read(*args, **kw)
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    pages = torch.zeros(1, 2, dtype=torch.int32)
    starts, lens = torch.tensor([0, 3], dtype=torch.int32), torch.tensor([9], dtype=torch.int32)
    for args in ((q.float(), c, pages, starts, lens), (q[:, :3], c, pages, starts, lens),
                 (q[..., :32], c, pages, starts, lens), (q, c, pages.long(), starts, lens),
                 (q, c, pages[0], starts, lens), (q, c, pages, starts[:1], lens),
                 (q, c, pages, starts.long(), lens), (q, c, pages, starts, lens.long()),
                 (q, c, pages, starts, lens)):
        with pytest.raises(ValueError):
            kv.attention(*args)
    b16 = kv.Cache.empty(2, 16, 2, 64, torch.float16, device="cpu")
    with pytest.raises(ValueError):
        kv.attention(q, b16, pages, starts, lens)
    k = torch.zeros(2, 2, 16, 64, dtype=torch.int8)
    s = torch.zeros(2, 2, 16)
    for bad in ((k, k), (k, k[:1]), (k.float(), k.float()), (k[..., ::2], k[..., ::2], s, s),
                (k, k, s, s[:1]), (k, k, s.half(), s), (k.half(), k.half(), s, s), (k[0], k[0])):
        with pytest.raises(ValueError):
            kv.Cache(*bad)


def test_token_bytes():
    """524,288 bytes a token over 32 layers of 32 heads of 128 in 16 bits."""
    assert 32 * kv.Cache.token_bytes(32, 128, torch.float16) == 524288
    assert kv.Cache.token_bytes(8, 128, torch.int8) == 2 * 8 * (128 + 4)

"""The KV path of one serving iteration on the card: Python side of
include/wait_kv.h (argument checks and marshalling; PyTorch allocates buffers
and supplies the stream).

* ``rotary_table`` / ``rotary``: vectors turned by their positions.
* ``Cache``: one layer's paged cache, in 16 bits or quantised to 8.
* ``append``: new keys and values into the cache, the keys turned on the way.
* ``read``: rows of the cache back as values.
* ``attention``: every token's attention over its request's pages.

Every function runs asynchronously on the current stream of its tensors'
device and needs the HIP library: there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import math
import struct
from typing import Optional

import torch

from . import binding as B

BF16, FP16, FP32, FP8, INT8 = 0, 1, 2, 3, 4
_TYPE = {torch.bfloat16: BF16, torch.float16: FP16, torch.float32: FP32,
         torch.float8_e4m3fn: FP8, torch.int8: INT8}
_WIDE = (torch.bfloat16, torch.float16, torch.float32)
CACHE_TYPES = (torch.bfloat16, torch.float16, torch.float8_e4m3fn, torch.int8)
EIGHT_BIT = (torch.float8_e4m3fn, torch.int8)


# The structs of include/wait_kv.h, packed: a call's marshalling is most of a
# small operator's time, and bytes cost a fraction of ctypes' structures.
ROWS = struct.Struct("Pqqi4x")              # ws_kv_rows
TURN = struct.Struct("PPiiii")              # ws_kv_turn
CACHE = struct.Struct("PPPPiiiii4x")        # ws_kv_cache
BATCH = struct.Struct("Pqi4xPPiiifiiii")    # ws_kv_batch

_fn = None


def _lib():
    global _fn
    if _fn is None:
        L = B.lib()
        p, i64, i32, s = C.c_void_p, C.c_int64, C.c_int32, C.c_char_p
        L.wait_kv_rotary.argtypes = [s, s, i64, i32, i32, s, i32, p]
        L.wait_kv_append.argtypes = [s, s, s, p, i64, s, p]
        L.wait_kv_read.argtypes = [s, p, i64, s, s, p]
        L.wait_kv_attention_workspace_bytes.argtypes = [s, s, C.POINTER(C.c_size_t)]
        L.wait_kv_attention.argtypes = [s, s, s, s, p, p, C.c_size_t, p]
        _fn = L
    return _fn


def _stream(index: int) -> int:
    return torch.cuda.current_stream(index).cuda_stream


# the same without building objects, where this PyTorch has them
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _stream)
_current = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _run(fn, index: int, *args):
    """fn(*args, the current stream) on GPU number `index`."""
    if index < 0:
        raise ValueError("the operators run on the GPU")
    if _current() == index:
        rc = fn(*args, _stream(index))
    else:
        with torch.cuda.device(index):
            rc = fn(*args, _stream(index))
    if rc:
        B._check(rc)


def _need(ok: bool, msg: str):
    if not ok:
        raise ValueError(msg)


def _rows(t: torch.Tensor, name: str, index: int, types=_WIDE) -> bytes:
    """The struct of t [tokens, heads, dim], on GPU number `index`."""
    step = t.stride()
    dtype = t.dtype
    if len(step) != 3 or dtype not in types or step[2] != 1 or t.get_device() != index:
        _need(len(step) == 3, f"{name} must be [tokens, heads, dim]")
        _need(dtype in types, f"{name} must be one of {types}, is {dtype}")
        _need(step[2] == 1 or t.shape[2] == 1, f"{name}: a vector's elements must be contiguous")
        _need(t.get_device() == index, f"{name} must be on the same device, is on {t.device}")
    return ROWS.pack(t.data_ptr(), step[0], step[1], _TYPE[dtype])


def _fresh(t: torch.Tensor) -> bytes:
    """The struct of a contiguous tensor made here."""
    _, heads, dim = t.shape
    return ROWS.pack(t.data_ptr(), heads * dim, dim, _TYPE[t.dtype])


def _apart(t: torch.Tensor, name: str):
    """Refuse an output whose rows share memory."""
    need = t.shape[2]
    for size, step in sorted(((t.shape[0], t.stride(0)), (t.shape[1], t.stride(1))),
                             key=lambda x: abs(x[1])):
        if size > 1:
            _need(abs(step) >= need, f"{name}: rows must not overlap")
            need = abs(step) * (size - 1) + need


def _turn(positions, table, n: int, dim: int, interleaved: bool, index: int) -> bytes:
    if positions is None or table is None:
        raise ValueError("a rotation needs positions and a table")
    size = table.shape
    kind = positions.dtype
    if (len(size) != 2 or table.dtype is not torch.float32 or not table.is_contiguous()
            or positions.shape != (n,) or not positions.is_contiguous()
            or (kind is not torch.int64 and kind is not torch.int32) or size[1] % 2
            or not 2 <= size[1] <= dim or positions.get_device() != index
            or table.get_device() != index):
        _need(len(size) == 2 and table.dtype == torch.float32 and table.is_contiguous(),
              "table must be [positions, part], fp32, contiguous")
        _need(positions.shape == (n,) and positions.is_contiguous()
              and kind in (torch.int64, torch.int32),
              "positions must be one int64 or int32 a token, contiguous")
        _need(size[1] % 2 == 0 and 2 <= size[1] <= dim,
              "the table's part must be even, at least 2 and at most the head dimension")
        raise ValueError("positions and table must be on the vectors' device")
    return TURN.pack(table.data_ptr(), positions.data_ptr(), kind is torch.int32, size[0], size[1],
                     bool(interleaved))


# ----------------------------------------------------------------- rotary ----


def rotary_frequencies(part: int, base: float = 10000.0, scaling: Optional[str] = None,
                       factor: float = 1.0, original: int = 4096, fast: float = 32.0,
                       slow: float = 1.0):
    """(radians a position for each of the part / 2 pairs, factor of the
    result).  Pair i turns base^(-2 i / part) a position; contexts longer by
    ``factor`` than the ``original`` positions scale that:

    * ``"linear"``: positions are divided by the factor;
    * ``"ntk"``: the base is raised so that the slowest pair turns that much
      slower and the fastest as before;
    * ``"yarn"``: pairs that turn ``fast`` times or more within the original
      positions stay, those that turn ``slow`` times or less are divided by the
      factor, the others are blended; the result is multiplied by
      0.1 ln(factor) + 1.
    """
    _need(part >= 2 and part % 2 == 0, "the turned part must be even")
    _need(base > 0 and factor >= 1, "base must be positive and factor at least 1")
    i = torch.arange(part // 2, dtype=torch.float64)
    if scaling == "ntk" and part > 2:
        base = base * factor ** (part / (part - 2.0))
    f = base ** (-2.0 * i / part)
    if scaling in (None, "none", "ntk"):
        return f, 1.0
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "yarn":
        _need(fast > slow, "fast must exceed slow")
        keep = ((original * f / (2.0 * math.pi) - slow) / (fast - slow)).clamp(0.0, 1.0)
        return f * keep + f / factor * (1.0 - keep), 0.1 * math.log(factor) + 1.0
    raise ValueError(f"unknown scaling {scaling!r}")


def rotary_table(positions: int, part: int, device="cuda", **scaling) -> torch.Tensor:
    """[positions, part] fp32: the cosines of the pairs' angles, then their
    sines; angles are computed in 64 bits."""
    f, by = rotary_frequencies(part, **scaling)
    a = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * f.to(device)
    return torch.cat([a.cos() * by, a.sin() * by], dim=1).float()


def rotary(x: torch.Tensor, positions: torch.Tensor, table: torch.Tensor, *,
           interleaved: bool = False, inverse: bool = False,
           out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [tokens, heads, dim] with the first ``table.shape[1]`` elements of
    every vector turned by the token's position: pairs (i, i + part / 2), or
    (2 i, 2 i + 1) where ``interleaved``.  ``inverse`` turns back; that is the
    gradient's way through a rotation.  ``out`` may be x.  A position outside
    the table gives NaN."""
    fn = _lib().wait_kv_rotary
    index = x.get_device()
    xr = _rows(x, "x", index)
    n, heads, dim = x.shape
    t = _turn(positions, table, n, dim, interleaved, index)
    if out is None:
        out = torch.empty_like(x)
    else:
        _need(out.shape == x.shape and out.dtype == x.dtype, "out must have x's shape and type")
        _apart(out, "out")
        _rows(out, "out", index)
    if n and heads:
        step = out.stride()
        _run(fn, index, xr, ROWS.pack(out.data_ptr(), step[0], step[1], _TYPE[out.dtype]), n, heads,
             dim, t, inverse)
    return out


# ------------------------------------------------------------------ cache ----


class Cache:
    """One layer's cache: k and v [pages, kv_heads, page_size, dim], bf16, fp16,
    float8_e4m3fn or int8; 8-bit caches have fp32 scales
    [pages, kv_heads, page_size], an element stands for code * scale.  Token
    slot s is offset s % page_size of page s / page_size.  The page size is a
    power of two up to 1024, dim 64, 128 or 256."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
                 v_scale: Optional[torch.Tensor] = None):
        size, dtype, index = k.shape, k.dtype, k.get_device()
        if (len(size) != 4 or size != v.shape or dtype is not v.dtype or dtype not in CACHE_TYPES
                or not k.is_contiguous() or not v.is_contiguous() or v.get_device() != index):
            raise ValueError("k and v must both be [pages, kv_heads, page_size, dim] of one of "
                             f"{CACHE_TYPES}, contiguous, on one device")
        kp = vp = 0
        if dtype in EIGHT_BIT:
            _need(k_scale is not None and v_scale is not None, "an 8-bit cache needs scales")
            rows = size[:3]
            for t in (k_scale, v_scale):
                if (t.shape != rows or t.dtype is not torch.float32 or not t.is_contiguous()
                        or t.get_device() != index):
                    raise ValueError("scales must be [pages, kv_heads, page_size], fp32, "
                                     "contiguous, on the cache's device")
            kp, vp = k_scale.data_ptr(), v_scale.data_ptr()
        else:
            _need(k_scale is None and v_scale is None, "a 16-bit cache has no scales")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.pages, self.kv_heads, self.page_size, self.dim = size
        self.dtype, self.device, self._index = dtype, k.device, index
        self._c = CACHE.pack(k.data_ptr(), v.data_ptr(), kp, vp, self.pages, self.page_size,
                             self.kv_heads, self.dim, _TYPE[dtype])

    @classmethod
    def empty(cls, pages: int, page_size: int, kv_heads: int, dim: int,
              dtype: torch.dtype = torch.bfloat16, device="cuda") -> "Cache":
        shape = (pages, kv_heads, page_size, dim)
        k, v = (torch.zeros(shape, dtype=dtype, device=device) for _ in range(2))
        if dtype not in EIGHT_BIT:
            return cls(k, v)
        return cls(k, v, *(torch.zeros(shape[:3], device=device) for _ in range(2)))

    @staticmethod
    def token_bytes(kv_heads: int, dim: int, dtype: torch.dtype) -> int:
        """Bytes a token of one layer holds, scales included."""
        return 2 * kv_heads * (dim * dtype.itemsize + (4 if dtype in EIGHT_BIT else 0))


def _slots(slots: torch.Tensor, index: int) -> int:
    size = slots.shape
    _need(len(size) == 1 and slots.dtype is torch.int64 and slots.is_contiguous()
          and slots.get_device() == index,
          "slots must be one int64 a token, contiguous, on the cache's device")
    return size[0]


def append(cache: Cache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, *,
           positions: Optional[torch.Tensor] = None, table: Optional[torch.Tensor] = None,
           interleaved: bool = False) -> None:
    """Rows of k and v [tokens, kv_heads, dim] into the cache's slots, rounded
    or quantised row by row (include/wait_kv.h).  A token whose slot is
    negative, or behind the cache's end, is left out.  With ``positions`` and
    ``table`` the keys are turned first, as by ``rotary``, without a rounding
    between."""
    fn = _lib().wait_kv_append
    index = cache._index
    kr, vr = _rows(k, "k", index), _rows(v, "v", index)
    n = _slots(slots, index)
    _need(k.shape == (n, cache.kv_heads, cache.dim) and k.shape == v.shape and k.dtype is v.dtype,
          "k and v must be [slots, kv_heads, dim] of one type")
    t = None
    if positions is not None or table is not None:
        t = _turn(positions, table, n, cache.dim, interleaved, index)
    _run(fn, index, cache._c, kr, vr, slots.data_ptr(), n, t)


def read(cache: Cache, slots: torch.Tensor, dtype: torch.dtype = torch.bfloat16,
         out: Optional[tuple] = None) -> tuple:
    """(k, v) [slots, kv_heads, dim] of the cache's slots, as values rounded
    once to ``dtype``; zeros for a slot that the cache does not have."""
    fn = _lib().wait_kv_read
    index = cache._index
    n = _slots(slots, index)
    shape = (n, cache.kv_heads, cache.dim)
    if out is None:
        _need(dtype in _WIDE, f"dtype must be one of {_WIDE}")
        k = torch.empty(*shape, dtype=dtype, device=cache.device)
        v = torch.empty_like(k)
        kr, vr = _fresh(k), _fresh(v)
    else:
        k, v = out
        _need(k.shape == shape and v.shape == shape and k.dtype is v.dtype,
              "out must be two [slots, kv_heads, dim] of one type")
        _apart(k, "k")
        _apart(v, "v")
        kr, vr = _rows(k, "k", index), _rows(v, "v", index)
    _run(fn, index, cache._c, slots.data_ptr(), n, kr, vr)
    return k, v


# -------------------------------------------------------------- attention ----


def attention(q: torch.Tensor, cache: Cache, pages: torch.Tensor, starts: torch.Tensor,
              kv_lens: torch.Tensor, *, max_q_len: Optional[int] = None,
              max_kv_len: Optional[int] = None, scale: Optional[float] = None,
              causal: bool = True, window: int = 0, return_lse: bool = False,
              out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Attention of q [tokens, heads, dim] (bf16 or fp16) over the pages of its
    requests.  Request b has the queries starts[b] .. starts[b + 1] - 1, the last
    of its kv_lens[b] tokens; key j is at offset j % page_size of page
    pages[b, j // page_size].  A query at position p sees the keys j <= p
    (``causal``), and of those j > p - window (``window`` > 0); one that sees
    none gets zeros and a log-sum of -infinity.  Head h reads KV head
    h // (heads // kv_heads).  Entries of ``pages`` outside the cache mark keys
    that are not there.

    ``starts``, ``kv_lens`` and ``pages`` are int32 and stay on the device;
    ``max_q_len`` and ``max_kv_len`` bound the lengths for the launch's layout
    (by default from the shapes) and longer requests are only slower.
    Returns out, or (out, lse [tokens, heads] fp32).  ``workspace`` (a uint8
    tensor of ``attention_workspace_bytes``) is taken from PyTorch where it is
    not given."""
    L = _lib()
    index = cache._index
    qr = _rows(q, "q", index, _WIDE[:2])
    size = q.shape
    _need(size[2] == cache.dim, "q and the cache must have one head dimension")
    _need(cache.dtype in EIGHT_BIT or q.dtype is cache.dtype,
          "q must have the type of a 16-bit cache")
    batch, need = _batch(size, cache, pages, starts, kv_lens, max_q_len, max_kv_len, scale, causal,
                         window)
    if out is None:
        out = torch.empty_like(q)
    else:
        _need(out.shape == size and out.dtype is q.dtype, "out must have q's shape and type")
        _apart(out, "out")
    lse = torch.empty(size[:2], dtype=torch.float32, device=q.device) if return_lse else None
    ptr, have = None, 0
    if workspace is not None:
        _need(workspace.is_contiguous() and workspace.get_device() == index,
              "workspace must be contiguous, on the cache's device")
        ptr, have = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    elif need:
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
        ptr, have = workspace.data_ptr(), need
    _run(L.wait_kv_attention, index, cache._c, batch, qr, _rows(out, "out", index),
         None if lse is None else lse.data_ptr(), ptr, have)
    return out if lse is None else (out, lse)


def _batch(size, cache, pages, starts, kv_lens, max_q_len, max_kv_len, scale, causal, window):
    """(the struct of a batch, the bytes of its workspace)."""
    index = cache._index
    T, heads, dim = size
    n_seq, cols = pages.shape if pages.dim() == 2 else (-1, 0)
    step = pages.stride()
    if (n_seq < 0 or pages.dtype is not torch.int32 or (step[1] != 1 and cols > 1)
            or pages.get_device() != index):
        raise ValueError("pages must be [requests, pages], int32, rows contiguous, on the cache's "
                         "device")
    for t, n in ((starts, n_seq + 1), (kv_lens, n_seq)):
        if (t.shape != (n,) or t.dtype is not torch.int32 or not t.is_contiguous()
                or t.get_device() != index):
            raise ValueError("starts (one more than the requests) and kv_lens (one each) must be "
                             "int32, contiguous, on the cache's device")
    _need(heads >= 1 and heads % cache.kv_heads == 0, "heads must be a multiple of the cache's")
    cap = cols * cache.page_size
    b = BATCH.pack(pages.data_ptr(), step[0] if n_seq > 1 else cols, cols, starts.data_ptr(),
                   kv_lens.data_ptr(), n_seq, T, heads,
                   1.0 / math.sqrt(dim) if scale is None else scale, bool(causal),
                   min(window, 0x7fffffff),
                   T if max_q_len is None else min(max_q_len, T),
                   cap if max_kv_len is None else min(max_kv_len, cap))
    need = C.c_size_t()
    rc = _lib().wait_kv_attention_workspace_bytes(cache._c, b, need)
    if rc:
        B._check(rc)
    return b, need.value


def attention_workspace_bytes(q: torch.Tensor, cache: Cache, pages: torch.Tensor,
                              starts: torch.Tensor, kv_lens: torch.Tensor, *,
                              max_q_len: Optional[int] = None, max_kv_len: Optional[int] = None,
                              window: int = 0) -> int:
    """Bytes that ``attention`` takes as its workspace for these shapes."""
    return _batch(q.shape, cache, pages, starts, kv_lens, max_q_len, max_kv_len, None, True,
                  window)[1]

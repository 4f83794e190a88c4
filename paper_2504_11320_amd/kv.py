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
from typing import Optional

import torch

from . import binding as B

BF16, FP16, FP32, FP8, INT8 = 0, 1, 2, 3, 4
_TYPE = {torch.bfloat16: BF16, torch.float16: FP16, torch.float32: FP32,
         torch.float8_e4m3fn: FP8, torch.int8: INT8}
_WIDE = (torch.bfloat16, torch.float16, torch.float32)
CACHE_TYPES = (torch.bfloat16, torch.float16, torch.float8_e4m3fn, torch.int8)
EIGHT_BIT = (torch.float8_e4m3fn, torch.int8)


class _Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64),
                ("type", C.c_int32)]


class _Turn(C.Structure):
    _fields_ = [("table", C.c_void_p), ("positions", C.c_void_p), ("positions_32", C.c_int32),
                ("n_table", C.c_int32), ("part", C.c_int32), ("interleaved", C.c_int32)]


class _Cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p),
                ("v_scale", C.c_void_p), ("pages", C.c_int32), ("page_size", C.c_int32),
                ("kv_heads", C.c_int32), ("dim", C.c_int32), ("type", C.c_int32)]


class _Batch(C.Structure):
    _fields_ = [("table", C.c_void_p), ("table_stride", C.c_int64), ("table_cols", C.c_int32),
                ("starts", C.c_void_p), ("kv_lens", C.c_void_p), ("n_seq", C.c_int32),
                ("n_tokens", C.c_int32), ("heads", C.c_int32), ("scale", C.c_float),
                ("causal", C.c_int32), ("window", C.c_int32), ("max_q_len", C.c_int32),
                ("max_kv_len", C.c_int32)]


_fn = None


def _lib():
    global _fn
    if _fn is None:
        L = B.lib()
        rows, turn, cache, batch = (C.POINTER(t) for t in (_Rows, _Turn, _Cache, _Batch))
        p, i64, i32 = C.c_void_p, C.c_int64, C.c_int32
        L.wait_kv_rotary.argtypes = [rows, rows, i64, i32, i32, turn, i32, p]
        L.wait_kv_append.argtypes = [cache, rows, rows, p, i64, turn, p]
        L.wait_kv_read.argtypes = [cache, p, i64, rows, rows, p]
        L.wait_kv_attention_workspace_bytes.argtypes = [cache, batch, C.POINTER(C.c_size_t)]
        L.wait_kv_attention.argtypes = [cache, batch, rows, rows, p, p, C.c_size_t, p]
        _fn = L
    return _fn


def _stream(device) -> int:
    _need(device.type == "cuda", "the operators run on the GPU")
    return torch.cuda.current_stream(device).cuda_stream


def _need(ok: bool, msg: str):
    if not ok:
        raise ValueError(msg)


def _on(device, **tensors):
    for name, t in tensors.items():
        _need(t.device == device, f"{name} must be on {device}, is on {t.device}")


def _rows(t: torch.Tensor, name: str, types=_WIDE) -> _Rows:
    _need(t.dim() == 3, f"{name} must be [tokens, heads, dim]")
    _need(t.dtype in types, f"{name} must be one of {types}, is {t.dtype}")
    _need(t.stride(2) == 1 or t.shape[2] == 1, f"{name}: a vector's elements must be contiguous")
    return _Rows(t.data_ptr(), t.stride(0), t.stride(1), _TYPE[t.dtype])


def _apart(t: torch.Tensor, name: str):
    """Refuse an output whose rows share memory."""
    need = t.shape[2]
    for size, step in sorted(((t.shape[0], t.stride(0)), (t.shape[1], t.stride(1))),
                             key=lambda x: abs(x[1])):
        if size > 1:
            _need(abs(step) >= need, f"{name}: rows must not overlap")
            need = abs(step) * (size - 1) + need


def _turn(positions, table, n: int, dim: int, interleaved: bool, device) -> _Turn:
    _need(positions is not None and table is not None, "a rotation needs positions and a table")
    _need(table.dim() == 2 and table.dtype == torch.float32 and table.is_contiguous(),
          "table must be [positions, part], fp32, contiguous")
    _need(positions.dim() == 1 and positions.shape[0] == n and positions.is_contiguous()
          and positions.dtype in (torch.int64, torch.int32),
          "positions must be one int64 or int32 a token, contiguous")
    part = table.shape[1]
    _need(part % 2 == 0 and 2 <= part <= dim,
          "the table's part must be even, at least 2 and at most the head dimension")
    _on(device, positions=positions, table=table)
    return _Turn(table.data_ptr(), positions.data_ptr(), positions.dtype == torch.int32,
                 table.shape[0], part, bool(interleaved))


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
    L = _lib()
    xr = _rows(x, "x")
    n, heads, dim = x.shape
    t = _turn(positions, table, n, dim, interleaved, x.device)
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    _need(out.shape == x.shape and out.dtype == x.dtype, "out must have x's shape and type")
    _on(x.device, out=out)
    _apart(out, "out")
    if n == 0 or heads == 0:
        return out
    B._check(L.wait_kv_rotary(xr, _rows(out, "out"), n, heads, dim, t, inverse,
                              _stream(x.device)))
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
        _need(k.dim() == 4 and k.shape == v.shape and k.dtype == v.dtype,
              "k and v must both be [pages, kv_heads, page_size, dim] of one type")
        _need(k.dtype in CACHE_TYPES, f"a cache's type is one of {CACHE_TYPES}")
        _need(k.is_contiguous() and v.is_contiguous(), "k and v must be contiguous")
        _on(k.device, v=v)
        ptr = [None, None]
        if k.dtype in EIGHT_BIT:
            _need(k_scale is not None and v_scale is not None, "an 8-bit cache needs scales")
            for i, (n, s) in enumerate((("k_scale", k_scale), ("v_scale", v_scale))):
                _need(s.shape == k.shape[:3] and s.dtype == torch.float32 and s.is_contiguous(),
                      f"{n} must be [pages, kv_heads, page_size], fp32, contiguous")
                _on(k.device, **{n: s})
                ptr[i] = s.data_ptr()
        else:
            _need(k_scale is None and v_scale is None, "a 16-bit cache has no scales")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.pages, self.kv_heads, self.page_size, self.dim = k.shape
        self.dtype, self.device = k.dtype, k.device
        self._c = _Cache(k.data_ptr(), v.data_ptr(), ptr[0], ptr[1], self.pages, self.page_size,
                         self.kv_heads, self.dim, _TYPE[k.dtype])

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


def _slots(slots: torch.Tensor, device) -> int:
    _need(slots.dim() == 1 and slots.dtype == torch.int64 and slots.is_contiguous(),
          "slots must be one int64 a token, contiguous")
    _on(device, slots=slots)
    return slots.shape[0]


def append(cache: Cache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, *,
           positions: Optional[torch.Tensor] = None, table: Optional[torch.Tensor] = None,
           interleaved: bool = False) -> None:
    """Rows of k and v [tokens, kv_heads, dim] into the cache's slots, rounded
    or quantised row by row (include/wait_kv.h).  A token whose slot is
    negative, or behind the cache's end, is left out.  With ``positions`` and
    ``table`` the keys are turned first, as by ``rotary``, without a rounding
    between."""
    L = _lib()
    kr, vr = _rows(k, "k"), _rows(v, "v")
    n = _slots(slots, cache.device)
    _need(k.shape == v.shape == (n, cache.kv_heads, cache.dim) and k.dtype == v.dtype,
          "k and v must be [slots, kv_heads, dim] of one type")
    _on(cache.device, k=k, v=v)
    t = None
    if positions is not None or table is not None:
        t = _turn(positions, table, n, cache.dim, interleaved, cache.device)
    B._check(L.wait_kv_append(cache._c, kr, vr, slots.data_ptr(), n, t, _stream(cache.device)))


def read(cache: Cache, slots: torch.Tensor, dtype: torch.dtype = torch.bfloat16,
         out: Optional[tuple] = None) -> tuple:
    """(k, v) [slots, kv_heads, dim] of the cache's slots, as values rounded
    once to ``dtype``; zeros for a slot that the cache does not have."""
    L = _lib()
    n = _slots(slots, cache.device)
    shape = (n, cache.kv_heads, cache.dim)
    if out is None:
        _need(dtype in _WIDE, f"dtype must be one of {_WIDE}")
        out = tuple(torch.empty(shape, dtype=dtype, device=cache.device) for _ in range(2))
    k, v = out
    _need(k.shape == v.shape == shape and k.dtype == v.dtype,
          "out must be two [slots, kv_heads, dim] of one type")
    _on(cache.device, k=k, v=v)
    _apart(k, "k")
    _apart(v, "v")
    B._check(L.wait_kv_read(cache._c, slots.data_ptr(), n, _rows(k, "k"), _rows(v, "v"),
                            _stream(cache.device)))
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
    qr = _rows(q, "q", _WIDE[:2])
    T, heads, dim = q.shape
    _need(dim == cache.dim, "q and the cache must have one head dimension")
    _need(heads >= 1 and heads % cache.kv_heads == 0, "heads must be a multiple of the cache's")
    _need(cache.dtype in EIGHT_BIT or q.dtype == cache.dtype,
          "q must have the type of a 16-bit cache")
    batch = _batch(q, cache, pages, starts, kv_lens, max_q_len, max_kv_len, scale, causal, window)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    _need(out.shape == q.shape and out.dtype == q.dtype, "out must have q's shape and type")
    _on(cache.device, q=q, out=out)
    _apart(out, "out")
    lse = torch.empty((T, heads), device=q.device) if return_lse else None
    need = C.c_size_t()
    B._check(L.wait_kv_attention_workspace_bytes(cache._c, batch, need))
    if need.value and workspace is None:
        workspace = torch.empty(need.value, dtype=torch.uint8, device=q.device)
    ptr, size = None, 0
    if workspace is not None:
        _need(workspace.is_contiguous(), "workspace must be contiguous")
        _on(cache.device, workspace=workspace)
        ptr, size = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    B._check(L.wait_kv_attention(cache._c, batch, qr, _rows(out, "out"),
                                 lse.data_ptr() if return_lse else None, ptr, size,
                                 _stream(q.device)))
    return (out, lse) if return_lse else out


def _batch(q, cache, pages, starts, kv_lens, max_q_len, max_kv_len, scale, causal, window):
    _need(pages.dim() == 2 and pages.dtype == torch.int32
          and (pages.stride(1) == 1 or pages.shape[1] <= 1),
          "pages must be [requests, pages], int32, rows contiguous")
    n_seq = pages.shape[0]
    for name, t, size in (("starts", starts, n_seq + 1), ("kv_lens", kv_lens, n_seq)):
        _need(t.dim() == 1 and t.shape[0] == size and t.dtype == torch.int32
              and t.is_contiguous(), f"{name} must be {size} int32, contiguous")
    _on(cache.device, pages=pages, starts=starts, kv_lens=kv_lens)
    T, heads, dim = q.shape
    cap = pages.shape[1] * cache.page_size
    return _Batch(pages.data_ptr(), pages.stride(0) if n_seq > 1 else pages.shape[1],
                  pages.shape[1], starts.data_ptr(), kv_lens.data_ptr(), n_seq, T, heads,
                  1.0 / math.sqrt(dim) if scale is None else scale, bool(causal), window,
                  T if max_q_len is None else min(max_q_len, T),
                  cap if max_kv_len is None else min(max_kv_len, cap))


def attention_workspace_bytes(q: torch.Tensor, cache: Cache, pages: torch.Tensor,
                              starts: torch.Tensor, kv_lens: torch.Tensor, *,
                              max_q_len: Optional[int] = None, max_kv_len: Optional[int] = None,
                              window: int = 0) -> int:
    """Bytes that ``attention`` takes as its workspace for these shapes."""
    b = _batch(q, cache, pages, starts, kv_lens, max_q_len, max_kv_len, None, True, window)
    need = C.c_size_t()
    B._check(_lib().wait_kv_attention_workspace_bytes(cache._c, b, need))
    return need.value

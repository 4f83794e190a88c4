"""The KV path of one serving iteration on the card: Python side of
include/wait_kv.h (the argument checks are in csrc/kv_binding.cpp; PyTorch
allocates buffers and supplies the stream).

* ``rotary_table`` / ``rotary``: vectors turned by their positions.
* ``Cache``: one layer's paged cache, in 16 bits or quantised to 8.
* ``append``: new keys and values into the cache, the keys turned on the way.
* ``read``: rows of the cache back as values.
* ``attention``: every token's attention over its request's pages.

Every function runs asynchronously on the current stream of its tensors'
device and needs the HIP library: there is no fallback.  Results carry no
gradients, and tensors that require one are refused where autograd records (a
rotation's gradient is ``rotary`` with ``inverse``, to be called from the
backward of a ``torch.autograd.Function``).
"""
from __future__ import annotations

import ctypes as C
import math
import os
import struct
from typing import Optional

import torch

from . import binding as B

BF16, FP16, FP32, FP8, INT8 = 0, 1, 2, 3, 4
CACHE_TYPES = (torch.bfloat16, torch.float16, torch.float8_e4m3fn, torch.int8)
EIGHT_BIT = (torch.float8_e4m3fn, torch.int8)


BINDING = os.path.join(B.PKG, "_kv.so")

# The structs of include/wait_kv.h, for calls of the C ABI through ``_lib``.
ROWS = struct.Struct("Pqqi4x")              # ws_kv_rows
TURN = struct.Struct("PPiiii")              # ws_kv_turn
CACHE = struct.Struct("PPPPiiiii4x")        # ws_kv_cache
BATCH = struct.Struct("Pqi4xPPiiifiiii")    # ws_kv_batch

_fn = _kv = None


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


def _native():
    """The checks and calls in C++ (csrc/kv_binding.cpp), bound to the library."""
    global _kv
    if _kv is None:
        if not os.path.exists(BINDING):
            raise RuntimeError(f"{BINDING} is missing: build it with paper_2504_11320_amd/build.py")
        from . import _kv as native
        L = _lib()
        # streams and devices without building objects, where this PyTorch can
        stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                         lambda i: torch.cuda.current_stream(i).cuda_stream)
        current = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        native.bind(*(C.cast(f, C.c_void_p).value for f in (
            L.wait_kv_rotary, L.wait_kv_append, L.wait_kv_read,
            L.wait_kv_attention_workspace_bytes, L.wait_kv_attention)),
            B._check, stream, current, torch.cuda.device)
        _kv = native
    return _kv


def _need(ok: bool, msg: str):
    if not ok:
        raise ValueError(msg)


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
    gradient's way through a rotation.  ``out`` may be x, and must not overlap
    it otherwise.  A position outside the table gives NaN."""
    return _native().rotary(x, positions, table, interleaved, inverse, out)


# ------------------------------------------------------------------ cache ----


def _held(i: int, name: str) -> property:
    def get(cache):
        return cache._tensors[i]

    def same(cache, tensor):   # what `cache.k *= 2` assigns
        if tensor is not cache._tensors[i]:
            raise AttributeError(f"a cache keeps its {name}: make another one")

    return property(get, same)


class Cache:
    """One layer's cache: k and v [pages, kv_heads, page_size, dim], bf16, fp16,
    float8_e4m3fn or int8; 8-bit caches have fp32 scales
    [pages, kv_heads, page_size], an element stands for code * scale.  Token
    slot s is offset s % page_size of page s / page_size.  The page size is a
    power of two up to 1024, dim 64, 128 or 256.  The tensors' addresses are
    kept: they cannot be exchanged, and their memory must stay theirs."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
                 v_scale: Optional[torch.Tensor] = None):
        self._c = _native().cache(k, v, k_scale, v_scale)
        self._tensors, self._index = (k, v, k_scale, v_scale), k.get_device()

    def __reduce__(self):   # copies and pickles have addresses of their own
        return type(self), self._tensors

    k, v, k_scale, v_scale = (_held(i, n) for i, n in enumerate(("k", "v", "k_scale", "v_scale")))
    pages, kv_heads, page_size, dim = (property(lambda self, i=i: self._tensors[0].shape[i])
                                       for i in range(4))
    dtype = property(lambda self: self._tensors[0].dtype)
    device = property(lambda self: self._tensors[0].device)

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


def append(cache: Cache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, *,
           positions: Optional[torch.Tensor] = None, table: Optional[torch.Tensor] = None,
           interleaved: bool = False) -> None:
    """Rows of k and v [tokens, kv_heads, dim] into the cache's slots, rounded
    or quantised row by row (include/wait_kv.h).  A token whose slot is
    negative, or behind the cache's end, is left out; the other slots must differ
    (two tokens with one slot leave a mixture of both).  With ``positions`` and
    ``table`` the keys are turned first, as by ``rotary``, without a rounding
    between."""
    _native().append(cache._c, cache._index, k, v, slots, positions, table, interleaved,
                     cache._tensors)


def read(cache: Cache, slots: torch.Tensor, dtype: torch.dtype = torch.bfloat16,
         out: Optional[tuple] = None) -> tuple:
    """(k, v) [slots, kv_heads, dim] of the cache's slots, as values rounded
    once to ``dtype``; zeros for a slot that the cache does not have."""
    a, b = (None, None) if out is None else out
    return _native().read(cache._c, cache._index, slots, dtype, a, b)


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
    (by default from the shapes).  Requests beyond them are computed all the
    same, only slower; bounds far above the lengths cost time and workspace too,
    so a caller that knows the lengths gives them.
    Returns out, or (out, lse [tokens, heads] fp32); rows of queries outside every
    request stay as they are in a given ``out``, and are undefined otherwise.
    ``out`` may be q, and must not overlap it otherwise.  ``workspace`` (a uint8
    tensor of ``attention_workspace_bytes``) is taken from PyTorch where it is
    not given."""
    return _native().attention(cache._c, cache._index, q, pages, starts, kv_lens, max_q_len,
                               max_kv_len, scale, causal, window, return_lse, out, workspace)


def attention_workspace_bytes(q: torch.Tensor, cache: Cache, pages: torch.Tensor,
                              starts: torch.Tensor, kv_lens: torch.Tensor, *,
                              max_q_len: Optional[int] = None, max_kv_len: Optional[int] = None,
                              window: int = 0) -> int:
    """Bytes that ``attention`` takes as its workspace for these shapes."""
    return _native().attention_workspace_bytes(cache._c, cache._index, q, pages, starts, kv_lens,
                                               max_q_len, max_kv_len, window)

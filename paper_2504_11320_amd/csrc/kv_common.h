// Shared parts of the KV-path operators: error reporting on the host,
// element types and conversions on the device.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <new>

#include "wait_kv.h"
#include "wait_sim.h"

// The message behind wait_sim_last_error() (wait_sim_host.hip).
__attribute__((visibility("hidden"))) int ws_record_failure(int code, const char *msg) noexcept;
__attribute__((visibility("hidden"))) void ws_clear_failure() noexcept;

namespace kv {

// ------------------------------------------------------------- host -----

// Body of an extern "C" entry point: no C++ exception crosses the C ABI.
template <class F>
int guarded(F &&body) noexcept {
  try {
    ws_clear_failure();
    return body();
  } catch (const std::bad_alloc &) {
    return ws_record_failure(WS_ENOMEM, "host memory allocation failed");
  } catch (...) {
    return ws_record_failure(WS_EINTERNAL, "internal error (unexpected C++ exception)");
  }
}

inline int invalid(const char *msg) { return ws_record_failure(WS_EINVAL, msg); }

// The status of a launch just made.
inline int launched() {
  hipError_t e = hipGetLastError();
  return e == hipSuccess ? WS_OK : ws_record_failure(WS_EDEVICE, hipGetErrorString(e));
}

inline int type_bytes(int t) { return t == WS_KV_FP32 ? 4 : t == WS_KV_BF16 || t == WS_KV_FP16 ? 2 : 1; }
inline bool is_wide(int t) { return t == WS_KV_BF16 || t == WS_KV_FP16 || t == WS_KV_FP32; }
inline bool is_8bit(int t) { return t == WS_KV_FP8 || t == WS_KV_INT8; }

// Whether `bytes`-wide accesses at multiples of `bytes` within every vector are
// aligned.
inline bool aligned(const ws_kv_rows &r, int bytes) {
  int e = type_bytes(r.type);
  return (uintptr_t)r.data % bytes == 0 && (uint64_t)r.token_stride * e % bytes == 0 &&
         (uint64_t)r.head_stride * e % bytes == 0;
}

inline int check_rows(const ws_kv_rows *r, int64_t n, const char *null_msg) {
  if (!r || (n > 0 && !r->data)) return invalid(null_msg);
  if (!is_wide(r->type)) return invalid("rows must be bf16, fp16 or fp32");
  if ((uintptr_t)r->data % type_bytes(r->type)) return invalid("rows must be aligned to their type");
  return WS_OK;
}

// Whether vectors of a share memory with vectors of b: n tokens of `heads` of
// dim elements of one size each.  Exact where the token strides are the same, as
// of parts of one buffer's rows; others share it if their ranges meet.
inline bool overlap(const ws_kv_rows &a, const ws_kv_rows &b, int64_t n, int64_t heads, int64_t dim) {
  using wide = __int128;
  if (n < 1 || heads < 1 || dim < 1) return false;
  const wide e = type_bytes(a.type), len = dim * e;
  struct Span {
    wide at, lo, hi;
  };
  auto span = [&](const ws_kv_rows &r) {
    const wide tokens = (wide)(n - 1) * r.token_stride * e, step = (wide)(heads - 1) * r.head_stride * e;
    const wide at = (wide)(uintptr_t)r.data, none = 0;
    return Span{at, at + (tokens < 0 ? tokens : none) + (step < 0 ? step : none),
                at + (tokens > 0 ? tokens : none) + (step > 0 ? step : none) + len};
  };
  const Span x = span(a), y = span(b);
  if (x.hi <= y.lo || y.hi <= x.lo) return false;
  if (n > 1 && a.token_stride != b.token_stride) return true;
  // heads i of a and j of b are `apart` bytes apart at one token, and by a
  // multiple of `step` more at others
  const wide step = n > 1 ? (wide)a.token_stride * e : 0;
  auto meet = [&](wide apart) {
    wide k = step ? -apart / step : 0;  // towards zero: k or a neighbour is nearest
    for (wide d = k - 1; d <= k + 1; ++d) {
      if (d <= -n || d >= n) continue;
      const wide gap = apart + d * step;
      if (gap > -len && gap < len) return true;
    }
    return false;
  };
  const bool same = a.head_stride == b.head_stride;
  for (int64_t i = 0; i < heads; ++i)
    for (int64_t j = 0; j < heads; ++j) {
      if (same && i && j) break;  // differences of heads, each once
      if (meet(y.at - x.at + ((wide)j * b.head_stride - (wide)i * a.head_stride) * e)) return true;
    }
  return false;
}
inline bool one_place(const ws_kv_rows &a, const ws_kv_rows &b) {
  return a.data == b.data && a.token_stride == b.token_stride && a.head_stride == b.head_stride;
}

inline int check_cache(const ws_kv_cache *c) {
  if (!c || !c->k || !c->v) return invalid("the cache's k and v must be non-NULL");
  if (c->dim != 64 && c->dim != 128 && c->dim != 256)
    return ws_record_failure(WS_EUNSUPPORTED, "the cache's head dimension must be 64, 128 or 256");
  if (c->page_size < 1 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)))
    return invalid("the page size must be a power of two up to 1024");
  if (c->pages < 1 || c->kv_heads < 1) return invalid("a cache needs pages and heads");
  if ((__int128)c->pages * c->kv_heads * c->page_size >= ((__int128)1 << 31))
    return ws_record_failure(WS_EUNSUPPORTED, "the cache has 2^31 rows or more");
  if (c->type != WS_KV_BF16 && c->type != WS_KV_FP16 && !is_8bit(c->type))
    return invalid("the cache's type must be bf16, fp16, fp8 or int8");
  if ((uintptr_t)c->k % 16 || (uintptr_t)c->v % 16) return invalid("k and v must be 16-byte aligned");
  if (is_8bit(c->type) ? (!c->k_scale || !c->v_scale) : (c->k_scale || c->v_scale))
    return invalid("an 8-bit cache has k_scale and v_scale, a 16-bit one has none");
  if ((uintptr_t)c->k_scale % 4 || (uintptr_t)c->v_scale % 4)
    return invalid("scales must be aligned to 4 bytes");
  return WS_OK;
}

// A rotation of vectors of dim elements.
inline int check_turn(const ws_kv_turn *t, int64_t n, int dim) {
  if (!t || (n > 0 && !t->positions)) return invalid("a rotation needs positions");
  if (t->n_table < 0 || (t->n_table > 0 && !t->table)) return invalid("a rotation needs its table");
  if (t->part < 2 || t->part > dim || t->part % 2)
    return invalid("the turned part must be even, at least 2 and at most the head dimension");
  if ((uintptr_t)t->table % 4 || (uintptr_t)t->positions % (t->positions_32 ? 4 : 8))
    return invalid("table and positions must be aligned to their types");
  return WS_OK;
}

inline int log2_of(int x) { return __builtin_ctz((unsigned)x); }

// ----------------------------------------------------------- device -----

using half2v = _Float16 __attribute__((ext_vector_type(2)));
using half8 = _Float16 __attribute__((ext_vector_type(8)));
using bf8v = __bf16 __attribute__((ext_vector_type(8)));
using bf2v = __bf16 __attribute__((ext_vector_type(2)));
using short4v = short __attribute__((ext_vector_type(4)));
using f32x4 = float __attribute__((ext_vector_type(4)));
using f32x16 = float __attribute__((ext_vector_type(16)));
using u32x2 = uint32_t __attribute__((ext_vector_type(2)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));

// Row of a cache that no key has: nothing is read for it.
constexpr int kNoRow = -1;

__device__ __forceinline__ float bf16_value(uint32_t bits) { return __uint_as_float(bits << 16); }

// Round to nearest, ties to even; a NaN stays one.
__device__ __forceinline__ uint16_t bf16_bits(float x) {
  return __builtin_bit_cast(uint16_t, (__bf16)x);
}

// Elements of a wide type as floats and back; T is one of the tags below.
struct Bf16 {
  using raw = uint16_t;
  static __device__ __forceinline__ float get(raw r) { return bf16_value(r); }
  static __device__ __forceinline__ raw put(float x) { return bf16_bits(x); }
};
struct Fp16 {
  using raw = uint16_t;
  static __device__ __forceinline__ float get(raw r) { return (float)__builtin_bit_cast(_Float16, r); }
  static __device__ __forceinline__ raw put(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
};
struct Fp32 {
  using raw = uint32_t;
  static __device__ __forceinline__ float get(raw r) { return __uint_as_float(r); }
  static __device__ __forceinline__ raw put(float x) { return __float_as_uint(x); }
};

// N elements of type T at p, in as few accesses as VEC allows (VEC elements
// each; the caller vouches for their alignment).
template <class T, int N, int VEC>
__device__ __forceinline__ void load_raw(const typename T::raw *p, typename T::raw (&x)[N]) {
  struct alignas(VEC * sizeof(typename T::raw)) Pack {
    typename T::raw r[VEC];
  };
#pragma unroll
  for (int i = 0; i < N; i += VEC) {
    Pack v = *reinterpret_cast<const Pack *>(p + i);
#pragma unroll
    for (int j = 0; j < VEC; ++j) x[i + j] = v.r[j];
  }
}
template <class T, int N, int VEC>
__device__ __forceinline__ void load_n(const typename T::raw *p, float (&x)[N]) {
  typename T::raw r[N];
  load_raw<T, N, VEC>(p, r);
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = T::get(r[i]);
}
// STREAM: past the caches, for outputs that these cannot hold.
template <class T, int N, int VEC, bool STREAM = false>
__device__ __forceinline__ void store_n(typename T::raw *p, const float (&x)[N]) {
  struct alignas(VEC * sizeof(typename T::raw)) Pack {
    typename T::raw r[VEC];
  };
#pragma unroll
  for (int i = 0; i < N; i += VEC) {
    Pack v;
#pragma unroll
    for (int j = 0; j < VEC; ++j) v.r[j] = T::put(x[i + j]);
    if constexpr (STREAM && sizeof(Pack) == 16)
      __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), reinterpret_cast<u32x4 *>(p + i));
    else
      *reinterpret_cast<Pack *>(p + i) = v;
  }
}

// Four 8-bit codes as four halves: both code sets are subsets of the 16-bit
// floats, so this is exact.  Integers: u = code + 128 behind the exponent of
// 1024 is 1024 + u, less 1152.
__device__ __forceinline__ u32x2 codes_to_half_fp8(uint32_t w) {
  half2v lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false);
  half2v hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true);
  return u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}
__device__ __forceinline__ u32x2 codes_to_half_int8(uint32_t w) {
  w ^= 0x80808080u;
  half2v lo = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u));
  half2v hi = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u));
  const half2v bias = {(_Float16)1152.0f, (_Float16)1152.0f};
  lo -= bias;
  hi -= bias;
  return u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}
template <int TYPE>
__device__ __forceinline__ u32x2 codes_to_half(uint32_t w) {
  if constexpr (TYPE == WS_KV_FP8) return codes_to_half_fp8(w);
  return codes_to_half_int8(w);
}

}  // namespace kv

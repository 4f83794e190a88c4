// A batch of requests over the pages of a cache, as attention and the
// operators beside it see it: a request's tokens and keys, the keys a token
// sees, the rows of the cache that they have; and the matrix instructions.
// Args has the fields of attention's arguments that are named here.
#pragma once

#include "kv_common.h"

namespace kv {

// The queries of request b and its keys.
struct Seq {
  int32_t q0, n, m;
};
template <class Args>
__device__ __forceinline__ Seq get_seq(const Args &a, int32_t b) {
  Seq s;
  s.q0 = min(max(a.starts[b], 0), a.n_tokens);
  s.n = min(max(a.starts[b + 1], s.q0), a.n_tokens) - s.q0;
  s.m = max(a.lens[b], 0);
  return s;
}

// The last request for which `before` holds, which holds up to some request and
// not behind it; -1 where for none.  A wave asks for 64 at once.
template <class Args, class F>
__device__ __forceinline__ int32_t last_at_most(const Args &a, F &&before) {
  int32_t b = -1;
  for (int32_t from = 0; from < a.n_seq; from += 64) {
    const int32_t i = from + (threadIdx.x & 63);
    const uint64_t yes = __ballot(i < a.n_seq && before(i));
    b += __popcll(yes);
    if (yes != ~0ull) break;
  }
  return __builtin_amdgcn_readfirstlane(b);
}

// Keys [lo, hi) that token i of the request sees.
struct Range {
  int32_t lo, hi;
};
template <class Args>
__device__ __forceinline__ Range token_range(const Args &a, const Seq &s, int32_t i) {
  Range r;
  const int32_t p = s.m - s.n + i;
  r.hi = min(s.m, a.capacity);
  if (a.causal) r.hi = max(min(r.hi, p + 1), 0);
  r.lo = a.window ? max(max(p, 0) - a.window + 1, 0) : 0;
  r.lo = min(r.lo, r.hi);
  return r;
}

// Key j of a request, 0 < end: its page's entry in the table, read ahead (the
// last key's behind the end), and the row of the cache that it has for KV head h.
template <class Args>
__device__ __forceinline__ int32_t page_entry(const Args &a, int32_t b, int32_t j, int32_t end) {
  return a.table[b * a.table_stride + (min(j, end - 1) >> a.page_shift)];
}
template <class Args>
__device__ __forceinline__ int32_t cache_row(const Args &a, int32_t page, int32_t h, int32_t j,
                                             int32_t end) {
  const bool is = (j < end) & ((uint32_t)page < (uint32_t)a.pages);
  const int32_t row = ((page * a.kv_heads + h) << a.page_shift) + (j & ((1 << a.page_shift) - 1));
  return is ? row : kNoRow;
}

template <bool BF>
__device__ __forceinline__ f32x4 mfma16(u32x4 x, u32x4 y, f32x4 c) {
  if constexpr (BF)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8v, x),
                                                   __builtin_bit_cast(bf8v, y), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, x),
                                                  __builtin_bit_cast(half8, y), c, 0, 0, 0);
}
template <bool BF>
__device__ __forceinline__ f32x16 mfma32(u32x4 x, u32x4 y, f32x16 c) {
  if constexpr (BF)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8v, x),
                                                   __builtin_bit_cast(bf8v, y), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, x),
                                                  __builtin_bit_cast(half8, y), c, 0, 0, 0);
}

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

template <int TYPE>
constexpr bool kBf = TYPE == WS_KV_BF16;
template <int TYPE>
constexpr bool kCodes = TYPE == WS_KV_FP8 || TYPE == WS_KV_INT8;

// 16 bytes a lane from memory to shared memory, the lanes' one after another
// from `to` on, without a register between.  They are there after
// await_copies(), for this wave; the compiler knows of neither.
__device__ __forceinline__ void copy_to_lds(const char *from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
               :
               : "v"(from), "s"(__builtin_amdgcn_readfirstlane(to))
               : "memory");
}
__device__ __forceinline__ void await_copies() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

}  // namespace kv

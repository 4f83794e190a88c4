// Rows of vectors: the angles of a rotation, rows into a cache, launches over
// many tokens.
#pragma once

#include <cmath>

#include "kv_common.h"

namespace kv {

struct TurnArgs {
  const float *table;
  const void *positions;
  int32_t positions_32, n_table, part;
};

// A token's position as its two words (of 32 bits: twice the only one), asked for
// and not yet waited for.
struct Position {
  uint32_t lo, hi;
};
__device__ __forceinline__ Position ask_position(const TurnArgs &t, int64_t i) {
  const uint32_t *p = (const uint32_t *)t.positions + (t.positions_32 ? i : 2 * i);
  return {p[0], p[t.positions_32 ? 0 : 1]};
}
// Nothing is asked for later than this that is written before it, and the
// position is used behind it only.
__device__ __forceinline__ void all_asked(Position &p) {
  asm volatile("" : "+v"(p.lo), "+v"(p.hi) : : "memory");
}
// The table's row of a position, or NULL where it has none.
__device__ __forceinline__ const float *turn_row(const TurnArgs &t, Position p) {
  const bool is = p.lo < (uint32_t)t.n_table && (t.positions_32 || p.hi == 0);
  return is ? t.table + (int64_t)p.lo * t.part : nullptr;
}

// How a row of 8-bit codes is scaled, by its largest magnitude's bits (these
// order as the magnitudes do, a NaN's behind the infinities).
template <int TYPE>
struct Coding {
  static constexpr float most = TYPE == WS_KV_FP8 ? 448.0f : 127.0f;
  float by, scale;  // of the codes, of the row
  bool some;        // not a row of zeros
  __device__ __forceinline__ explicit Coding(uint32_t top) {
    const float t = __uint_as_float(top);
    some = t >= 0x1p-100f && top < 0x7f800000u;
    by = some ? (1.0f / t) * most : 0.0f;
    scale = top >= 0x7f800000u ? NAN : some ? t / most : 0.0f;
  }
  __device__ __forceinline__ float clipped(float u) const {
    return __builtin_amdgcn_fmed3f(u * by, -most, most);
  }
  // Eight codes.
  __device__ __forceinline__ u32x2 codes(const float (&u)[8]) const {
    u32x2 code = {0, 0};
    if (!some) return code;
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = clipped(u[i]);
    if constexpr (TYPE == WS_KV_FP8) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
        code[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], w, true);
      }
    } else {
      // at 1.5 * 2^23 the last place of a float is 1: the low byte is the code
      uint32_t n[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) n[i] = __float_as_uint(y[i] + 12582912.0f);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t lo = __builtin_amdgcn_perm(n[4 * i + 1], n[4 * i], 0x0c0c0400u);
        const uint32_t hi = __builtin_amdgcn_perm(n[4 * i + 3], n[4 * i + 2], 0x04000c0cu);
        code[i] = lo | hi;
      }
    }
    return code;
  }
};
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// The eight elements of this lane into the cache's row: G lanes hold a row.
template <int TYPE, int G>
__device__ __forceinline__ void put_row(void *base, float *scales, int64_t row, int lane, int dim,
                                        const float (&u)[8]) {
  if constexpr (TYPE == WS_KV_BF16) {
    store_n<Bf16, 8, 8>((uint16_t *)base + row * dim + lane * 8, u);
  } else if constexpr (TYPE == WS_KV_FP16) {
    store_n<Fp16, 8, 8>((uint16_t *)base + row * dim + lane * 8, u);
  } else {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, magnitude(u[i]));
#pragma unroll
    for (int m = 1; m < G; m *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, m));
    const Coding<TYPE> c(top);
    *reinterpret_cast<u32x2 *>((uint8_t *)base + row * dim + lane * 8) = c.codes(u);
    if (lane == 0) scales[row] = c.scale;
  }
}

// Outputs from this size on are larger than the second level caches together,
// and are written past them, which took a fifth off the time of 8192 x 32 vectors
// of 128 bf16 elements (67 MB each way): 21.5 us.
constexpr int64_t kStreamBytes = (int64_t)32 << 20;

// Launches over n tokens, of which each has fewer than 2^32 threads, the most that
// one can have, in whole units of tokens.  launch(from, n) does the tokens
// from .. from + n - 1.
template <class F>
int token_ranges(int64_t n, int64_t threads_a_token, int unit, F &&launch) {
  const int64_t most = (((int64_t)1 << 32) - 256) / threads_a_token / unit * unit;
  if (most < 1) return ws_record_failure(WS_EUNSUPPORTED, "too many elements a token");
  for (int64_t from = 0; from < n; from += most) {
    launch(from, n - from < most ? n - from : most);
    if (int rc = launched()) return rc;
  }
  return WS_OK;
}

inline void skip_positions(TurnArgs &t, int64_t n) {
  if (t.positions) t.positions = (const char *)t.positions + n * (t.positions_32 ? 4 : 8);
}

// Elements of the widest aligned access of both, at most 16 bytes.
inline int widest(const ws_kv_rows &a, const ws_kv_rows &b) {
  for (int bytes = 16; bytes > type_bytes(a.type); bytes /= 2)
    if (aligned(a, bytes) && aligned(b, bytes)) return bytes / type_bytes(a.type);
  return 1;
}

}  // namespace kv

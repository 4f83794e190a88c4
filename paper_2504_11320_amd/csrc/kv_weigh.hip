// The attention that cached keys received.
//
// S_j = sum over the rows (token, head of a group) that see key j of
// 2^(scale log2(e) q . k_j - log2(e) lse): attention's weights again, from its
// log-sums, added up over the rows instead of the keys.  Matrix instructions
// compute Q K^T with the keys as columns, so that a key's weights are in one lane
// column and add up without leaving it, or as rows, each in a register.
#include <algorithm>
#include <cmath>

#include "kv_batch.h"
#include "wait_kv_budget.h"

namespace {

using namespace kv;

struct Args {
  const uint16_t *q;
  int64_t qt, qh;
  const float *lse;
  const char *k;
  const float *ks;
  float *weights;
  const int32_t *table;
  int64_t table_stride;
  int32_t capacity;  // keys that the table's columns hold
  const int32_t *starts, *lens;
  int32_t n_seq, n_tokens;
  int32_t heads, kv_heads, group;
  int32_t pages, page_shift;
  float scale;  // times log2(e)
  int32_t causal, window, accumulate;
  // what the launch is laid out for
  int32_t few_parts;     // workgroups of a request and head, of few rows
  int32_t both;          // requests of more than 16 rows are the many-rows blocks'
  int32_t tiles, parts;  // of a request's keys and of its rows, of many rows
  float *sums;           // [part][request][KV head][key]
};

constexpr float kLog2E = 1.44269504088896340736f;

// 16 bytes of codes as 16-bit floats of the queries' type, exactly: two operands.
template <int TYPE, bool BF>
__device__ __forceinline__ void codes_to_16(u32x4 x, u32x4 &lo, u32x4 &hi) {
  if constexpr (!BF) {
    const u32x2 a = codes_to_half<TYPE>(x[0]), b = codes_to_half<TYPE>(x[1]);
    const u32x2 c = codes_to_half<TYPE>(x[2]), d = codes_to_half<TYPE>(x[3]);
    lo = u32x4{a[0], a[1], b[0], b[1]};
    hi = u32x4{c[0], c[1], d[0], d[1]};
  } else {
    uint32_t y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (TYPE == WS_KV_FP8) {
        y[2 * i] = __builtin_bit_cast(
            uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], 1.0f, false));
        y[2 * i + 1] = __builtin_bit_cast(
            uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], 1.0f, true));
      } else {
        float f[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = (float)(int8_t)(x[i] >> (8 * j));
        // whole numbers up to 128: the upper halves are the bf16 values
        y[2 * i] = __builtin_amdgcn_perm(__float_as_uint(f[1]), __float_as_uint(f[0]), 0x07060302u);
        y[2 * i + 1] = __builtin_amdgcn_perm(__float_as_uint(f[3]), __float_as_uint(f[2]), 0x07060302u);
      }
    }
    lo = u32x4{y[0], y[1], y[2], y[3]};
    hi = u32x4{y[4], y[5], y[6], y[7]};
  }
}

// log2(e) times a row's log-sum; one that saw nothing counts nothing.
__device__ __forceinline__ float row_log(float lse) {
  return lse == -INFINITY ? INFINITY : lse * kLog2E;
}

// A batch's rows (token, head of the group) are numbered token * group + head.
// Rows [lo, hi) see key j.
__device__ __forceinline__ Range rows_of_key(const Args &a, const Seq &s, int32_t j, int32_t rows) {
  const int64_t old = (int64_t)s.m - s.n;  // the first token's position
  const int64_t none = 0;
  Range r = {0, rows};
  if (a.causal) r.lo = (int32_t)min((int64_t)rows, max(none, (j - old) * a.group));
  if (a.window) r.hi = (int32_t)min((int64_t)rows, max(none, (j + (int64_t)a.window - old) * a.group));
  return r;
}

// What a key's weight was, where that counts.
__device__ __forceinline__ float old_weight(const Args &a, const Seq &s, int32_t key, int32_t row) {
  const bool counts = a.accumulate && key < s.m - s.n && row != kNoRow;
  return counts ? a.weights[row] : 0.0f;
}

// ------------------------------------------------------- few rows -------
//
// Up to 16 rows of a request and KV head: the bytes of the keys bound this.  Each
// wave takes 8 KB of keys at a time, the next ones asked for as soon as the
// products have taken the last; more rows go over the same keys again.

constexpr int kFewRows = 16;

template <int TYPE, int D>
struct Few {
  static constexpr int esz = kCodes<TYPE> ? 1 : 2;
  static constexpr int steps = D / 32;         // of the product over d
  static constexpr int kloads = D * esz / 64;  // 16-byte loads of 16 keys
  static constexpr int tiles = 8 / kloads < 4 ? 8 / kloads : 4;  // of 16 keys, of a wave
  static constexpr int keys = 16 * tiles;
};

template <int TYPE, bool BF, int D>
__device__ __forceinline__ void few_rows(const Args &a, int32_t id) {
  using F = Few<TYPE, D>;
  constexpr bool CODES = kCodes<TYPE>;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n16 = lane & 15, g = lane >> 4, mine = lane & (F::keys - 1);
  const int32_t part = id % a.few_parts, pair = id / a.few_parts;
  const int32_t h = pair % a.kv_heads, b = pair / a.kv_heads;
  const Seq s = get_seq(a, b);
  const int32_t rows = s.n * a.group;
  if (a.both && rows > kFewRows) return;
  const int32_t end = min(s.m, a.capacity), step = a.few_parts * 4 * F::keys;
  int32_t k0 = (part * 4 + wave) * F::keys;
  if (k0 >= end) return;

  u32x4 q[F::steps];
  float log[4];  // of rows 4 g + r
  auto load_rows = [&](int32_t r0) {
    const int32_t row = r0 + n16;
    const bool live = row < rows;
    const int32_t token = live ? row / a.group : 0;
    const int32_t head = h * a.group + (live ? row - token * a.group : 0);
    const int64_t at = s.q0 + token;
    const uint16_t *p = a.q + at * a.qt + head * a.qh;
    const bool wide = ((a.qt | a.qh) & 7) == 0 && ((uintptr_t)a.q & 15) == 0;
#pragma unroll
    for (int i = 0; i < F::steps; ++i) {
      const int d = CODES ? 64 * (i / 2) + 16 * g + 8 * (i % 2) : 32 * i + 8 * g;
      if (!live) {
        q[i] = u32x4{0, 0, 0, 0};
      } else if (wide) {
        q[i] = *reinterpret_cast<const u32x4 *>(p + d);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          q[i][j] = (uint32_t)p[d + 2 * j] | (uint32_t)p[d + 2 * j + 1] << 16;
      }
    }
    const float l = live ? row_log(a.lse[at * a.heads + head]) : INFINITY;
#pragma unroll
    for (int r = 0; r < 4; ++r) log[r] = __shfl(l, 4 * g + r);
  };

  u32x4 kreg[F::tiles][F::kloads];
  float by = a.scale, weight = 0.0f;
  auto load_keys = [&](int32_t at_row, int32_t key) {
    if constexpr (CODES) by = a.ks[max(at_row, 0)];
    weight = old_weight(a, s, key, at_row);
#pragma unroll
    for (int t = 0; t < F::tiles; ++t) {
      const int64_t r = max(__shfl(at_row, 16 * t + n16), 0);
      const char *p = a.k + r * (D * F::esz) + 16 * g;
#pragma unroll
      for (int i = 0; i < F::kloads; ++i) kreg[t][i] = *reinterpret_cast<const u32x4 *>(p + 64 * i);
    }
  };

  int32_t page = page_entry(a, b, k0 + mine, end);
  int32_t next_page = page_entry(a, b, k0 + step + mine, end);
  if (rows > 0) load_rows(0);
  int32_t row_at = cache_row(a, page, h, k0 + mine, end);
  load_keys(row_at, k0 + mine);
  for (; k0 < end; k0 += step) {
    const bool more = end - k0 > step;
    const int32_t next_at = more ? cache_row(a, next_page, h, k0 + step + mine, end) : kNoRow;
    if (more) next_page = page_entry(a, b, min(k0 + step, end) + step + mine, end);
    const float factor = CODES ? by * a.scale : a.scale, was = weight;
    const int32_t at_row = row_at;
    row_at = next_at;
    // rows that see some of the keys, and those that see all of them
    const int32_t last = min(k0 + F::keys, end) - 1;
    const Range at_first = rows_of_key(a, s, k0, rows), at_last = rows_of_key(a, s, last, rows);
    const Range some = {at_first.lo, at_last.hi}, every = {at_last.lo, at_first.hi};
    float sum[F::tiles] = {};
    for (int32_t r0 = 0; r0 < rows; r0 += 16) {
      const bool final = r0 + 16 >= rows;
      const bool skip = r0 >= some.hi || r0 + 16 <= some.lo;
      if (skip && !final) continue;
      if (rows > 16) load_rows(r0);
      f32x4 z[F::tiles];
#pragma unroll
      for (int t = 0; t < F::tiles; ++t) {
        z[t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < F::kloads; ++i) {
          if constexpr (CODES) {
            u32x4 lo, hi;
            codes_to_16<TYPE, BF>(kreg[t][i], lo, hi);
            z[t] = mfma16<BF>(q[2 * i], lo, z[t]);
            z[t] = mfma16<BF>(q[2 * i + 1], hi, z[t]);
          } else {
            z[t] = mfma16<BF>(q[i], kreg[t][i], z[t]);
          }
        }
      }
      if (final && more) load_keys(next_at, k0 + step + mine);
      const bool all = every.lo <= r0 && every.hi >= min(r0 + 16, rows);
#pragma unroll
      for (int t = 0; t < F::tiles; ++t) {
        const float f = CODES ? __shfl(factor, 16 * t + n16) : factor;
        Range see = {0, 16};
        if (!all) {
          see = rows_of_key(a, s, k0 + 16 * t + n16, rows);
          see.lo -= r0 + 4 * g;
          see.hi -= r0 + 4 * g;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float p = exp2_of(__builtin_fmaf(z[t][r], f, -log[r]));
          sum[t] += all || (r >= see.lo && r < see.hi) ? p : 0.0f;
        }
      }
    }
    float own = 0.0f;
#pragma unroll
    for (int t = 0; t < F::tiles; ++t) {
      sum[t] += __shfl_xor(sum[t], 16);
      sum[t] += __shfl_xor(sum[t], 32);
      if (g == t) own = sum[t];
    }
    if (at_row != kNoRow && lane < F::keys) a.weights[at_row] = was + own;
    if (rows == 0 && more) load_keys(next_at, k0 + step + mine);
  }
}

// ------------------------------------------------------- many rows ------
//
// A wave keeps 64 keys (32 of D = 256) in registers as the products' left
// operands; the rows come through shared memory, three blocks of 64 in turn, one
// in use and two on their way.  With the keys as rows of the product a lane has
// one row's log-sum and 16 keys' sums of each 32, which it adds up in registers
// until the end.  Where there are few keys for many rows, the rows are split over
// workgroups too and a second kernel adds the parts in their order.

template <int TYPE, int D>
struct Many {
  static constexpr int esz = kCodes<TYPE> ? 1 : 2;
  static constexpr int ktiles = D == 256 ? 1 : 2;  // of 32 keys, of a wave
  static constexpr int keys = 128 * ktiles;        // of a workgroup
  static constexpr int rows = D == 256 ? 32 : 64;  // of a block in shared memory
  static constexpr int steps = D / 16;             // of the product over d
  static constexpr int row_bytes = D * 2;
  static constexpr int chunks = D / 8;             // of 16 bytes, of a row
  static constexpr int copies = rows * chunks / 256;  // of a thread, of a block
  static constexpr int side = rows * row_bytes;
  static constexpr int block = side + rows * 4;    // and the log-sums
  static constexpr int smem = 3 * block;
};

// 4 bytes a lane from memory to shared memory, as copy_to_lds.
__device__ __forceinline__ void copy_word_to_lds(const float *from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off"
               :
               : "v"(from), "s"(__builtin_amdgcn_readfirstlane(to))
               : "memory");
}
// Copies but the last N of this wave have arrived.
template <int N>
__device__ __forceinline__ void await_copies_but() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// All waves are here, and have read what they asked of shared memory.
__device__ __forceinline__ void meet() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Chunk c of row r lies at chunk c ^ swizzle, which spreads the 32 rows that are
// read at one chunk over the banks.
template <int D>
__device__ __forceinline__ int row_swizzle(int r) {
  return D == 64 ? (r >> 1) & 7 : r & 15;
}

// Rows [lo, hi) of a part of those that see some key of a workgroup's.
struct Parts {
  int32_t lo, hi, each, parts;
};
template <int TYPE, int D>
__device__ __forceinline__ Parts parts_of(const Args &a, const Seq &s, int32_t tile, int32_t end) {
  using M = Many<TYPE, D>;
  const int32_t k0 = tile * M::keys, rows = s.n * a.group;
  Parts p;
  p.lo = rows_of_key(a, s, k0, rows).lo / M::rows * M::rows;
  p.hi = rows_of_key(a, s, min(k0 + M::keys, end) - 1, rows).hi;
  // a tile that the launch was not laid out for has no room for parts
  const int32_t blocks = p.hi > p.lo ? (p.hi - p.lo + M::rows - 1) / M::rows : 0;
  const int32_t most = tile < a.tiles ? a.parts : 1;
  p.each = max(1, (blocks + most - 1) / most) * M::rows;
  p.parts = max(1, (blocks * M::rows + p.each - 1) / p.each);
  return p;
}

template <int TYPE, bool BF, int D>
__device__ __forceinline__ void many_rows(const Args &a, int32_t id, char *smem) {
  using M = Many<TYPE, D>;
  constexpr bool CODES = kCodes<TYPE>;
  constexpr int own = 32 * M::ktiles;  // keys of a wave
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n32 = lane & 31, hh = lane >> 5;
  // the first keys have most rows, and go first
  const int32_t pairs = a.n_seq * a.kv_heads;
  const int32_t pair = id % pairs, part = id / pairs % a.parts;
  const int32_t h = pair % a.kv_heads, b = pair / a.kv_heads;
  const Seq s = get_seq(a, b);
  const int32_t rows = s.n * a.group;
  if (rows <= kFewRows) return;
  const int32_t end = min(s.m, a.capacity);
  const uint32_t shared = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;

  for (int32_t tile = id / pairs / a.parts; tile * M::keys < end; tile += a.tiles) {
    const Parts split = parts_of<TYPE, D>(a, s, tile, end);
    if (part >= split.parts) continue;
    const int32_t lo = split.lo + part * split.each, hi = min(split.hi, lo + split.each);
    const int32_t k0 = tile * M::keys + wave * own;  // this wave's keys
    // the keys, in the layout of the product
    u32x4 k[M::ktiles][M::steps];
    float f[CODES ? M::ktiles : 1][16];
#pragma unroll
    for (int t = 0; t < M::ktiles; ++t) {
      const int32_t key = k0 + 32 * t + n32;
      const int64_t r = max(cache_row(a, page_entry(a, b, key, end), h, key, end), 0);
      const char *p = a.k + r * (D * M::esz) + 16 * hh;
      if constexpr (CODES) {
        const float scale = a.scale * a.ks[r];
#pragma unroll
        for (int i = 0; i < M::steps / 2; ++i)
          codes_to_16<TYPE, BF>(*reinterpret_cast<const u32x4 *>(p + 32 * i), k[t][2 * i],
                                k[t][2 * i + 1]);
#pragma unroll
        for (int r = 0; r < 16; ++r) f[t][r] = __shfl(scale, 8 * (r / 4) + 4 * hh + r % 4);
      } else {
#pragma unroll
        for (int i = 0; i < M::steps; ++i) k[t][i] = *reinterpret_cast<const u32x4 *>(p + 32 * i);
      }
    }
    // the key whose sum this lane has in the end
    const int32_t key = k0 + (M::ktiles == 2 ? 32 * (n32 & 1) : 0) + 8 * (n32 >> 3) + 4 * hh +
                        ((n32 >> 1) & 3);
    const int32_t row_at = cache_row(a, page_entry(a, b, key, end), h, key, end);
    const float was = old_weight(a, s, key, row_at);
    // rows that see some of the wave's keys, and those that see all of them
    const int32_t last = min(k0 + own, end) - 1;
    Range some = {0, 0}, every = {0, 0};
    if (k0 < end) {
      const Range at_first = rows_of_key(a, s, k0, rows), at_last = rows_of_key(a, s, last, rows);
      some = {at_first.lo, min(at_last.hi, hi)};
      every = {at_last.lo, min(at_first.hi, hi)};
    }

    // copies: rows of this thread's, and where they are
    const char *from[M::copies];
    int32_t head[M::copies];
    auto row_at_q = [&](int32_t row, int32_t *in) {
      const int32_t token = row / a.group;
      *in = row - token * a.group;
      return (const char *)(a.q + (int64_t)(s.q0 + token) * a.qt + (int64_t)(h * a.group + *in) * a.qh);
    };
    auto row_of_copy = [&](int i) { return (i * 256 + (int)threadIdx.x) / M::chunks; };
#pragma unroll
    for (int i = 0; i < M::copies; ++i) {
      const int r = row_of_copy(i);
      from[i] = row_at_q(min(lo + r, rows - 1), &head[i]) +
                16 * ((int)threadIdx.x % M::chunks ^ row_swizzle<D>(r));
    }
    int32_t unused;
    const char *end_row = row_at_q(rows - 1, &unused);
    // log-sums: a quarter of a block for each wave
    constexpr int quarter = M::rows / 4;
    const int32_t log_row = wave * quarter + (lane & (quarter - 1));
    int32_t log_in = (lo + log_row) % a.group;
    int64_t log_at = (int64_t)(s.q0 + (lo + log_row) / a.group) * a.heads + h * a.group + log_in;
    const int64_t log_end = (int64_t)(s.q0 + s.n) * a.heads + h * a.group + a.group - 1 - a.heads;
    const int32_t turn = M::rows / a.group, rest = M::rows - turn * a.group;
    const int64_t ahead = ((int64_t)turn * a.qt + (int64_t)rest * a.qh) * 2;
    const int64_t carry = (a.qt - (int64_t)a.group * a.qh) * 2;
    auto copy = [&](int32_t r0, int buffer) {
      const uint32_t to = shared + buffer * M::block;
      const bool cut = r0 + M::rows > rows;
#pragma unroll
      for (int i = 0; i < M::copies; ++i) {
        const int r = row_of_copy(i);
        const char *p = from[i];
        if (cut && r0 + r >= rows)
          p = end_row + 16 * ((int)threadIdx.x % M::chunks ^ row_swizzle<D>(r));
        copy_to_lds(p, to + (i * 256 + wave * 64) * 16);
        from[i] += ahead;
        if (rest) {
          head[i] += rest;
          if (head[i] >= a.group) {
            head[i] -= a.group;
            from[i] += carry;
          }
        }
      }
      if (lane < quarter)
        copy_word_to_lds(a.lse + min(log_at, log_end), to + M::side + wave * quarter * 4);
      log_at += (int64_t)turn * a.heads + rest;
      log_in += rest;
      if (log_in >= a.group) {
        log_in -= a.group;
        log_at += a.heads - a.group;
      }
    };

    float sum[M::ktiles][16];
#pragma unroll
    for (int t = 0; t < M::ktiles; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) sum[t][r] = 0.0f;

    const int32_t blocks = hi > lo ? (hi - lo + M::rows - 1) / M::rows : 0;
    meet();  // nobody reads what an earlier turn left
    for (int i = 0; i < 2 && i < blocks; ++i) copy(lo + i * M::rows, i);
    int buffer = 0;
    for (int32_t i = 0; i < blocks; ++i) {
      if (i + 1 < blocks)
        await_copies_but<M::copies + 1>();
      else
        await_copies();
      meet();
      const int32_t r0 = lo + i * M::rows;
      if (i + 2 < blocks) copy(r0 + 2 * M::rows, buffer == 0 ? 2 : buffer - 1);
      const char *q = smem + buffer * M::block;
      const float *logs = (const float *)(q + M::side);
#pragma unroll
      for (int u = 0; u < M::rows / 32; ++u) {
        const int32_t w0 = r0 + 32 * u;
        if (w0 >= some.hi || w0 + 32 <= some.lo) continue;
        const float log = row_log(logs[32 * u + n32]);
        f32x16 z[M::ktiles];
#pragma unroll
        for (int t = 0; t < M::ktiles; ++t) z[t] = f32x16{};
#pragma unroll
        for (int e = 0; e < M::steps; ++e) {
          const int c = CODES ? 4 * (e / 2) + 2 * hh + e % 2 : 2 * e + hh;
          const u32x4 x = *reinterpret_cast<const u32x4 *>(
              q + (32 * u + n32) * M::row_bytes + (c ^ row_swizzle<D>(n32)) * 16);
#pragma unroll
          for (int t = 0; t < M::ktiles; ++t) z[t] = mfma32<BF>(k[t][e], x, z[t]);
        }
        if (w0 >= every.lo && w0 + 32 <= every.hi) {
#pragma unroll
          for (int t = 0; t < M::ktiles; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              sum[t][r] += exp2_of(__builtin_fmaf(z[t][r], CODES ? f[t][r] : a.scale, -log));
        } else {
          const int32_t row = w0 + n32;
          Range see = {0, 0};
          if (row < hi) see = token_range(a, s, row / a.group);
#pragma unroll
          for (int t = 0; t < M::ktiles; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int32_t j = k0 + 32 * t + 8 * (r / 4) + 4 * hh + r % 4;
              const float p = exp2_of(__builtin_fmaf(z[t][r], CODES ? f[t][r] : a.scale, -log));
              sum[t][r] += j >= see.lo && j < see.hi ? p : 0.0f;
            }
        }
      }
      buffer = buffer == 2 ? 0 : buffer + 1;
    }
    // over the 32 rows' lanes: each step halves the keys that a lane has
    auto fold = [&](float a0, float a1, int m) {
      const bool up = lane & m;
      return (up ? a1 : a0) + __shfl_xor(up ? a0 : a1, m);
    };
    float one[M::ktiles];
#pragma unroll
    for (int t = 0; t < M::ktiles; ++t) {
#pragma unroll
      for (int r = 0; r < 8; ++r) sum[t][r] = fold(sum[t][r], sum[t][r + 8], 16);
#pragma unroll
      for (int r = 0; r < 4; ++r) sum[t][r] = fold(sum[t][r], sum[t][r + 4], 8);
#pragma unroll
      for (int r = 0; r < 2; ++r) sum[t][r] = fold(sum[t][r], sum[t][r + 2], 4);
      one[t] = fold(sum[t][0], sum[t][1], 2);
    }
    float total;
    if constexpr (M::ktiles == 2)
      total = fold(one[0], one[1], 1);
    else
      total = one[0] + __shfl_xor(one[0], 1);
    const bool mine = key < end && (M::ktiles == 2 || (lane & 1) == 0);
    if (split.parts > 1) {
      if (mine)
        a.sums[((int64_t)part * pairs + pair) * a.tiles * M::keys + key] = total;
    } else if (mine && row_at != kNoRow) {
      a.weights[row_at] = was + total;
    }
  }
}

template <int TYPE, bool BF, int D>
__global__ void __launch_bounds__(256, 2) few_kernel(Args a) {
  few_rows<TYPE, BF, D>(a, blockIdx.x);
}

template <int TYPE, bool BF, int D>
__global__ void __launch_bounds__(256, 2) many_kernel(Args a, int32_t many) {
  __shared__ alignas(16) char smem[Many<TYPE, D>::smem];
  if ((int32_t)blockIdx.x < many)
    many_rows<TYPE, BF, D>(a, blockIdx.x, smem);
  else
    few_rows<TYPE, BF, D>(a, blockIdx.x - many);
}

// The parts of a key's sum, in their order.
template <int TYPE, int D>
__global__ void __launch_bounds__(256) join_kernel(Args a) {
  using M = Many<TYPE, D>;
  constexpr int each = M::keys / 256 > 0 ? 1 : 256 / M::keys;  // tiles of a workgroup
  const int32_t groups = (a.tiles + each - 1) / each;
  const int32_t pair = blockIdx.x / groups;
  const int32_t tile = blockIdx.x % groups * each + threadIdx.x / M::keys;
  const int32_t h = pair % a.kv_heads, b = pair / a.kv_heads;
  const Seq s = get_seq(a, b);
  const int32_t end = min(s.m, a.capacity), key = tile * M::keys + threadIdx.x % M::keys;
  if (s.n * a.group <= kFewRows || tile >= a.tiles || key >= end) return;
  const Parts split = parts_of<TYPE, D>(a, s, tile, end);
  if (split.parts == 1) return;
  const int32_t row_at = cache_row(a, page_entry(a, b, key, end), h, key, end);
  if (row_at == kNoRow) return;
  const int64_t pairs = (int64_t)a.n_seq * a.kv_heads, next = pairs * a.tiles * M::keys;
  const float *p = a.sums + (int64_t)pair * a.tiles * M::keys + key;
  float sum = 0.0f;
  for (int32_t i = 0; i < split.parts; ++i) sum += p[i * next];
  a.weights[row_at] = old_weight(a, s, key, row_at) + sum;
}

// -------------------------------------------------------------- host -----

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

int check_weigh(const ws_kv_cache *c, const ws_kv_batch *b) {
  if (int rc = check_cache(c)) return rc;
  if (!b) return invalid("weigh: the batch must be non-NULL");
  if (b->n_seq < 0 || b->n_tokens < 0 || b->heads < 1) return invalid("weigh: bad sizes");
  if (b->heads % c->kv_heads) return invalid("weigh: heads must be a multiple of the cache's");
  if (b->table_cols < 0 || b->table_stride < 0) return invalid("weigh: bad page table");
  if (!(b->scale > 0.0f) || !std::isfinite(b->scale))
    return invalid("weigh: the scale must be positive and finite");
  if (b->window < 0) return invalid("weigh: the window must not be negative");
  if (b->max_q_len < 0 || b->max_kv_len < 0) return invalid("weigh: bad length bounds");
  if ((int64_t)b->n_tokens * b->heads >= (int64_t)1 << 31 ||
      (int64_t)b->n_seq * b->heads >= (int64_t)1 << 31 ||
      (int64_t)b->table_cols * c->page_size >= (int64_t)1 << 30)
    return ws_record_failure(WS_EUNSUPPORTED,
                             "weigh: 2^31 rows or requests times heads, or 2^30 keys a request");
  return WS_OK;
}

// How a batch is laid out over workgroups.
struct Layout {
  bool many;
  int32_t tiles, parts;
  int64_t bytes;
};

constexpr int many_keys(int dim) { return dim == 256 ? 128 : 256; }

Layout layout_of(const ws_kv_cache &c, const ws_kv_batch &b) {
  Layout L{};
  const int64_t group = b.heads / c.kv_heads, capacity = (int64_t)b.table_cols * c.page_size;
  const int64_t longest = std::max<int64_t>(1, std::min<int64_t>(b.max_kv_len, capacity));
  const int64_t rows = group * std::max(1, std::min(b.max_q_len, b.n_tokens));
  const int64_t pairs = (int64_t)b.n_seq * c.kv_heads;
  L.many = rows > kFewRows;
  L.tiles = (int32_t)ceil_div(longest, many_keys(c.dim));
  // four workgroups a CU, of four blocks of rows at least
  const int64_t wanted = ceil_div(1024, std::max<int64_t>(1, pairs * L.tiles));
  L.parts = (int32_t)std::max<int64_t>(1, std::min(wanted, rows / 256));
  if (L.many && L.parts > 1) L.bytes = pairs * L.tiles * many_keys(c.dim) * L.parts * 4;
  return L;
}

template <int TYPE, bool BF, int D>
int weigh_launch(Args a, const Layout &L, int64_t longest, hipStream_t stream) {
  const int64_t pairs = (int64_t)a.n_seq * a.kv_heads;
  const int64_t turns = ceil_div(longest, 4 * Few<TYPE, D>::keys);
  a.few_parts = (int32_t)std::max<int64_t>(1, std::min(turns, ceil_div(1024, pairs)));
  const int64_t few = pairs * a.few_parts, many = L.many ? pairs * L.tiles * L.parts : 0;
  if ((few + many) * 256 >= (int64_t)1 << 32 || few + many >= (int64_t)1 << 31)
    return ws_record_failure(WS_EUNSUPPORTED, "weigh: too many workgroups");
  if (!L.many) {
    few_kernel<TYPE, BF, D><<<dim3((uint32_t)few), 256, 0, stream>>>(a);
    return launched();
  }
  many_kernel<TYPE, BF, D><<<dim3((uint32_t)(few + many)), 256, 0, stream>>>(a, (int32_t)many);
  if (int rc = launched()) return rc;
  if (L.bytes) {
    const int64_t joins = pairs * ceil_div(L.tiles, D == 256 ? 2 : 1);
    join_kernel<TYPE, D><<<dim3((uint32_t)joins), 256, 0, stream>>>(a);
    return launched();
  }
  return WS_OK;
}

template <int TYPE, bool BF>
int weigh_dim(int dim, const Args &a, const Layout &L, int64_t longest, hipStream_t stream) {
  if (dim == 64) return weigh_launch<TYPE, BF, 64>(a, L, longest, stream);
  if (dim == 128) return weigh_launch<TYPE, BF, 128>(a, L, longest, stream);
  return weigh_launch<TYPE, BF, 256>(a, L, longest, stream);
}

// Whether byte ranges meet.
bool overlap(const void *a, int64_t na, const void *b, int64_t nb) {
  const char *x = (const char *)a, *y = (const char *)b;
  return na > 0 && nb > 0 && x < y + nb && y < x + na;
}

}  // namespace

extern "C" {

int wait_kv_weigh_workspace_bytes(const ws_kv_cache *cache, const ws_kv_batch *batch,
                                  size_t *bytes) {
  return guarded([&]() -> int {
    if (!bytes) return invalid("bytes must be non-NULL");
    if (int rc = check_weigh(cache, batch)) return rc;
    *bytes = batch->n_seq && batch->table_cols ? (size_t)layout_of(*cache, *batch).bytes : 0;
    return WS_OK;
  });
}

int wait_kv_weigh(const ws_kv_cache *cache, const ws_kv_batch *batch, const ws_kv_rows *q,
                  const float *lse, float *weights, int32_t accumulate, void *d_workspace,
                  size_t ws_bytes, void *hip_stream) {
  return guarded([&]() -> int {
    if (int rc = check_weigh(cache, batch)) return rc;
    const ws_kv_batch &b = *batch;
    if (int rc = check_rows(q, b.n_tokens, "weigh: q must be non-NULL")) return rc;
    if (q->type == WS_KV_FP32) return invalid("weigh: q must be bf16 or fp16");
    if (!is_8bit(cache->type) && q->type != cache->type)
      return invalid("weigh: q must have the type of a 16-bit cache");
    if ((uintptr_t)lse % 4 || (uintptr_t)weights % 4)
      return invalid("weigh: log-sums and weights must be aligned to 4 bytes");
    if (b.n_seq == 0) return WS_OK;
    if (!weights || (b.n_tokens > 0 && !lse))
      return invalid("weigh: log-sums and weights must be non-NULL");
    if (!b.starts || !b.kv_lens || (b.table_cols > 0 && !b.table))
      return invalid("weigh: the page table, starts and lengths must be non-NULL");
    if ((uintptr_t)b.starts % 4 || (uintptr_t)b.kv_lens % 4 || (uintptr_t)b.table % 4)
      return invalid("weigh: the page table, starts and lengths must be aligned to 4 bytes");
    const int64_t cells = (int64_t)cache->pages * cache->kv_heads * cache->page_size;
    if (overlap(weights, cells * 4, lse, (int64_t)b.n_tokens * b.heads * 4) ||
        overlap(weights, cells * 4, cache->k, cells * cache->dim * type_bytes(cache->type)) ||
        (cache->k_scale && overlap(weights, cells * 4, cache->k_scale, cells * 4)))
      return invalid("weigh: the weights must not overlap the log-sums or the keys");
    const int64_t capacity = (int64_t)b.table_cols * cache->page_size;
    if (capacity == 0) return WS_OK;
    Layout L = layout_of(*cache, b);
    if (L.bytes && (!d_workspace || ws_bytes < (size_t)L.bytes))
      return ws_record_failure(WS_EWORKSPACE, "weigh: the workspace is too small");
    if ((uintptr_t)d_workspace % 4) return invalid("weigh: the workspace must be aligned to 4 bytes");
    // many rows are copied 16 bytes at a time
    if (!aligned(*q, 16)) L.many = false;
    Args a{};
    a.q = (const uint16_t *)q->data;
    a.qt = q->token_stride;
    a.qh = q->head_stride;
    a.lse = lse;
    a.k = (const char *)cache->k;
    a.ks = cache->k_scale;
    a.weights = weights;
    a.table = b.table;
    a.table_stride = b.table_stride;
    a.capacity = (int32_t)capacity;
    a.starts = b.starts;
    a.lens = b.kv_lens;
    a.n_seq = b.n_seq;
    a.n_tokens = b.n_tokens;
    a.heads = b.heads;
    a.kv_heads = cache->kv_heads;
    a.group = b.heads / cache->kv_heads;
    a.pages = cache->pages;
    a.page_shift = log2_of(cache->page_size);
    a.scale = (float)((double)b.scale * 1.4426950408889634074);
    a.causal = b.causal != 0;
    a.window = b.window;
    a.accumulate = accumulate != 0;
    const int64_t longest = std::max<int64_t>(1, std::min<int64_t>(b.max_kv_len, capacity));
    a.both = L.many;
    a.tiles = L.tiles;
    a.parts = L.parts;
    a.sums = (float *)d_workspace;
    hipStream_t s = (hipStream_t)hip_stream;
    const bool bf = q->type == WS_KV_BF16;
    switch (cache->type) {
      case WS_KV_BF16: return weigh_dim<WS_KV_BF16, true>(cache->dim, a, L, longest, s);
      case WS_KV_FP16: return weigh_dim<WS_KV_FP16, false>(cache->dim, a, L, longest, s);
      case WS_KV_FP8:
        return bf ? weigh_dim<WS_KV_FP8, true>(cache->dim, a, L, longest, s)
                  : weigh_dim<WS_KV_FP8, false>(cache->dim, a, L, longest, s);
      default:
        return bf ? weigh_dim<WS_KV_INT8, true>(cache->dim, a, L, longest, s)
                  : weigh_dim<WS_KV_INT8, false>(cache->dim, a, L, longest, s);
    }
  });
}

}  // extern "C"

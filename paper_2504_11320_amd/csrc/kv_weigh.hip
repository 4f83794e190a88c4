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
  uint32_t by_group;  // 2^32 / group, rounded up: a whole quotient of small numbers
  int32_t pages, page_shift;
  float scale;  // times log2(e)
  int32_t causal, window, accumulate;
  // what the launch is laid out for
  int32_t few_parts;     // waves of a request and head, of few rows
  int32_t both;          // requests of more than 16 rows are the many-rows blocks'
  int32_t tiles;         // of a request's keys, of many rows
  int32_t part_rows;     // rows of a part; 0: they are not split
  int32_t numbers;       // of parts: of all requests
  float *sums;           // [number of a part][KV head][key]
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

// log2(e) times a row's log-sum; one that saw nothing counts nothing of a score,
// unless that is not finite, which leaves NaN.
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
// Up to 16 rows of a request and KV head: the bytes of the keys bound this.  A wave
// by itself takes 8 KB of keys at a time, the next ones asked for as soon as the
// products have taken the last; more rows go over the same keys again.  128
// requests of 513 to 1512 keys, 32 heads of 128: fp8 (591 MB) 127 us (4.7 TB/s; 111
// without writing the weights, whose 64 bytes a page and head are half lines),
// bf16 (1.1 GB) 222 us (5.0 TB/s).  All keys are read, also where a window leaves few
// of them: one token over 131,072 keys takes 30 us with a window of 257 as without.  Half the keys at a time took 162 us, two sets
// of registers for the keys 146: fewer waves then hide the memory's latency.

constexpr int kFewRows = 16;

template <int TYPE, int D>
struct Few {
  static constexpr int esz = kCodes<TYPE> ? 1 : 2;
  static constexpr int steps = D / 32;         // of the product over d
  static constexpr int kloads = D * esz / 64;  // 16-byte loads of 16 keys
  static constexpr int tiles = 8 / kloads < 4 ? 8 / kloads : 4;  // of 16 keys, of a wave
  static constexpr int keys = 16 * tiles;
};

// Launches go round the 8 dies.  Of waves that are workgroups, those of four heads in
// a row go to one die, whose cache then has the lines that the scales and weights of
// neighbouring heads share: 131 to 128 us for the decode batch above.  (Four waves of
// one workgroup have neighbouring heads as they are numbered.)
__device__ __forceinline__ int32_t near_pairs(int32_t id, int32_t pairs) {
  if (id >= pairs / 32 * 32) return id;
  return (id & ~31) | (id & 7) << 2 | (id >> 3 & 3);
}

template <int TYPE, bool BF, int D, bool ALONE>
__device__ __forceinline__ void few_rows(const Args &a, int32_t id) {  // of a wave
  using F = Few<TYPE, D>;
  constexpr bool CODES = kCodes<TYPE>;
  const int lane = threadIdx.x & 63;
  const int n16 = lane & 15, g = lane >> 4, mine = lane & (F::keys - 1);
  const int32_t pairs = a.n_seq * a.kv_heads;
  const int32_t part = id / pairs, pair = ALONE ? near_pairs(id % pairs, pairs) : id % pairs;
  if (part >= a.few_parts) return;
  const int32_t h = pair % a.kv_heads, b = pair / a.kv_heads;
  const Seq s = get_seq(a, b);
  const int32_t rows = s.n * a.group;
  if (a.both && rows > kFewRows) return;
  const int32_t end = min(s.m, a.capacity), step = a.few_parts * F::keys;
  int32_t k0 = part * F::keys;
  if (k0 >= end) return;

  u32x4 q[F::steps];
  float log[4];  // of rows 4 g + r; -infinity: one that counts nothing, or none at all
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
    const float l = live ? a.lse[at * a.heads + head] * kLog2E : -INFINITY;
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
    auto load_next = [&] {
      next_page = page_entry(a, b, min(k0 + step, end) + step + mine, end);
      load_keys(next_at, k0 + step + mine);
    };
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
      if (final && more) load_next();
      const bool all = every.lo <= r0 && every.hi >= min(r0 + 16, rows);
#pragma unroll
      for (int t = 0; t < F::tiles; ++t) {
        const float f = CODES ? __shfl(factor, 16 * t + n16) : factor;
        float p[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          // by a choice: a score that is not finite makes any sum with it NaN
          p[r] = exp2_of(__builtin_fmaf(z[t][r], f, -log[r]));
          p[r] = log[r] == -INFINITY ? 0.0f : p[r];
        }
        if (!all) {
          const Range see = rows_of_key(a, s, k0 + 16 * t + n16, rows);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int32_t row = r0 + 4 * g + r;
            p[r] = ((row >= see.lo) & (row < see.hi)) ? p[r] : 0.0f;
          }
        }
        sum[t] += (p[0] + p[1]) + (p[2] + p[3]);
      }
    }
    float own = 0.0f;
#pragma unroll
    for (int t = 0; t < F::tiles; ++t) {
      sum[t] += __shfl_xor(sum[t], 16);
      sum[t] += __shfl_xor(sum[t], 32);
      if (g == t) own = sum[t];
    }
    if (rows == 0 && more) load_next();
    // waited for here: behind the store the wait would be for that too
#pragma unroll
    for (int t = 0; t < F::tiles; ++t)
#pragma unroll
      for (int i = 0; i < F::kloads; ++i) asm volatile("" : "+v"(kreg[t][i]));
    asm volatile("" : "+v"(by), "+v"(weight), "+v"(next_page));
    if (at_row != kNoRow && lane < F::keys) a.weights[at_row] = was + own;
  }
}

// ------------------------------------------------------- many rows ------
//
// A wave keeps 64 keys (32 of D = 256) in registers as the products' right
// operands; the rows come through shared memory, three blocks of 64 (32) in turn,
// one in use and two on their way.  The products of 32 rows run beside the
// exponentials of the 32 before.  Where there are few keys for many rows, the
// rows are split over workgroups too and a second kernel adds the parts in their
// order.
//
// Two prompts of 6011 and 8192 over 32 heads of 128 bf16 (324 GFLOP): 363 to 384 us
// between cards, 0.87 PFLOP/s, 63 % of what a library product of 8192^3 reaches here.
// No unit is full: matrix units are busy 40 % of the time, vector units 56 %, and a
// quarter of the waves' cycles are waits; both units' work in one loop by itself would
// take 193 us.  Of 361 us in one run the products without the exponentials took 294,
// and all but the copies 310: neither hides wholly behind the others.  32 keys a wave and
// three workgroups a CU took 416 us, eight waves that share the copies 404.  The last
// 32 of 131,072 tokens, 64 heads on 8, int8: 110 us, four blocks of rows for each 256
// keys behind a start of several us; keeping the rows in shared memory from one tile
// of keys to the next did not change that.

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
  static constexpr int smem = 3 * side + 4 * rows * 4;  // and the log-sums of four blocks
};

constexpr int kAhead = 3;  // products whose operands are under way

// 16 bytes, or 4, a lane from memory to shared memory: as copy_to_lds, from an
// address for all lanes and an offset of each.
__device__ __forceinline__ void copy_from(const void *base, uint32_t off, uint32_t to) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :
               : "v"(off), "s"(base), "s"(__builtin_amdgcn_readfirstlane(to))
               : "memory");
}
__device__ __forceinline__ void copy_word_from(const void *base, uint32_t off, uint32_t to) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1"
               :
               : "v"(off), "s"(base), "s"(__builtin_amdgcn_readfirstlane(to))
               : "memory");
}
// Copies but the last N of this wave have arrived.
template <int N>
__device__ __forceinline__ void await_copies_but() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// All waves are here, and have read and written what they asked of shared memory.
__device__ __forceinline__ void meet() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Chunk c of row r lies at chunk c ^ swizzle, which spreads the 32 rows that are
// read at one chunk over the banks.
template <int D>
__device__ __forceinline__ int row_swizzle(int r) {
  return D == 64 ? (r >> 1) & 7 : r & 15;
}

// The number of the first part of request b: parts are numbered so that they need
// no count of those before, and no two requests share one.
__device__ __forceinline__ int32_t first_part(const Args &a, int32_t b) {
  if (!a.part_rows) return b;
  const int32_t at = min(max(a.starts[b], 0), a.n_tokens);
  return (int32_t)((uint32_t)(at * a.group) / (uint32_t)a.part_rows) + b;  // below 2^31 rows
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
  const int32_t most = tile < a.tiles && a.part_rows && rows ? (rows - 1) / a.part_rows + 1 : 1;
  p.each = max(1, (blocks + most - 1) / most) * M::rows;
  p.parts = max(1, (blocks * M::rows + p.each - 1) / p.each);
  return p;
}

template <int TYPE, bool BF, int D>
__device__ __forceinline__ void many_rows(const Args &a, int32_t id, char *smem) {
  using M = Many<TYPE, D>;
  constexpr bool CODES = kCodes<TYPE>;
  constexpr int own = 32 * M::ktiles;  // keys of a wave
  constexpr int tiles = M::rows / 32;  // of a block's rows
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n32 = lane & 31, hh = lane >> 5, mine = lane & (own - 1);
  // the first keys have most rows, and go first
  const int32_t h = id % a.kv_heads, nth = id / a.kv_heads % a.numbers;
  const int32_t b =
      a.part_rows ? last_at_most(a, [&](int32_t i) { return first_part(a, i) <= nth; }) : nth;
  if (b < 0) return;
  const int32_t part = __builtin_amdgcn_readfirstlane(nth - first_part(a, b));
  const Seq s = get_seq(a, b);
  const int32_t rows = s.n * a.group;
  if (rows <= kFewRows) return;
  const int32_t end = min(s.m, a.capacity);
  const uint32_t shared = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
  float *const logs = (float *)(smem + 3 * M::side);

  for (int32_t tile = id / a.kv_heads / a.numbers; tile * M::keys < end; tile += a.tiles) {
    const Parts split = parts_of<TYPE, D>(a, s, tile, end);
    if (part >= split.parts) continue;
    const int32_t lo = split.lo + part * split.each, hi = min(split.hi, lo + split.each);
    const int32_t blocks = hi > lo ? (hi - lo + M::rows - 1) / M::rows : 0;
    const int32_t k0 = tile * M::keys + wave * own, key = k0 + mine;  // the wave's and the lane's
    const int32_t row_at = cache_row(a, page_entry(a, b, key, end), h, key, end);

    // the keys, in the layout of the product
    u32x4 k[M::ktiles][M::steps];
    float f[M::ktiles];
#pragma unroll
    for (int t = 0; t < M::ktiles; ++t) {
      const int64_t r = max(__shfl(row_at, 32 * t + n32), 0);
      const char *p = a.k + r * (D * M::esz) + 16 * hh;
      f[t] = CODES ? a.ks[r] : 1.0f;
#pragma unroll
      for (int i = 0; i < M::steps / (CODES ? 2 : 1); ++i)
        k[t][CODES ? 2 * i : i] = *reinterpret_cast<const u32x4 *>(p + 32 * i);
    }
    float had = old_weight(a, s, key, row_at);

    // A block's copies: its first row is head g0 of token t0, and its row r lies
    // r + g0 heads behind that token's first.  Blocks go from the last rows to the
    // first: the workgroups of a head that run together then read the same ones.
    const int32_t first = lo + (blocks - 1) * M::rows, t0 = first / a.group;
    const int32_t turn = M::rows / a.group, rest = M::rows - turn * a.group;
    const char *qbase = (const char *)(a.q + (int64_t)(s.q0 + t0) * a.qt + (int64_t)h * a.group * a.qh);
    const float *lbase = a.lse + (int64_t)(s.q0 + t0) * a.heads + h * a.group;
    int32_t g0 = first - t0 * a.group, l0 = g0;
    const int32_t row_of_copy = (int)threadIdx.x / M::chunks;  // and 256 / chunks further each
    const int32_t row_of_log = wave * (M::rows / 4) + (lane & (M::rows / 4 - 1));
    auto token_of = [&](int32_t x) {
      return a.group == 1 ? x : (int32_t)__umulhi((uint32_t)x, a.by_group);
    };
    auto q_offset = [&](int32_t r, int32_t x) {
      const int32_t t = token_of(x);
      return (uint32_t)t * (uint32_t)(2 * a.qt) + (uint32_t)(x - t * a.group) * (uint32_t)(2 * a.qh) +
             16u * ((threadIdx.x % M::chunks) ^ row_swizzle<D>(r));
    };
    auto log_offset = [&](int32_t x) {
      const int32_t t = token_of(x);
      return (uint32_t)(t * a.heads + x - t * a.group) * 4u;
    };
    // Offsets change where heads do not fill blocks, and behind the last block, the
    // first one here, whose rows behind the last are that row again.
    uint32_t off[M::copies], log_off = 0;
    // the queries of the block at row r0
    auto copy_rows = [&](int32_t r0, int buffer) {
      const uint32_t to = shared + buffer * M::side;
      const bool anew = rest || r0 + M::rows >= first;
#pragma unroll
      for (int i = 0; i < M::copies; ++i) {
        const int32_t r = row_of_copy + i * (256 / M::chunks);
        if (anew) off[i] = q_offset(r, g0 + min(r, rows - 1 - r0));
        copy_from(qbase, off[i], to + (i * 256 + wave * 64) * 16);
      }
      qbase -= (int64_t)turn * a.qt * 2;
      g0 -= rest;
      if (g0 < 0) {
        g0 += a.group;
        qbase -= a.qt * 2;
      }
    };
    // and their log-sums, a quarter for each wave; of a block that is not there
    // something else, since copies are counted
    auto copy_logs = [&](int32_t r0, int slot) {
      if (rest || r0 + M::rows >= first) log_off = log_offset(l0 + min(row_of_log, rows - 1 - r0));
      if (lane < M::rows / 4)
        copy_word_from(r0 >= lo ? lbase : a.lse, r0 >= lo ? log_off : 0,
                       shared + 3 * M::side + (slot * M::rows + wave * (M::rows / 4)) * 4);
      lbase -= (int64_t)turn * a.heads;
      l0 -= rest;
      if (l0 < 0) {
        l0 += a.group;
        lbase -= a.heads;
      }
    };
    // as they are subtracted, by the wave that copied them
    auto ready_logs = [&](int slot) {
      if (lane < M::rows / 4) {
        float *p = logs + slot * M::rows + row_of_log;
        *p = -row_log(*p);
      }
    };
    meet();  // nobody reads what an earlier turn left
    if (blocks > 0) {
      copy_logs(first, 0);
      copy_rows(first, 0);
      copy_logs(first - M::rows, 1);
    }
    if (blocks > 1) {
      copy_rows(first - M::rows, 1);
      copy_logs(first - 2 * M::rows, 2);
    }
    // rows that see some of the wave's keys, and those that see all of them
    const int32_t last = min(k0 + own, end) - 1;
    Range some = {0, 0}, every = {0, 0};
    if (k0 < end) {
      const Range at_first = rows_of_key(a, s, k0, rows), at_last = rows_of_key(a, s, last, rows);
      some = {at_first.lo, min(at_last.hi, hi)};
      every = {at_last.lo, min(at_first.hi, hi)};
    }
#pragma unroll
    for (int t = 0; t < M::ktiles; ++t) {
      f[t] *= a.scale;
      if constexpr (CODES) {
#pragma unroll
        for (int i = 0; i < M::steps; i += 2) codes_to_16<TYPE, BF>(k[t][i], k[t][i], k[t][i + 1]);
      }
      // waited for here: a wait in the loop would be for the copies too
#pragma unroll
      for (int i = 0; i < M::steps; ++i) asm volatile("" : "+v"(k[t][i]));
      asm volatile("" : "+v"(f[t]));
    }
    asm volatile("" : "+v"(had));

    float sum[M::ktiles][2] = {};
    f32x16 za[M::ktiles], zb[M::ktiles];
    f32x4 logs_of[4];         // of the rows that wait for their exponentials
    int32_t waiting = 0;      // 0: none do, 1: all keys see them, 2: not all
    int32_t waiting_row = 0;  // the first of them
    // Element r of 16 is row 8 (r / 4) + 4 hh + r % 4.
    auto add = [&](const f32x16 (&z)[M::ktiles], int e) {
      const int t = e / 16, r = e % 16;
      sum[t][r & 1] += exp2_of(__builtin_fmaf(z[t][r], f[t], logs_of[r / 4][r % 4]));
    };
    auto add_seen = [&](const f32x16 (&z)[M::ktiles]) {
#pragma unroll
      for (int t = 0; t < M::ktiles; ++t) {
        Range see = rows_of_key(a, s, k0 + 32 * t + n32, rows);
        see.lo -= waiting_row + 4 * hh;
        see.hi = min(see.hi, hi) - (waiting_row + 4 * hh);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float p = exp2_of(__builtin_fmaf(z[t][r], f[t], logs_of[r / 4][r % 4]));
          const int at = 8 * (r / 4) + r % 4;
          sum[t][r & 1] += ((at >= see.lo) & (at < see.hi)) ? p : 0.0f;
        }
      }
    };
    auto read = [&](const char *q, int e) {
      const int c = CODES ? 4 * (e / 2) + 2 * hh + e % 2 : 2 * e + hh;
      return *reinterpret_cast<const u32x4 *>(q + (c ^ row_swizzle<D>(n32)) * 16);
    };
    auto product = [&](f32x16 (&z)[M::ktiles], u32x4 x, int e) {
#pragma unroll
      for (int t = 0; t < M::ktiles; ++t) z[t] = mfma32<BF>(x, k[t][e], z[t]);
    };
    // One block of 32 rows into z, beside what waits in `before`.
    auto step = [&](f32x16 (&z)[M::ktiles], const f32x16 (&before)[M::ktiles], const char *q,
                    const float *log, int32_t w0) {
      const bool none = w0 >= some.hi || w0 + 32 <= some.lo;
      if (waiting == 1 && !none) {
#pragma unroll
        for (int t = 0; t < M::ktiles; ++t) z[t] = f32x16{};
        // operands are asked for kAhead products before theirs, and each product's
        // share of the exponentials stays behind it
        u32x4 x[M::steps];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) x[e] = read(q, e);
        constexpr int per = 16 * M::ktiles / M::steps;
#pragma unroll
        for (int e = 0; e < M::steps; ++e) {
          __builtin_amdgcn_sched_barrier(0);
          if (e + kAhead < M::steps) x[e + kAhead] = read(q, e + kAhead);
          product(z, x[e], e);
#pragma unroll
          for (int i = 0; i < per; ++i) add(before, e * per + i);
        }
        __builtin_amdgcn_sched_barrier(0);
      } else {
        if (waiting == 1) {
#pragma unroll
          for (int e = 0; e < 16 * M::ktiles; ++e) add(before, e);
        } else if (waiting == 2) {
          add_seen(before);
        }
        if (!none) {
#pragma unroll
          for (int t = 0; t < M::ktiles; ++t) z[t] = f32x16{};
#pragma unroll
          for (int e = 0; e < M::steps; ++e) product(z, read(q, e), e);
        }
      }
      waiting = none ? 0 : w0 >= every.lo && w0 + 32 <= every.hi ? 1 : 2;
      waiting_row = w0;
      if (!none) {
#pragma unroll
        for (int i = 0; i < 4; ++i) logs_of[i] = *reinterpret_cast<const f32x4 *>(log + 8 * i + 4 * hh);
      }
    };

    int buffer = 0;
    for (int32_t i = 0; i < blocks; ++i) {
      // the queries of this block and the log-sums of the next are there
      if (i + 1 < blocks)
        await_copies_but<M::copies + 1>();
      else
        await_copies();
      if (i == 0) ready_logs(0);
      meet();
      const int32_t r0 = first - i * M::rows;
      if (i + 2 < blocks) {
        copy_rows(r0 - 2 * M::rows, buffer == 0 ? 2 : buffer - 1);
        copy_logs(r0 - 3 * M::rows, (i + 3) & 3);
      }
      if (i + 1 < blocks) ready_logs((i + 1) & 3);
      const char *q = smem + buffer * M::side + n32 * M::row_bytes;
      const float *log = logs + (i & 3) * M::rows;
      if constexpr (tiles == 2) {
        step(za, zb, q, log, r0);
        step(zb, za, q + 32 * M::row_bytes, log + 32, r0 + 32);
      } else if (i & 1) {
        step(zb, za, q, log, r0);
      } else {
        step(za, zb, q, log, r0);
      }
      buffer = buffer == 2 ? 0 : buffer + 1;
    }
    auto finish = [&](const f32x16 (&z)[M::ktiles]) {
      if (waiting == 1) {
#pragma unroll
        for (int e = 0; e < 16 * M::ktiles; ++e) add(z, e);
      } else if (waiting == 2) {
        add_seen(z);
      }
    };
    if (tiles == 2 || blocks % 2 == 0)
      finish(zb);
    else
      finish(za);
    // the two halves' rows
    auto join = [&](const float (&x)[M::ktiles][2]) {
      const float one = x[0][0] + x[0][1];
      if constexpr (M::ktiles == 2) {
        const float other = x[1][0] + x[1][1];
        return (hh ? other : one) + __shfl_xor(hh ? one : other, 32);
      } else {
        return one + __shfl_xor(one, 32);
      }
    };
    float total = join(sum);
    const bool has = key < end && lane < own;
    if (__any(has && row_at != kNoRow && total != total)) {
      // Again, rows that saw nothing left out by a choice, by the wave alone.  A choice
      // in the loop above took 3 to 5 % more of everything; here a key that is NaN to
      // rows that see it takes its wave up to four times as long.
      float again[M::ktiles][2] = {};
      for (int32_t r0 = max(some.lo, lo) / 32 * 32; r0 < some.hi; r0 += 32) {
        const int32_t row = min(r0 + n32, rows - 1), token = row / a.group;
        const int32_t head = h * a.group + row - token * a.group;
        const int64_t at = s.q0 + token;
        const char *q = (const char *)(a.q + at * a.qt + head * a.qh);
        const float l = -a.lse[at * a.heads + head] * kLog2E;  // +infinity: saw nothing
        f32x16 z[M::ktiles];
#pragma unroll
        for (int t = 0; t < M::ktiles; ++t) z[t] = f32x16{};
#pragma unroll
        for (int e = 0; e < M::steps; ++e) {
          const int c = CODES ? 4 * (e / 2) + 2 * hh + e % 2 : 2 * e + hh;
          product(z, *reinterpret_cast<const u32x4 *>(q + 16 * c), e);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int32_t in = 8 * (r / 4) + 4 * hh + r % 4;
          const float log = __shfl(l, in);
#pragma unroll
          for (int t = 0; t < M::ktiles; ++t) {
            const Range see = rows_of_key(a, s, k0 + 32 * t + n32, rows);
            const float p = exp2_of(__builtin_fmaf(z[t][r], f[t], log));
            const bool counts =
                (r0 + in >= see.lo) & (r0 + in < min(see.hi, hi)) & (log != INFINITY);
            again[t][r & 1] += counts ? p : 0.0f;
          }
        }
      }
      const float chosen = join(again);
      total = total != total ? chosen : total;
    }
    if (split.parts > 1) {
      const int64_t number = first_part(a, b) + part;  // again: registers are short above
      if (has) a.sums[(number * a.kv_heads + h) * a.tiles * M::keys + key] = total;
    } else if (has && row_at != kNoRow) {
      a.weights[row_at] = had + total;
    }
  }
}

template <int TYPE, bool BF, int D>
__global__ void __launch_bounds__(64, 2) few_kernel(Args a) {
  few_rows<TYPE, BF, D, true>(a, blockIdx.x);
}

template <int TYPE, bool BF, int D>
__global__ void __launch_bounds__(256, 2) many_kernel(Args a, int32_t many) {
  __shared__ alignas(16) char smem[Many<TYPE, D>::smem];
  if ((int32_t)blockIdx.x < many)
    many_rows<TYPE, BF, D>(a, blockIdx.x, smem);
  else
    few_rows<TYPE, BF, D, false>(
        a, __builtin_amdgcn_readfirstlane((blockIdx.x - many) * 4 + (threadIdx.x >> 6)));
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
  const int64_t each_part = (int64_t)a.tiles * M::keys, next = a.kv_heads * each_part;
  const float *p = a.sums + first_part(a, b) * next + h * each_part + key;
  float sum = 0.0f;
  constexpr int ahead = 16;  // parts under way
  for (int32_t i = 0; i < split.parts; i += ahead) {
    float x[ahead];
#pragma unroll
    for (int j = 0; j < ahead; ++j) x[j] = p[min(i + j, split.parts - 1) * next];
#pragma unroll
    for (int j = 0; j < ahead; ++j) sum += i + j < split.parts ? x[j] : 0.0f;
  }
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
  int32_t tiles, part_rows, numbers;
  int64_t bytes;
};

constexpr int many_keys(int dim) { return dim == 256 ? 128 : 256; }

Layout layout_of(const ws_kv_cache &c, const ws_kv_batch &b) {
  Layout L{};
  const int64_t group = b.heads / c.kv_heads, capacity = (int64_t)b.table_cols * c.page_size;
  const int64_t longest = std::max<int64_t>(1, std::min<int64_t>(b.max_kv_len, capacity));
  const int64_t rows = group * std::max(1, std::min(b.max_q_len, b.n_tokens));
  L.many = rows > kFewRows;
  L.tiles = (int32_t)ceil_div(longest, many_keys(c.dim));
  // Parts of a 1024th of the batch's blocks of rows against tiles of keys, four
  // workgroups a CU (causal, half of it is work); the rows are those that there are,
  // however many requests have few of them.  One prompt of 8192 over 16 heads on one KV
  // head: 205 us, 276 with half as many parts, 438 with a quarter.  A prompt of 512
  // behind 1024 keys beside 31 single tokens, 32 heads on 8: 34 us, 73 with as many
  // parts for each request as for the longest, most of them empty.
  // A part has four blocks at least, where joining costs what it saves: the last 32 of
  // 8192 tokens, 64 heads on 8, 17 us, 24 with two; two where there would be a
  // workgroup for half of the CUs at most: 63 tokens, 128 heads on 8, D = 64, 11.8 us,
  // 16.1 with four.  Up to 64 MB of sums.
  const int64_t block = c.dim == 256 ? 32 : 64, all_rows = (int64_t)b.n_tokens * group;
  const int64_t tiles = (int64_t)c.kv_heads * L.tiles;
  const int64_t keys = tiles * many_keys(c.dim) * 4;  // sums of a part
  const int64_t least = ceil_div(all_rows, rows) * tiles <= 128 ? 2 : 4;
  int64_t each = std::max(least, ceil_div(ceil_div(all_rows, block) * tiles, 1024));
  auto numbers = [&] { return ceil_div(all_rows, each * block) + b.n_seq; };
  while (each * block < rows && numbers() * keys > (int64_t)64 << 20) each *= 2;
  if (L.many && each * block < rows && numbers() * keys <= (int64_t)64 << 20) {
    L.part_rows = (int32_t)(each * block);
    L.numbers = (int32_t)numbers();
    L.bytes = L.numbers * keys;
  } else {
    L.numbers = b.n_seq;
  }
  return L;
}

template <int TYPE, bool BF, int D>
int weigh_launch(Args a, const Layout &L, int64_t longest, hipStream_t stream) {
  const int64_t pairs = (int64_t)a.n_seq * a.kv_heads;
  // Of few rows: 64 waves a CU, of 8 KB of keys at a time, if there are so many.
  const int64_t turns = ceil_div(longest, Few<TYPE, D>::keys);
  a.few_parts = (int32_t)std::min(turns, ceil_div(16384, pairs));
  const int64_t few = pairs * a.few_parts, many = L.many ? (int64_t)L.numbers * a.kv_heads * L.tiles : 0;
  if (few * 64 + (many + 1) * 256 >= (int64_t)1 << 32 || few + many >= (int64_t)1 << 31)
    return ws_record_failure(WS_EUNSUPPORTED, "weigh: too many workgroups");
  if (!L.many) {
    few_kernel<TYPE, BF, D><<<dim3((uint32_t)few), 64, 0, stream>>>(a);
    return launched();
  }
  many_kernel<TYPE, BF, D>
      <<<dim3((uint32_t)(many + ceil_div(few, 4))), 256, 0, stream>>>(a, (int32_t)many);
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
    const Span w = span(weights, (__int128)cache->pages * cache->kv_heads * cache->page_size * 4);
    const CacheSpans in_cache(*cache);
    auto taken = [&](const Span &x) {  // by what the call reads
      return shares(x, in_cache) ||
             shares(x, {span(*q, b.n_tokens, b.heads, cache->dim),
                      span(lse, (__int128)b.n_tokens * b.heads * 4),
                      table_span(b.table, b.n_seq, b.table_stride, b.table_cols),
                      span(b.starts, 4 * ((__int128)b.n_seq + 1)), span(b.kv_lens, 4 * (__int128)b.n_seq)});
    };
    if (taken(w)) return invalid("weigh: the weights must not overlap the cache, q or another input");
    const int64_t capacity = (int64_t)b.table_cols * cache->page_size;
    if (capacity == 0) return WS_OK;
    Layout L = layout_of(*cache, b);
    if (L.bytes && (!d_workspace || ws_bytes < (size_t)L.bytes))
      return ws_record_failure(WS_EWORKSPACE, "weigh: the workspace is too small");
    if ((uintptr_t)d_workspace % 4) return invalid("weigh: the workspace must be aligned to 4 bytes");
    const Span space = span(d_workspace, L.bytes);
    if (shares(space, w) || taken(space)) return invalid("weigh: the workspace must be its own memory");
    // many rows are copied 16 bytes at a time, a block's from one address with
    // offsets of 32 bits
    const int64_t group = b.heads / cache->kv_heads, block = 64 / group + 2;
    if (!aligned(*q, 16) || group > 4096 || q->token_stride < 0 || q->head_stride < 0 ||
        q->token_stride >= (int64_t)1 << 31 || q->head_stride >= (int64_t)1 << 31 ||
        2 * (block * q->token_stride + group * q->head_stride) >= (int64_t)1 << 32 ||
        4 * block * b.heads >= (int64_t)1 << 32)
      L.many = false;
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
    a.by_group = (uint32_t)((((int64_t)1 << 32) + a.group - 1) / a.group);
    a.pages = cache->pages;
    a.page_shift = log2_of(cache->page_size);
    a.scale = (float)((double)b.scale * 1.4426950408889634074);
    a.causal = b.causal != 0;
    a.window = b.window;
    a.accumulate = accumulate != 0;
    const int64_t longest = std::max<int64_t>(1, std::min<int64_t>(b.max_kv_len, capacity));
    a.both = L.many;
    a.tiles = L.tiles;
    a.part_rows = L.part_rows;
    a.numbers = L.numbers;
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

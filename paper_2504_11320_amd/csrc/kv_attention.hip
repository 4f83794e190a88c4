// Attention over the pages of a cache.
//
// With z_j = scale * log2(e) * q . k_j over the keys a query sees, one pass
// keeps a running reference m, l = sum_j 2^(z_j - m) and o = sum_j 2^(z_j - m) v_j,
// both multiplied by 2^(m - m') whenever m grows to m'; the result is o / l.
// Parts over different keys join the same way.  In an 8-bit cache with scales
// s_j (keys) and t_j (values), z_j has s_j as a factor, and the weight of the
// value's code is 2^(z_j - m) t_j: m runs over z_j + log2 |t_j|, which keeps these
// weights within [-1, 1], where the 16-bit floats are densest.
//
// Matrix instructions compute S^T = K Q^T and O^T = V^T P^T.  S^T leaves a
// query's scores in one lane column, four neighbouring keys in a lane, and that
// is the layout in which the next product takes P^T if its sum over keys is
// taken in the order (lane group, register); so weights never leave their lane.
// V^T comes from shared memory by transposing reads.
#include <algorithm>
#include <cmath>

#include "kv_batch.h"

namespace {

using namespace kv;

struct Args {
  const uint16_t *q;
  int64_t qt, qh;
  uint16_t *out;
  int64_t ot, oh;
  float *lse;
  const char *k, *v;
  const float *ks, *vs;
  const int32_t *table;
  int64_t table_stride;
  int32_t capacity;  // keys that the table's columns hold
  const int32_t *starts, *lens;
  int32_t n_seq, n_tokens;
  int32_t heads, kv_heads, group;
  int32_t pages, page_shift;
  float scale;  // times log2(e)
  int32_t causal, window;
  int32_t q_bf16;
  // results of parts, the sums o and (m, l): few rows [request][KV head]
  // [few_room][part] or [KV head][row of the batch][part], many rows
  // [token][head][part]
  float *few_o, *many_o;
  float2 *few_ml, *many_ml;
  int32_t few_splits, few_chunk;    // of a few-rows launch: parts, keys a part
  int32_t few_blocks;               // row blocks of a request
  int32_t few_room;                 // rows of a request that may have parts
  int32_t few_head, few_seq, few_token;  // slots from a KV head, request or token to the next
  int32_t many_splits, many_chunk;  // of a many-rows launch
  int32_t both;          // requests of more than 16 rows are the many-rows blocks'
  int32_t row_blocks;    // numbers of row blocks of the many-rows launch
};

constexpr int kFewRows = 16;  // of a few-rows block

// Of the keys k0 .. k0 + 63 that are there, those within the range, as bits.
__device__ __forceinline__ uint64_t keys_seen(Range r, int32_t k0, uint64_t there) {
  auto below = [](int32_t n) {
    return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1;
  };
  return below(r.hi - k0) & ~below(r.lo - k0) & there;
}

// Keys of the rows r0 .. r1 (inclusive): the first token's first to the last
// token's last, from a multiple of `unit` on.
__device__ __forceinline__ Range block_range(const Args &a, const Seq &s, int32_t r0, int32_t r1,
                                             int32_t unit) {
  Range first = token_range(a, s, r0 / a.group), last = token_range(a, s, r1 / a.group);
  Range r;
  r.hi = last.hi;
  r.lo = min(first.lo, r.hi) / unit * unit;
  return r;
}

__device__ __forceinline__ int32_t parts_of(Range r, int32_t chunk, int32_t splits) {
  return max(1, min(splits, (r.hi - r.lo + chunk - 1) / chunk));
}

// The parts of a few-rows block.  A request that has more rows than its launch
// was laid out for has no room for parts.
__device__ __forceinline__ int32_t few_parts(const Args &a, Range r, int32_t rows) {
  return rows > a.few_room ? 1 : parts_of(r, a.few_chunk, a.few_splits);
}

// The slot in the workspace of the first part of a few-rows row.
__device__ __forceinline__ int64_t few_slot(const Args &a, const Seq &s, int32_t b, int32_t h,
                                            int32_t row) {
  return ((int64_t)h * a.few_head + (int64_t)b * a.few_seq + (int64_t)s.q0 * a.few_token + row) *
         a.few_splits;
}

template <bool BF>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  if constexpr (BF) {
    const bf2v p = {(__bf16)x, (__bf16)y};
    return __builtin_bit_cast(uint32_t, p);
  } else {
    const half2v p = {(_Float16)x, (_Float16)y};
    return __builtin_bit_cast(uint32_t, p);
  }
}

// Four 16-bit elements down a column of four rows: within 16 lanes, lane i
// names row i / 4 and the columns 4 (i % 4) .. + 3 of a 4 x 16 tile and gets
// column i.
__device__ __forceinline__ u32x2 read_column(const char *p) {
  using lds_short4 = __attribute__((address_space(3))) short4v;
  short4v x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4 *)p);
  return __builtin_bit_cast(u32x2, x);
}

// A row of a bf16 query as halves times a power of two, 2^-e with 2^e the row's
// largest magnitude's; what this loses lies 2^-25 and more below that.
__device__ __forceinline__ int row_exponent(uint32_t top_bits) {
  return min(max((int)(top_bits >> 23) - 127, -100), 126);
}
__device__ __forceinline__ u32x4 bf16_to_half(u32x4 x, float by) {
  u32x4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    y[i] = pack2<false>(__uint_as_float(x[i] << 16) * by, __uint_as_float(x[i] & 0xffff0000u) * by);
  return y;
}
__device__ __forceinline__ uint32_t top_of(u32x4 x) {  // bf16 magnitudes, as fp32 bits
  uint32_t t = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) t = max(t, max((x[i] << 16) & 0x7fffffffu, x[i] & 0x7fff0000u));
  return t;
}

// Values that are not finite must reach the rows that see them and no others,
// and a weight of zero does not keep them out of a product.  So where some row
// of a block does not see all of a tile, they go into the product as zeros, and
// are added to the rows that see them after the loop (add_unbounded): the
// result is an infinity or a NaN whatever the weight.
template <bool BF>
__device__ __forceinline__ uint32_t unbounded_mask(uint32_t w) {
  constexpr uint32_t hi = BF ? 0x7f800000u : 0x7c000000u, lo = hi >> 16;
  return ((w & hi) == hi ? 0xffff0000u : 0u) | ((w & lo) == lo ? 0xffffu : 0u);
}
template <bool BF>
__device__ __forceinline__ bool take_unbounded(u32x4 &x) {
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t m = unbounded_mask<BF>(x[i]);
    any |= m;
    x[i] &= ~m;
  }
  return any != 0;
}
// The same of fp8 codes, of which 0x7f and 0xff are NaN.
__device__ __forceinline__ bool take_nan_codes(u32x4 &x) {
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t seven = x[i] & 0x7f7f7f7fu;
    const uint32_t top = (seven + 0x01010101u) & 0x80808080u;  // where a byte was 0x7f
    const uint32_t m = (top >> 7) * 0xffu;
    any |= m;
    x[i] &= ~m;
  }
  return any != 0;
}

// Element d of a row of values, if it is not finite; otherwise zero.
template <int TYPE, int D>
__device__ __forceinline__ float unbounded_value(const Args &a, int32_t row, int d) {
  float x;
  if constexpr (TYPE == WS_KV_BF16)
    x = Bf16::get(((const uint16_t *)a.v)[(int64_t)row * D + d]);
  else if constexpr (TYPE == WS_KV_FP16)
    x = Fp16::get(((const uint16_t *)a.v)[(int64_t)row * D + d]);
  else
    x = !isfinite(a.vs[row]) ||
                (TYPE == WS_KV_FP8 && (((const uint8_t *)a.v)[(int64_t)row * D + d] & 0x7f) == 0x7f)
            ? NAN
            : 0.0f;
  return isfinite(x) ? 0.0f : x;
}

// Below this the reference of the softmax no longer follows a value's scale, the
// weight still does: with the smallest scale of a stored row, 2^-100 / 448, it is
// 2^-13, a normal number in 16 bits.  Where all values seen have smaller scales
// (zeros), each key adds up to 2^96 to l, and 2^30 of them stay finite.
constexpr float kLeastLog = -96.0f;
// A scale that is not finite leaves the reference alone: it is the outputs that
// cannot be finite, not the log-sum.
__device__ __forceinline__ float reference_log(float scale) {
  return isfinite(scale) ? fmaxf(log2f(fabsf(scale)), kLeastLog) : kLeastLog;
}

// o / l in the output's type; a query that sees nothing has l = 0.
__device__ __forceinline__ float safe_inverse(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }
__device__ __forceinline__ uint16_t out_bits(const Args &a, float x) {
  return a.q_bf16 ? Bf16::put(x) : Fp16::put(x);
}
__device__ __forceinline__ float natural_lse(float m, float l) {
  return l == 0.0f ? -INFINITY : 0.69314718055994530942f * (m + log2f(l));
}

// ------------------------------------------------------- few rows -------
//
// Up to 16 rows (tokens x heads of a group) of a request and KV head: each
// cached element is read once for all of them, so the cache's bytes bound this.
// The waves take 32 keys each in turn, with their own running sums, and join at
// the end; long requests are split over workgroups too.  Keys go from memory
// into the matrix layout directly; values by way of shared memory, 32 rows a
// wave, for the transposing read.  128 requests of 513 to 1512 keys, 32 heads of
// 128: fp8 193 us (5.8 TB/s), bf16 367 us (5.9 TB/s), where a sum over 4 GiB
// reads 6.2 TB/s.

template <int TYPE, int D, int W>  // W waves
struct Few {
  static constexpr int esz = kCodes<TYPE> ? 1 : 2;
  static constexpr int steps = D / 32;            // of the product over d
  static constexpr int tiles = D / 16;            // of the result
  static constexpr int kloads = D * esz / 64;     // 16-byte loads of a key tile
  static constexpr int chunks = D * esz / 16;     // 16-byte chunks of a row
  static constexpr int vrows = 64 / chunks;       // rows of one value load
  static constexpr int vloads = 32 / vrows;
  static constexpr int row_bytes = D * 2;         // a row of values in shared memory
  static constexpr int wave_bytes = 32 * row_bytes + 32 * 12;
  static constexpr int join_stride = D + 4;       // floats
  static constexpr int join_bytes = W * 16 * (join_stride + 2) * 4;
  static constexpr int smem = wave_bytes * W > join_bytes ? wave_bytes * W : join_bytes;
};

// 16-byte chunk c of key row `key` lies at chunk c ^ few_swizzle(key), which
// spreads the 8 rows that 32 lanes of a transposing read touch over the banks.
template <int D>
__device__ __forceinline__ int few_swizzle(int key) {
  return D == 64 ? ((key >> 1) & 3) << 1 : (key & 7) << 1;
}

template <int TYPE, int D, int W>
__device__ __forceinline__ void few_rows(const Args &a, int32_t id, char *smem) {
  using F = Few<TYPE, D, W>;
  constexpr bool BF = kBf<TYPE>;
  constexpr bool CODES = kCodes<TYPE>;
  constexpr int stride = 32 * W;  // keys of one turn of the waves
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n16 = lane & 15, g = lane >> 4;
  // the row blocks of a request and head follow one another: they read the same
  // keys at about the same time
  const int32_t split = id % a.few_splits;
  int32_t at = id / a.few_splits;
  const int32_t first = at % a.few_blocks * kFewRows;
  at /= a.few_blocks;
  const int32_t h = at % a.kv_heads, b = at / a.kv_heads;
  const Seq s = get_seq(a, b);
  const int32_t rows = s.n * a.group;
  if (a.both && rows > kFewRows) return;

  char *vbuf = smem + wave * F::wave_bytes;
  float *kscale = (float *)(vbuf + 32 * F::row_bytes), *vlog = kscale + 32, *vscale = vlog + 32;

  for (int32_t r0 = first; r0 < rows; r0 += kFewRows * a.few_blocks) {
    const int32_t r1 = min(r0 + kFewRows, rows) - 1;
    const Range block = block_range(a, s, r0, r1, 32);
    const int32_t parts = few_parts(a, block, rows);
    if (split >= parts) continue;
    const int32_t begin = block.lo + split * a.few_chunk;
    const int32_t end = split == parts - 1 ? block.hi : begin + a.few_chunk;
    const int32_t row = r0 + n16;
    const bool live = row <= r1;
    const int32_t token = live ? row / a.group : 0;
    const int32_t head = h * a.group + (live ? row - token * a.group : 0);
    Range see = token_range(a, s, token);
    if (!live) see = {0, 0};
    // keys that every row of the block sees
    const Range lo_all = token_range(a, s, r1 / a.group), hi_all = token_range(a, s, r0 / a.group);

    // the queries, in the layout of the product
    u32x4 q[F::steps];
    float by = a.scale;
    {
      const uint16_t *p = a.q + (int64_t)(s.q0 + token) * a.qt + (int64_t)head * a.qh;
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
      if (CODES && a.q_bf16) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < F::steps; ++i) top = max(top, top_of(q[i]));
        top = max(top, (uint32_t)__shfl_xor((int)top, 16));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        const int e = row_exponent(top);
#pragma unroll
        for (int i = 0; i < F::steps; ++i) q[i] = bf16_to_half(q[i], ldexpf(1.0f, -e));
        by *= ldexpf(1.0f, e);
      }
    }

    f32x4 o[F::tiles];
#pragma unroll
    for (int i = 0; i < F::tiles; ++i) o[i] = f32x4{0, 0, 0, 0};
    float m = -INFINITY, l = 0.0f;
    bool bad = false;  // a value was taken out

    u32x4 kreg[2][F::kloads], vreg[F::vloads];
    float ks = 0.0f, vs = 0.0f;
    // scales first: they are waited for first
    auto load_keys = [&](int32_t at_row) {
      if constexpr (CODES) {
        ks = a.ks[max(at_row, 0)];
        vs = a.vs[max(at_row, 0)];
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int64_t r = max(__shfl(at_row, 16 * t + n16), 0);
        const char *p = a.k + r * (D * F::esz) + 16 * g;
#pragma unroll
        for (int i = 0; i < F::kloads; ++i)
          kreg[t][i] = *reinterpret_cast<const u32x4 *>(p + 64 * i);
      }
    };
    auto load_values = [&](int32_t at_row) {
#pragma unroll
      for (int i = 0; i < F::vloads; ++i) {
        const int64_t r = max(__shfl(at_row, i * F::vrows + lane / F::chunks), 0);
        vreg[i] = *reinterpret_cast<const u32x4 *>(a.v + r * (D * F::esz) + 16 * (lane % F::chunks));
      }
    };

    int32_t k0 = begin + 32 * wave;
    const int32_t mine = lane & 31;
    int32_t row_at = kNoRow, next_page = 0;
    if (k0 < end) {
      const int32_t page = page_entry(a, b, k0 + mine, end);
      next_page = page_entry(a, b, k0 + stride + mine, end);
      row_at = cache_row(a, page, h, k0 + mine, end);
      load_keys(row_at);
      load_values(row_at);
    }
    for (; k0 < end; k0 += stride) {
      const bool more = k0 + stride < end;
      // pages are asked for before the rows behind them, so that waiting for a
      // page is not waiting for those
      int32_t next_at = cache_row(a, next_page, h, k0 + stride + mine, end);
      next_page = page_entry(a, b, k0 + 2 * stride + mine, end);
      const uint32_t there = (uint32_t)__ballot(row_at != kNoRow);
      const bool all = k0 >= lo_all.lo && k0 + 32 <= min(hi_all.hi, end) && there == 0xffffffffu;
      if constexpr (CODES) {
        if (!all && !isfinite(vs)) {
          bad |= row_at != kNoRow;
          vs = 0.0f;
        }
        if (lane < 32) {
          kscale[lane] = ks;
          vlog[lane] = reference_log(vs);
          vscale[lane] = vs;
        }
      }
      // scores: lane (n16, g) gets keys 16 t + 4 g + r of its row
      f32x4 z[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        z[t] = f32x4{0, 0, 0, 0};
        if constexpr (CODES) {
#pragma unroll
          for (int i = 0; i < F::kloads; ++i) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const u32x2 x = codes_to_half<TYPE>(kreg[t][i][2 * half]);
              const u32x2 y = codes_to_half<TYPE>(kreg[t][i][2 * half + 1]);
              z[t] = mfma16<false>(u32x4{x[0], x[1], y[0], y[1]}, q[2 * i + half], z[t]);
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < F::kloads; ++i) z[t] = mfma16<BF>(kreg[t][i], q[i], z[t]);
        }
      }
      if (more) load_keys(next_at);
      // values to shared memory; rows that are not there as zeros, because a
      // weight of zero does not take away a NaN
      if (!all) {
#pragma unroll
        for (int i = 0; i < F::vloads; ++i) {
          if (!(there >> (i * F::vrows + lane / F::chunks) & 1)) vreg[i] = u32x4{0, 0, 0, 0};
          if constexpr (!CODES) bad |= take_unbounded<BF>(vreg[i]);
          if constexpr (TYPE == WS_KV_FP8) bad |= take_nan_codes(vreg[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < F::vloads; ++i) {
        const int key = i * F::vrows + lane / F::chunks, c = lane % F::chunks;
        const u32x4 x = vreg[i];
        char *to = vbuf + key * F::row_bytes;
        const int sw = few_swizzle<D>(key);
        if constexpr (CODES) {
          const u32x2 x0 = codes_to_half<TYPE>(x[0]), x1 = codes_to_half<TYPE>(x[1]);
          const u32x2 x2 = codes_to_half<TYPE>(x[2]), x3 = codes_to_half<TYPE>(x[3]);
          *reinterpret_cast<u32x4 *>(to + ((2 * c) ^ sw) * 16) = u32x4{x0[0], x0[1], x1[0], x1[1]};
          *reinterpret_cast<u32x4 *>(to + ((2 * c + 1) ^ sw) * 16) = u32x4{x2[0], x2[1], x3[0], x3[1]};
        } else {
          *reinterpret_cast<u32x4 *>(to + (c ^ sw) * 16) = x;
        }
      }
      if (more) load_values(next_at);
      row_at = next_at;

      float w[8], ref[8], vsc[8];
      if constexpr (CODES) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const f32x4 sk = *reinterpret_cast<const f32x4 *>(kscale + 16 * t + 4 * g);
          const f32x4 lv = *reinterpret_cast<const f32x4 *>(vlog + 16 * t + 4 * g);
          const f32x4 sv = *reinterpret_cast<const f32x4 *>(vscale + 16 * t + 4 * g);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            w[4 * t + r] = z[t][r] * (by * sk[r]);
            ref[4 * t + r] = lv[r];
            vsc[4 * t + r] = sv[r];
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = z[i / 4][i % 4] * by;
      }
      if (!all) {
        const uint32_t in = (uint32_t)keys_seen(see, k0, there) >> (4 * g);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = in & 1u << (16 * (i / 4) + i % 4) ? w[i] : -INFINITY;
      }
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, CODES ? w[i] + ref[i] : w[i]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      top = fmaxf(top, m);
      const float base = top == -INFINITY ? 0.0f : top;
      const float shrink = exp2_of(m - base);
      m = top;
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        w[i] = exp2_of(w[i] - base);
        sum += w[i];
        if constexpr (CODES) w[i] *= vsc[i];
      }
      l = l * shrink + sum;
      if (__any(shrink != 1.0f)) {
#pragma unroll
        for (int i = 0; i < F::tiles; ++i) o[i] *= shrink;
      }
      const u32x4 p = {pack2<BF>(w[0], w[1]), pack2<BF>(w[2], w[3]), pack2<BF>(w[4], w[5]),
                       pack2<BF>(w[6], w[7])};
      __builtin_amdgcn_wave_barrier();
      const int key = 4 * g + n16 / 4;
      const int sub = ((n16 & 3) >> 1) * 16 + (n16 & 1) * 8;
      const char *v0 = vbuf + key * F::row_bytes + sub;
      const char *v1 = v0 + 16 * F::row_bytes;
      const int sw = few_swizzle<D>(key);  // the same for key + 16
#pragma unroll
      for (int i = 0; i < F::tiles; ++i) {
        const int c = ((2 * i) ^ sw) * 16;
        const u32x2 x = read_column(v0 + c), y = read_column(v1 + c);
        o[i] = mfma16<BF>(u32x4{x[0], x[1], y[0], y[1]}, p, o[i]);
      }
      __builtin_amdgcn_wave_barrier();
    }
    if (__any(bad)) {
      for (k0 = begin + 32 * wave; k0 < end; k0 += stride) {
        const uint32_t there = (uint32_t)__ballot(
            cache_row(a, page_entry(a, b, k0 + mine, end), h, k0 + mine, end) != kNoRow);
        if (k0 >= lo_all.lo && k0 + 32 <= min(hi_all.hi, end) && there == 0xffffffffu) continue;
        for (int32_t j = k0; j < min(k0 + 32, end); ++j) {
          const int32_t at = cache_row(a, page_entry(a, b, j, end), h, j, end);
          if (at == kNoRow || j < see.lo || j >= see.hi) continue;
#pragma unroll
          for (int i = 0; i < F::tiles; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              o[i][r] += unbounded_value<TYPE, D>(a, at, 16 * i + 4 * g + r);
        }
      }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);

    // the waves join through shared memory
    __syncthreads();
    float *jo = (float *)smem, *jm = jo + W * 16 * F::join_stride, *jl = jm + W * 16;
#pragma unroll
    for (int i = 0; i < F::tiles; ++i)
      *reinterpret_cast<f32x4 *>(jo + (wave * 16 + n16) * F::join_stride + 16 * i + 4 * g) = o[i];
    if (g == 0) {
      jm[wave * 16 + n16] = m;
      jl[wave * 16 + n16] = l;
    }
    __syncthreads();
    constexpr int per = D / 4;  // threads of a row, four elements each
    for (int r = threadIdx.x / per; r <= r1 - r0; r += 64 * W / per) {
      const int d = threadIdx.x % per * 4;
      float mw[W], top = -INFINITY;
#pragma unroll
      for (int i = 0; i < W; ++i) top = fmaxf(top, mw[i] = jm[i * 16 + r]);
      const float base = top == -INFINITY ? 0.0f : top;
      float total = 0.0f;
      f32x4 x = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const float e = exp2_of(mw[i] - base);
        total += jl[i * 16 + r] * e;
        x += *reinterpret_cast<const f32x4 *>(jo + (i * 16 + r) * F::join_stride + d) * e;
      }
      const int32_t tok = (r0 + r) / a.group;
      const int32_t hd = h * a.group + (r0 + r) - tok * a.group;
      const int64_t q_row = s.q0 + tok;
      if (parts == 1) {
        const float inv = safe_inverse(total);
        uint16_t *p = a.out + q_row * a.ot + (int64_t)hd * a.oh + d;
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = out_bits(a, x[i] * inv);
        if (a.lse && d == 0) a.lse[q_row * a.heads + hd] = natural_lse(top, total);
      } else {
        const int64_t to = few_slot(a, s, b, h, r0 + r) + split;
        *reinterpret_cast<f32x4 *>(a.few_o + to * D + d) = x;
        if (d == 0) a.few_ml[to] = make_float2(top, total);
      }
    }
    __syncthreads();
  }
}

template <int TYPE, int D, int W>
__global__ void __launch_bounds__(64 * W, D == 256 ? 1 : 2) few_rows_kernel(Args a) {
  __shared__ alignas(16) char smem[Few<TYPE, D, W>::smem];
  few_rows<TYPE, D, W>(a, blockIdx.x, smem);
}

// ------------------------------------------------------ many rows -------
//
// 256 rows of a request and KV head in a workgroup of eight waves, 32 rows each;
// tiles of keys and of values in shared memory, two of each.  Two waves share a
// SIMD, and they take turns: while the one multiplies, the other does its
// softmax, with a barrier at each change, so that the matrix and the vector
// units both have work.  (D = 256: four waves of 32 rows, for want of
// registers.)  Prompts of 6011 and 8192 tokens, 32 heads of 128, causal: bf16 750
// us (864 TFLOP/s; 1412 in a library product of 8192^3), fp8 915 us, where the
// scales' products come on top; D = 64 485 us, of half the products.

// for the scheduler: kinds of instructions, and products whose operands are read
// ahead
constexpr int kMatrix = 0x8, kLdsRead = 0x100;
constexpr int kAhead = 3;

template <int D>
constexpr int kManyRows = D == 256 ? 128 : 256;

template <int TYPE, int D>
struct Many {
  static constexpr int esz = kCodes<TYPE> ? 1 : 2;
  static constexpr int groups = D == 256 ? 1 : 2;  // that take turns
  static constexpr int threads = 256 * groups;
  static constexpr int keys = D == 256 ? 32 : 64;  // of a tile
  static constexpr int ktiles = keys / 32;
  static constexpr int steps = D / 16;             // of the product over d
  static constexpr int tiles = D / 32;             // of the result
  static constexpr int row_bytes = D * 2;
  static constexpr int side = keys * row_bytes;    // a tile of keys, or of values
  static constexpr int chunks = D * esz / 16;      // 16-byte loads of a row
  static constexpr int loads = 2 * keys * chunks / threads;  // of a thread, keys and values
  static constexpr int scales = kCodes<TYPE> ? keys * 12 : 0;
  static constexpr int smem = 4 * side + 2 * scales;
};

// A loaded value is waited for here.  Left to its first use inside a loop, the
// wait would be for every load that is outstanding there.
template <class T>
__device__ __forceinline__ void here_by_now(T &x) {
  asm volatile("" : "+v"(x));
}

// The first row block of request b: blocks are numbered so that they need no
// count of those before, and no two requests share one.
template <int D>
__device__ __forceinline__ int32_t first_block(const Args &a, int32_t b) {
  const int32_t at = min(max(a.starts[b], 0), a.n_tokens);
  return (int32_t)((int64_t)at * a.group / kManyRows<D>) + b;
}

// Chunk c of key row `key` lies at chunk c ^ swizzle: keys are read 32 rows at
// one chunk, values 4 rows of 64 bytes at a time.
template <int D>
__device__ __forceinline__ int key_swizzle(int key) {
  return D == 64 ? (key >> 1) & 7 : key & 15;
}
template <int D>
__device__ __forceinline__ int value_swizzle(int key) {
  return D == 64 ? ((key >> 1) & 1) << 2 : (key & 3) << 2;
}

template <int TYPE, int D>
__device__ __forceinline__ void many_rows(const Args &a, int32_t id, char *smem) {
  using M = Many<TYPE, D>;
  constexpr bool BF = kBf<TYPE>;
  constexpr bool CODES = kCodes<TYPE>;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n32 = lane & 31, hh = lane >> 5;
  // the blocks of a head that run together read the same keys
  const int32_t h = id % a.kv_heads;
  const int32_t work = id / a.kv_heads;
  const int32_t split = work / a.row_blocks, nth = work % a.row_blocks;
  const int32_t b = last_at_most(a, [&](int32_t i) { return first_block<D>(a, i) <= nth; });
  if (b < 0) return;
  const Seq s = get_seq(a, b);
  const int32_t rows = s.n * a.group;
  const int32_t blocks = (rows + kManyRows<D> - 1) / kManyRows<D>;
  const int32_t back = nth - first_block<D>(a, b);
  if (rows <= kFewRows || back < 0 || back >= blocks) return;
  // the longest blocks, those of the last rows, first
  const int32_t r0 = (blocks - 1 - back) * kManyRows<D>;
  const int32_t r1 = min(r0 + kManyRows<D>, rows) - 1;
  const Range block = block_range(a, s, r0, r1, M::keys);
  const int32_t parts = parts_of(block, a.many_chunk, a.many_splits);
  if (split >= parts) return;
  const int32_t begin = block.lo + split * a.many_chunk;
  const int32_t end = split == parts - 1 ? block.hi : begin + a.many_chunk;
  const int32_t n = (end - begin + M::keys - 1) / M::keys;  // tiles
  const int32_t w0 = r0 + 32 * wave, w1 = min(w0 + 31, r1);  // this wave's rows
  const int32_t row = w0 + n32;
  const bool live = row <= r1;
  const int32_t token = live ? row / a.group : r1 / a.group;
  const int32_t head = h * a.group + (live ? row - token * a.group : 0);
  Range see = token_range(a, s, token);
  if (!live) see = {0, 0};
  // keys that some row of the wave sees, that all of them do, and all of the
  // block
  Range some = {0, 0}, every = {0, 0};
  if (w0 <= r1) {
    const Range first = token_range(a, s, w0 / a.group), last = token_range(a, s, w1 / a.group);
    some = {first.lo, last.hi};
    every = {last.lo, first.hi};
  }
  const Range block_every = {token_range(a, s, r1 / a.group).lo, token_range(a, s, r0 / a.group).hi};

  u32x4 q[M::steps];
  float by = a.scale;
  {
    const uint16_t *p = a.q + (int64_t)(s.q0 + token) * a.qt + (int64_t)head * a.qh;
    const bool wide = ((a.qt | a.qh) & 7) == 0 && ((uintptr_t)a.q & 15) == 0;
#pragma unroll
    for (int i = 0; i < M::steps; ++i) {
      const int d = 16 * i + 8 * hh;
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
    if (CODES && a.q_bf16) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < M::steps; ++i) top = max(top, top_of(q[i]));
      top = max(top, (uint32_t)__shfl_xor((int)top, 32));
      const int e = row_exponent(top);
#pragma unroll
      for (int i = 0; i < M::steps; ++i) q[i] = bf16_to_half(q[i], ldexpf(1.0f, -e));
      by *= ldexpf(1.0f, e);
    }
#pragma unroll
    for (int i = 0; i < M::steps; ++i) here_by_now(q[i]);
  }

  f32x16 o[M::tiles];
#pragma unroll
  for (int i = 0; i < M::tiles; ++i) o[i] = f32x16{};
  float m = -INFINITY, l = 0.0f;

  // Tiles on their way.  In step t the keys of tile t + 1 and the values of tile
  // t come in.  Each lane finds the row of one key of a tile; 16-bit tiles go
  // from memory to shared memory directly, codes through registers, where they
  // become halves.
  const uint32_t shared = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
  const int32_t mine = lane & (M::keys - 1);
  int32_t page = 0, key_row = 0;
  uint64_t key_there = 0, value_there = 0, there_before = 0;  // rows that are there
  u32x4 reg[CODES ? M::loads : 1];
  float ks = 0.0f, vs = 0.0f;
  bool bad = false;  // a value was taken out
  auto is_value = [&](int i) {  // whether load i is one of values
    return M::loads > 1 ? i >= M::loads / 2 : wave >= 4;
  };
  auto key_of = [&](int i) {
    return (i * M::threads + (int)threadIdx.x) / M::chunks % M::keys;
  };
  int32_t at[M::loads];  // rows of this thread's loads
  auto spread = [&](int32_t keys, int32_t values) {
#pragma unroll
    for (int i = 0; i < M::loads; ++i)
      at[i] = __builtin_amdgcn_ds_bpermute(4 * key_of(i), is_value(i) ? values : keys);
  };
  auto find = [&](int32_t t, uint64_t &there) {  // this lane's key's row, of tile t
    const int32_t found = cache_row(a, page, h, begin + t * M::keys + mine, end);
    there = __ballot(found != kNoRow);
    return max(found, 0);
  };
  auto ask = [&](int32_t t) { page = page_entry(a, b, begin + t * M::keys + mine, end); };
  // The end of step t: the rows of step t + 1, and the pages of that behind it.
  // (In step t + 1 itself, waiting for them would be waiting for its copies.)
  auto look = [&](int32_t t) {
    there_before = value_there;
    value_there = key_there;
    const int32_t values = key_row;
    key_row = find(t + 2, key_there);
    spread(key_row, values);
    ask(t + 3);
  };
  auto load = [&](int32_t t, bool keys, bool values) {
#pragma unroll
    for (int i = 0; i < M::loads; ++i) {
      if (!(is_value(i) ? values : keys)) continue;
      const char *from = (is_value(i) ? a.v : a.k) + (uint64_t)(uint32_t)at[i] * (D * M::esz);
      const int c = threadIdx.x % M::chunks;
      if constexpr (CODES) {
        reg[i] = *reinterpret_cast<const u32x4 *>(from + 16 * c);
      } else {
        // shared memory is filled in order, so the swizzle is in what is read
        const int sw = is_value(i) ? value_swizzle<D>(key_of(i)) : key_swizzle<D>(key_of(i));
        const int tile = is_value(i) ? 2 + (t & 1) : (t + 1) & 1;
        const int first = (i % (M::loads / 2) * M::threads + wave * 64) * 16;
        copy_to_lds(from + 16 * (c ^ sw), shared + tile * M::side + first);
      }
    }
    if (CODES && keys && wave == 0) {
      ks = a.ks[key_row];
      vs = a.vs[key_row];
    }
  };
  // What load(t) asked for is there, and in its place: rows that are not there
  // as zeros, because a weight of zero does not take away a NaN.
  auto arrive = [&](int32_t t, bool keys, bool values) {
    const int32_t k0 = begin + t * M::keys, k1 = k0 + M::keys;
    const bool edge = k0 < block_every.lo || k1 > block_every.hi;
    if constexpr (CODES) {
#pragma unroll
      for (int i = 0; i < M::loads; ++i) {
        const bool v = is_value(i);
        if (!(v ? values : keys)) continue;
        const int key = key_of(i), c = threadIdx.x % M::chunks;
        const int tile = v ? 2 + (t & 1) : (t + 1) & 1;
        const int sw = v ? value_swizzle<D>(key) : key_swizzle<D>(key);
        char *to = smem + tile * M::side + key * M::row_bytes;
        u32x4 x = reg[i];
        if (v && (edge || value_there != ~0ull)) {
          if (!(value_there >> key & 1)) x = u32x4{0, 0, 0, 0};
          if (TYPE == WS_KV_FP8 && edge) bad |= take_nan_codes(x);
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const u32x2 y = codes_to_half<TYPE>(x[2 * half]), z = codes_to_half<TYPE>(x[2 * half + 1]);
          *reinterpret_cast<u32x4 *>(to + ((2 * c + half) ^ sw) * 16) = u32x4{y[0], y[1], z[0], z[1]};
        }
      }
      if (keys && wave == 0 && lane < M::keys) {
        const bool next_edge = k1 < block_every.lo || k1 + M::keys > block_every.hi;
        const bool there = key_there >> lane & 1;
        if (!there | (next_edge & !isfinite(vs))) {
          bad |= there;
          vs = 0.0f;
        }
        float *sc = (float *)(smem + 4 * M::side + ((t + 1) & 1) * M::scales);
        sc[lane] = ks;
        sc[M::keys + lane] = reference_log(vs);
        sc[2 * M::keys + lane] = vs;
      }
    } else {
      await_copies();
      if (values && (edge || value_there != ~0ull)) {
#pragma unroll
        for (int i = 0; i < M::loads / 2; ++i) {
          u32x4 *at = (u32x4 *)(smem + (2 + (t & 1)) * M::side + (i * M::threads + threadIdx.x) * 16);
          u32x4 x = *at;
          if (!(value_there >> key_of(i) & 1)) x = u32x4{0, 0, 0, 0};
          if (edge) bad |= take_unbounded<BF>(x);
          *at = x;
        }
      }
    }
  };
  // Scores of tile t: lane (n32, hh), register r of z[k]: key 32 k + 8 (r / 4) +
  // 4 hh + r % 4.  Their weights p[c]: keys 16 c + 4 hh + (0..3) and + 8.
  f32x16 z[M::ktiles];
  u32x4 p[2 * M::ktiles];
  // Product number e of the values of tile t, and of the scores: each has as many
  // as the other.
  constexpr int products = 2 * M::ktiles * M::tiles;
  static_assert(products == M::ktiles * M::steps, "");
  auto value_product = [&](int32_t t, int e) {
    const int c = e / M::tiles, i = e % M::tiles;
    const int i16 = lane & 15, q2 = (lane >> 4) & 1;
    const int key = 4 * hh + i16 / 4;
    const int sw = value_swizzle<D>(key);  // the same for key + 8, + 16, ...
    const char *at = smem + (2 + (t & 1)) * M::side + key * M::row_bytes + (i16 & 1) * 8 +
                     ((4 * i + 2 * q2 + ((i16 & 3) >> 1)) ^ sw) * 16 + 16 * c * M::row_bytes;
    const u32x2 x = read_column(at), y = read_column(at + 8 * M::row_bytes);
    o[i] = mfma32<BF>(u32x4{x[0], x[1], y[0], y[1]}, p[c], o[i]);
  };
  auto score_product = [&](int32_t t, int e) {
    const int i = e / M::ktiles, k = e % M::ktiles;
    const int sw = key_swizzle<D>(n32);  // the same for key + 32
    const u32x4 x = *reinterpret_cast<const u32x4 *>(
        smem + (t & 1) * M::side + (n32 + 32 * k) * M::row_bytes + ((2 * i + hh) ^ sw) * 16);
    if (i == 0) z[k] = f32x16{};
    z[k] = mfma32<BF>(x, q[i], z[k]);
  };
  auto add_values = [&](int32_t t) {
#pragma unroll
    for (int e = 0; e < products; ++e) value_product(t, e);
  };
  auto score = [&](int32_t t) {
#pragma unroll
    for (int e = 0; e < products; ++e) score_product(t, e);
  };
  // Both, in turn, so that a product does not wait for the one before it.  They
  // run 32 cycles each, a read from shared memory takes a few times that: the
  // reads of kAhead pairs are under way before the first.
  auto multiply = [&](int32_t t) {
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int e = 0; e < products; ++e) {
      value_product(t - 1, e);
      score_product(t, e);
    }
    __builtin_amdgcn_sched_group_barrier(kLdsRead, 3 * kAhead, 0);
#pragma unroll
    for (int e = 0; e < products - kAhead; ++e) {
      __builtin_amdgcn_sched_group_barrier(kMatrix, 2, 0);
      __builtin_amdgcn_sched_group_barrier(kLdsRead, 3, 0);
    }
    __builtin_amdgcn_sched_group_barrier(kMatrix, 2 * kAhead, 0);
    __builtin_amdgcn_s_setprio(0);
  };
  auto weigh = [&](int32_t t, uint64_t there) {
    const int32_t k0 = begin + t * M::keys;
    if (k0 >= some.hi || k0 + M::keys <= some.lo) {  // none that this wave sees
#pragma unroll
      for (int c = 0; c < 2 * M::ktiles; ++c) p[c] = u32x4{0, 0, 0, 0};
      return;
    }
    const bool full = k0 >= every.lo && k0 + M::keys <= min(every.hi, end) && there == ~0ull;
    const float *sc = (const float *)(smem + 4 * M::side + (t & 1) * M::scales);
    auto scales = [&](int which, int k, int r4) {
      return *reinterpret_cast<const f32x4 *>(sc + which * M::keys + 32 * k + 8 * r4 + 4 * hh);
    };
    if constexpr (CODES) {
#pragma unroll
      for (int k = 0; k < M::ktiles; ++k)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const f32x4 sk = scales(0, k, r / 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) z[k][r + e] *= sk[e];
        }
    }
    if (!full) {
      const uint64_t in = keys_seen(see, k0, there) >> (4 * hh);
      const uint32_t half[2] = {(uint32_t)in, (uint32_t)(in >> 32)};
#pragma unroll
      for (int k = 0; k < M::ktiles; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          z[k][r] = half[k] & 1u << (8 * (r / 4) + r % 4) ? z[k][r] : -INFINITY;
    }
    // the largest score, times log2(e) and the scale; of codes, plus log2 of the
    // value's scale
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < M::ktiles; ++k)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        f32x4 x = {z[k][r], z[k][r + 1], z[k][r + 2], z[k][r + 3]};
        if constexpr (CODES) {
          const f32x4 lv = scales(1, k, r / 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = __builtin_fmaf(x[e], by, lv[e]);
        }
        top = fmaxf(fmaxf(top, x[0]), x[1]);
        top = fmaxf(fmaxf(top, x[2]), x[3]);
      }
    top = fmaxf(top, __shfl_xor(top, 32));
    top = fmaxf(CODES ? top : top * by, m);
    const float base = top == -INFINITY ? 0.0f : top;
    const float shrink = exp2_of(m - base);
    m = top;
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < 2 * M::ktiles; ++c) {
#pragma unroll
      for (int r4 = 0; r4 < 2; ++r4) {
        f32x4 w;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          w[r] = exp2_of(__builtin_fmaf(z[c / 2][8 * (c % 2) + 4 * r4 + r], by, -base));
          sum[r4] += w[r];
        }
        if constexpr (CODES) w *= scales(2, c / 2, 2 * (c % 2) + r4);
        p[c][2 * r4] = pack2<BF>(w[0], w[1]);
        p[c][2 * r4 + 1] = pack2<BF>(w[2], w[3]);
      }
    }
    l = l * shrink + (sum[0] + sum[1]);
    if (__any(shrink != 1.0f)) {
#pragma unroll
      for (int i = 0; i < M::tiles; ++i) o[i] *= shrink;
    }
  };

  auto turn = [] {
    if constexpr (M::groups > 1) __syncthreads();
  };

  if (n > 0) {
    ask(0);
    const int32_t first = find(0, key_there);
    key_row = first;
    ask(1);
    spread(first, first);
    load(-1, true, false);
    arrive(-1, true, false);
    value_there = key_there;
    key_row = find(1, key_there);
    spread(key_row, first);
    ask(2);
    __syncthreads();
    // step t: the first waves multiply for tile t and weigh it, the others weigh
    // tile t - 1 and multiply for t
    load(0, n > 1, true);
    if (M::groups == 1 || wave < 4) {
      score(0);
      turn();
      weigh(0, value_there);
      arrive(0, n > 1, true);
      look(0);
      __syncthreads();
      for (int32_t t = 1; t < n; ++t) {
        load(t, t + 1 < n, true);
        multiply(t);
        turn();
        weigh(t, value_there);
        arrive(t, t + 1 < n, true);
        look(t);
        __syncthreads();
      }
    } else {
      turn();
      score(0);
      arrive(0, n > 1, true);
      look(0);
      __syncthreads();
      for (int32_t t = 1; t < n; ++t) {
        load(t, t + 1 < n, true);
        weigh(t - 1, there_before);
        turn();
        multiply(t);
        arrive(t, t + 1 < n, true);
        look(t);
        __syncthreads();
      }
      weigh(n - 1, there_before);
    }
    add_values(n - 1);
  }
  if (__syncthreads_or(bad)) {
    for (int32_t k0 = begin; k0 < end; k0 += M::keys) {
      if (k0 >= block_every.lo && k0 + M::keys <= block_every.hi) continue;
      for (int32_t j = k0; j < min(k0 + M::keys, end); ++j) {
        const int32_t found = cache_row(a, page_entry(a, b, j, end), h, j, end);
        if (found == kNoRow || j < see.lo || j >= see.hi) continue;
#pragma unroll
        for (int i = 0; i < M::tiles; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            o[i][r] += unbounded_value<TYPE, D>(a, found, 32 * i + 8 * (r / 4) + 4 * hh + r % 4);
      }
    }
  }
  l += __shfl_xor(l, 32);

  // register r of o[i]: d = 32 i + 8 (r / 4) + 4 hh + r % 4 of row n32
  if (!live) return;
  const int64_t q_row = s.q0 + token;
  if (parts == 1) {
    const float inv = safe_inverse(l);
    uint16_t *to = a.out + q_row * a.ot + (int64_t)head * a.oh;
    const bool wide = ((a.ot | a.oh) & 3) == 0 && ((uintptr_t)a.out & 7) == 0;
#pragma unroll
    for (int i = 0; i < M::tiles; ++i) {
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const int d = 32 * i + 8 * r4 + 4 * hh;
        uint16_t x[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = out_bits(a, o[i][4 * r4 + r] * inv);
        if (wide) {
          *reinterpret_cast<u32x2 *>(to + d) =
              u32x2{(uint32_t)x[0] | (uint32_t)x[1] << 16, (uint32_t)x[2] | (uint32_t)x[3] << 16};
        } else {
#pragma unroll
          for (int r = 0; r < 4; ++r) to[d + r] = x[r];
        }
      }
    }
    if (a.lse && hh == 0) a.lse[q_row * a.heads + head] = natural_lse(m, l);
  } else {
    const int64_t to = (q_row * a.heads + head) * a.many_splits + split;
#pragma unroll
    for (int i = 0; i < M::tiles; ++i)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4)
        *reinterpret_cast<f32x4 *>(a.many_o + to * D + 32 * i + 8 * r4 + 4 * hh) =
            f32x4{o[i][4 * r4], o[i][4 * r4 + 1], o[i][4 * r4 + 2], o[i][4 * r4 + 3]};
    if (hh == 0) a.many_ml[to] = make_float2(m, l);
  }
}

// A batch of both kinds in one launch: the long workgroups first, the others
// where these leave room.
template <int D>
constexpr int kWideWaves = D == 256 ? 4 : 8;

template <int TYPE, int D>
__global__ void __launch_bounds__(64 * kWideWaves<D>, D == 256 ? 1 : 2) rows_kernel(Args a, int32_t many) {
  constexpr int few_smem = Few<TYPE, D, kWideWaves<D>>::smem, many_smem = Many<TYPE, D>::smem;
  __shared__ alignas(16) char smem[few_smem > many_smem ? few_smem : many_smem];
  if ((int32_t)blockIdx.x < many)
    many_rows<TYPE, D>(a, blockIdx.x, smem);
  else
    few_rows<TYPE, D, kWideWaves<D>>(a, blockIdx.x - many, smem);
}

// ----------------------------------------------------------- joining ----
//
// D / 4 lanes join parts of a (token, head), four elements each.

template <int D>
constexpr int kJoinLanes = D / 4;

struct Joined {
  f32x4 o;
  float m, l;
};

__device__ __forceinline__ void join(Joined &j, f32x4 o, float m, float l) {
  const float top = fmaxf(j.m, m), base = top == -INFINITY ? 0.0f : top;
  const float ej = exp2_of(j.m - base), e = exp2_of(m - base);
  j.m = top;
  j.l = j.l * ej + l * e;
  j.o = j.o * ej + o * e;
}

// The parts first, first + step, ...: four at a time are under way.
template <int D>
__device__ __forceinline__ Joined join_parts(const float *part_o, const float2 *part_ml,
                                             int32_t first, int32_t step, int32_t parts) {
  constexpr int ahead = 4;
  const int lane = threadIdx.x % kJoinLanes<D>;
  Joined j = {f32x4{0, 0, 0, 0}, -INFINITY, 0.0f};
  for (int32_t k = first; k < parts; k += ahead * step) {
    f32x4 o[ahead];
    float2 ml[ahead];
#pragma unroll
    for (int i = 0; i < ahead; ++i) {
      const int64_t at = min(k + i * step, parts - 1);
      ml[i] = part_ml[at];
      o[i] = *reinterpret_cast<const f32x4 *>(part_o + at * D + 4 * lane);
    }
#pragma unroll
    for (int i = 0; i < ahead; ++i)
      if (k + i * step < parts) join(j, o[i], ml[i].x, ml[i].y);
  }
  return j;
}

template <int D>
__device__ __forceinline__ void put_joined(const Args &a, const Joined &j, int64_t q_row,
                                           int32_t head) {
  const int lane = threadIdx.x % kJoinLanes<D>;
  const float inv = safe_inverse(j.l);
  uint16_t *p = a.out + q_row * a.ot + (int64_t)head * a.oh + 4 * lane;
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = out_bits(a, j.o[i] * inv);
  if (a.lse && lane == 0) a.lse[q_row * a.heads + head] = natural_lse(j.m, j.l);
}

// Few rows have many parts: a workgroup shares a (request, head), of which it
// takes the tokens `nth`, `nth` + `step`, ...
template <int D>
__device__ __forceinline__ void join_few(const Args &a, int32_t id, int32_t nth, int32_t step) {
  constexpr int lanes = kJoinLanes<D>, groups = 256 / lanes;
  __shared__ Joined shared[groups][lanes];
  const int lane = threadIdx.x % lanes, mine = threadIdx.x / lanes;
  const int32_t head = id % a.heads, b = id / a.heads;
  const Seq s = get_seq(a, b);
  const int32_t rows = s.n * a.group;
  if (rows == 0 || rows > a.few_room) return;
  for (int32_t i = nth; i < s.n; i += step) {
    const int32_t row = i * a.group + head % a.group, r0 = row / kFewRows * kFewRows;
    const int32_t parts =
        few_parts(a, block_range(a, s, r0, min(r0 + kFewRows, rows) - 1, 32), rows);
    if (parts == 1) continue;
    const int64_t at = few_slot(a, s, b, head / a.group, row);
    shared[mine][lane] = join_parts<D>(a.few_o + at * D, a.few_ml + at, mine, groups, parts);
    __syncthreads();
    if (mine == 0) {
      Joined j = shared[0][lane];
#pragma unroll
      for (int g = 1; g < groups; ++g) {
        const Joined x = shared[g][lane];
        join(j, x.o, x.m, x.l);
      }
      put_joined<D>(a, j, s.q0 + i, head);
    }
    __syncthreads();
  }
}

// Many rows have few parts: a wave to 64 / kJoinLanes heads of a token.
template <int D>
__device__ __forceinline__ void join_many(const Args &a, int32_t id, int32_t keys) {
  constexpr int several = 64 / kJoinLanes<D>;
  const int32_t head_groups = (a.heads + several - 1) / several;
  const int32_t token = id / head_groups;
  if (token >= a.n_tokens) return;
  const int32_t head = id % head_groups * several + (threadIdx.x & 63) / kJoinLanes<D>;
  const int32_t b = last_at_most(a, [&](int32_t i) { return a.starts[i] <= token; });
  if (b < 0 || head >= a.heads) return;
  const Seq s = get_seq(a, b);
  const int32_t rows = s.n * a.group, i = token - s.q0;
  if (i < 0 || i >= s.n || rows <= kFewRows) return;
  const int32_t r0 = (i * a.group + head % a.group) / kManyRows<D> * kManyRows<D>;
  const int32_t parts = parts_of(block_range(a, s, r0, min(r0 + kManyRows<D>, rows) - 1, keys),
                                 a.many_chunk, a.many_splits);
  if (parts == 1) return;
  const int64_t at = ((int64_t)token * a.heads + head) * a.many_splits;
  put_joined<D>(a, join_parts<D>(a.many_o + at * D, a.many_ml + at, 0, 1, parts), token, head);
}

// Both in one launch: 64 heads with 32 parts each 4.9 us; 543 x 32 rows, most of
// them with 3, 7.4 us (12 with a wave a row, whose waves come in two turns).
template <int D>
__global__ void __launch_bounds__(256) join_kernel(Args a, int32_t few, int32_t step, int32_t keys) {
  if ((int32_t)blockIdx.x < few)
    join_few<D>(a, blockIdx.x / step, blockIdx.x % step, step);
  else
    join_many<D>(a, ((int32_t)blockIdx.x - few) * 4 + (threadIdx.x >> 6), keys);
}

// -------------------------------------------------------------- host -----

// How a batch is laid out over workgroups.
struct Layout {
  bool many, wide;
  int32_t few_splits, few_chunk, few_blocks, few_room, few_head, few_seq, few_token, many_splits, many_chunk, row_blocks;
  int64_t few_slots, many_slots;  // results of parts in the workspace
  int64_t bytes;
};

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Parts of at least `least` and at most `most` keys, multiples of `unit`, as
// many as give `wanted` workgroups.
void split_keys(int64_t keys, int64_t groups, int64_t wanted, int64_t least, int64_t most,
                int32_t unit, int32_t *splits, int32_t *chunk) {
  int64_t n = ceil_div(wanted, groups);
  int64_t c = ceil_div(keys, n);
  c = c < least ? least : c > most ? most : c;
  c = ceil_div(c, unit) * unit;
  *chunk = (int32_t)c;
  *splits = (int32_t)(keys > c ? ceil_div(keys, c) : 1);
}

Layout layout_of(const ws_kv_cache &c, const ws_kv_batch &b) {
  Layout L{};
  const int32_t group = b.heads / c.kv_heads;
  int64_t max_q = b.max_q_len < 1 ? 1 : b.max_q_len;
  int64_t max_kv = b.max_kv_len < 1 ? 1 : b.max_kv_len;
  max_q = max_q > b.n_tokens ? b.n_tokens : max_q;
  const int64_t capacity = (int64_t)b.table_cols * c.page_size;
  max_kv = max_kv > capacity ? capacity : max_kv;
  if (max_kv < 1) max_kv = 1;
  const int64_t pairs = (int64_t)b.n_seq * c.kv_heads;
  const int64_t max_rows = max_q * group;
  // Blocks of 16 rows read the keys again, out of a cache where they run at the
  // same time; up to four of them are quicker than one block of 256 rows over
  // many keys: 16 requests of 10 to 16 tokens, 4 heads a KV head, over 1000 to
  // 2000 keys in fp8 37 us against 62, of 5 to 8 tokens 24 against 57.  Over few
  // keys they are not: 32 prompts of 30 to 60 tokens 45 us against 32.
  L.many = max_rows > 4 * kFewRows || (max_rows > kFewRows && max_kv < 16 * max_rows);
  L.few_blocks = L.many ? 1 : (int32_t)ceil_div(max_rows, kFewRows);
  L.few_room = L.many ? kFewRows : (int32_t)max_rows;
  const int64_t many_rows = c.dim == 256 ? kManyRows<256> : kManyRows<128>;
  int64_t few_keys = max_kv, many_keys = max_kv;
  if (b.window) {
    few_keys = std::min<int64_t>(max_kv, (int64_t)b.window + kFewRows + 32);
    many_keys = std::min<int64_t>(max_kv, (int64_t)b.window + many_rows + 64);
  }
  // Few rows: with a workgroup of four waves and 512 of them at once the card is
  // full; below that eight waves share a pair, one workgroup a CU.
  const int64_t few_groups = pairs * L.few_blocks;
  L.wide = L.many || few_groups < 512;
  split_keys(few_keys, few_groups, L.wide ? 256 : 512, L.wide ? 1024 : 512, 4096, 256, &L.few_splits,
             &L.few_chunk);
  L.row_blocks = (int32_t)((int64_t)b.n_tokens * group / many_rows + b.n_seq);
  // workgroups that have rows: as many as the tokens fill
  const int64_t full = ceil_div((int64_t)b.n_tokens * group, many_rows) * c.kv_heads;
  // Joining costs by the rows, so many of them take longer parts: a prompt of 512
  // over 32 heads 26 us with parts of 512 keys and 28 with 256; a prompt of 1024
  // over 4 heads 29 us with 512 and 24 with 256.  D = 256 has tiles of 32 keys.
  const int64_t least = (full >= 64 ? 512 : 256) / (c.dim == 256 ? 2 : 1);
  split_keys(many_keys, full, 256, least, (int64_t)1 << 30, 64, &L.many_splits, &L.many_chunk);
  // room for the rows that the bounds allow, or for those that there are
  const int64_t bound = pairs * L.few_room, rows = (int64_t)b.n_tokens * b.heads;
  L.few_head = (int32_t)(rows < bound ? rows / c.kv_heads : L.few_room);
  L.few_seq = (int32_t)(rows < bound ? 0 : (int64_t)c.kv_heads * L.few_room);
  L.few_token = rows < bound ? group : 0;
  if (L.few_splits > 1) L.few_slots = std::min(rows, bound) * L.few_splits;
  if (L.many && L.many_splits > 1)
    L.many_slots = (int64_t)b.n_tokens * b.heads * L.many_splits;
  L.bytes = (L.few_slots + L.many_slots) * (c.dim + 2) * 4;
  return L;
}

int check_batch(const ws_kv_cache *c, const ws_kv_batch *b) {
  if (int rc = check_cache(c)) return rc;
  if (!b) return invalid("attention: the batch must be non-NULL");
  if (b->n_seq < 0 || b->n_tokens < 0 || b->heads < 1) return invalid("attention: bad sizes");
  if (b->heads % c->kv_heads) return invalid("attention: heads must be a multiple of the cache's");
  if (b->table_cols < 0 || b->table_stride < 0) return invalid("attention: bad page table");
  if (!(b->scale > 0.0f) || !std::isfinite(b->scale))
    return invalid("attention: the scale must be positive and finite");
  if (b->window < 0) return invalid("attention: the window must not be negative");
  if (b->max_q_len < 0 || b->max_kv_len < 0) return invalid("attention: bad length bounds");
  if ((int64_t)b->n_tokens * b->heads >= (int64_t)1 << 31 ||
      (int64_t)b->n_seq * b->heads >= (int64_t)1 << 31 ||
      (int64_t)b->table_cols * c->page_size >= (int64_t)1 << 30)
    return ws_record_failure(WS_EUNSUPPORTED,
                             "attention: 2^31 rows or requests times heads, or 2^30 keys a request");
  return WS_OK;
}

template <int TYPE, int D>
int attention_launch(const Args &a, const Layout &L, hipStream_t stream) {
  const int64_t pairs = (int64_t)a.n_seq * a.kv_heads;
  const int64_t few = pairs * L.few_splits * L.few_blocks;
  const int64_t many = L.many ? (int64_t)a.kv_heads * L.many_splits * L.row_blocks : 0;
  constexpr int wide = kWideWaves<D>;
  // a request whose few rows have parts has at most so many tokens
  const int32_t step = std::max(1, L.few_room / a.group);
  const int64_t join_few = L.few_slots ? (int64_t)a.n_seq * a.heads * step : 0;
  constexpr int several = 64 / kJoinLanes<D>;
  const int64_t waves = (int64_t)a.n_tokens * ceil_div(a.heads, several);
  const int64_t join = L.bytes ? join_few + (L.many_slots ? ceil_div(waves, 4) : 0) : 0;
  // a launch has fewer than 2^32 threads
  if ((few + many) * 64 * (L.wide ? wide : 4) >= (int64_t)1 << 32 || join * 256 >= (int64_t)1 << 32)
    return ws_record_failure(WS_EUNSUPPORTED, "attention: too many workgroups");
  if (L.many) {
    rows_kernel<TYPE, D><<<dim3((uint32_t)(few + many)), 64 * wide, 0, stream>>>(a, (int32_t)many);
  } else if (L.wide) {
    few_rows_kernel<TYPE, D, wide><<<dim3((uint32_t)few), 64 * wide, 0, stream>>>(a);
  } else {
    few_rows_kernel<TYPE, D, 4><<<dim3((uint32_t)few), 256, 0, stream>>>(a);
  }
  if (int rc = launched()) return rc;
  if (join) {
    join_kernel<D><<<dim3((uint32_t)join), 256, 0, stream>>>(a, (int32_t)join_few, step,
                                                             Many<TYPE, D>::keys);
    return launched();
  }
  return WS_OK;
}

template <int TYPE>
int attention_dim(int dim, const Args &a, const Layout &L, hipStream_t stream) {
  if (dim == 64) return attention_launch<TYPE, 64>(a, L, stream);
  if (dim == 128) return attention_launch<TYPE, 128>(a, L, stream);
  return attention_launch<TYPE, 256>(a, L, stream);
}

}  // namespace

extern "C" {

int wait_kv_attention_workspace_bytes(const ws_kv_cache *cache, const ws_kv_batch *batch,
                                      size_t *bytes) {
  return guarded([&]() -> int {
    if (!bytes) return invalid("bytes must be non-NULL");
    if (int rc = check_batch(cache, batch)) return rc;
    *bytes = batch->n_seq && batch->n_tokens ? (size_t)layout_of(*cache, *batch).bytes : 0;
    return WS_OK;
  });
}

int wait_kv_attention(const ws_kv_cache *cache, const ws_kv_batch *batch, const ws_kv_rows *q,
                      const ws_kv_rows *out, float *lse, void *d_workspace, size_t ws_bytes,
                      void *hip_stream) {
  return guarded([&]() -> int {
    if (int rc = check_batch(cache, batch)) return rc;
    const ws_kv_batch &b = *batch;
    if (int rc = check_rows(q, b.n_tokens, "attention: q must be non-NULL")) return rc;
    if (int rc = check_rows(out, b.n_tokens, "attention: out must be non-NULL")) return rc;
    if (q->type == WS_KV_FP32 || q->type != out->type)
      return invalid("attention: q and out must both be bf16 or both fp16");
    if (!is_8bit(cache->type) && q->type != cache->type)
      return invalid("attention: q must have the type of a 16-bit cache");
    if (!one_place(*q, *out) && overlap(*q, *out, b.n_tokens, b.heads, cache->dim))
      return invalid("attention: out must be q or not overlap it");
    if ((uintptr_t)lse % 4) return invalid("attention: lse must be aligned to 4 bytes");
    if (b.n_seq == 0 || b.n_tokens == 0) return WS_OK;
    if (!b.starts || !b.kv_lens || (b.table_cols > 0 && !b.table))
      return invalid("attention: the page table, starts and lengths must be non-NULL");
    if ((uintptr_t)b.starts % 4 || (uintptr_t)b.kv_lens % 4 || (uintptr_t)b.table % 4)
      return invalid("attention: the page table, starts and lengths must be aligned to 4 bytes");
    const Layout L = layout_of(*cache, b);
    if (L.bytes && (!d_workspace || ws_bytes < (size_t)L.bytes))
      return ws_record_failure(WS_EWORKSPACE, "attention: the workspace is too small");
    if ((uintptr_t)d_workspace % 16) return invalid("attention: the workspace must be 16-byte aligned");
    Args a{};
    a.q = (const uint16_t *)q->data;
    a.qt = q->token_stride;
    a.qh = q->head_stride;
    a.out = (uint16_t *)out->data;
    a.ot = out->token_stride;
    a.oh = out->head_stride;
    a.lse = lse;
    a.k = (const char *)cache->k;
    a.v = (const char *)cache->v;
    a.ks = cache->k_scale;
    a.vs = cache->v_scale;
    a.table = b.table;
    a.table_stride = b.table_stride;
    a.capacity = b.table_cols * cache->page_size;
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
    a.q_bf16 = q->type == WS_KV_BF16;
    if (L.bytes) {
      a.few_o = (float *)d_workspace;
      a.many_o = a.few_o + L.few_slots * cache->dim;
      a.few_ml = (float2 *)(a.many_o + L.many_slots * cache->dim);
      a.many_ml = a.few_ml + L.few_slots;
    }
    a.few_splits = L.few_splits;
    a.few_chunk = L.few_chunk;
    a.few_blocks = L.few_blocks;
    a.few_room = L.few_room;
    a.few_head = L.few_head;
    a.few_seq = L.few_seq;
    a.few_token = L.few_token;
    a.many_splits = L.many_splits;
    a.many_chunk = L.many_chunk;
    a.both = L.many;
    a.row_blocks = L.row_blocks;
    hipStream_t s = (hipStream_t)hip_stream;
    switch (cache->type) {
      case WS_KV_BF16: return attention_dim<WS_KV_BF16>(cache->dim, a, L, s);
      case WS_KV_FP16: return attention_dim<WS_KV_FP16>(cache->dim, a, L, s);
      case WS_KV_FP8: return attention_dim<WS_KV_FP8>(cache->dim, a, L, s);
      default: return attention_dim<WS_KV_INT8>(cache->dim, a, L, s);
    }
  });
}

}  // extern "C"

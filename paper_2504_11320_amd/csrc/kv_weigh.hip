// The attention that cached keys received.
//
// S_j = sum over the rows (token, head of a group) that see key j of
// 2^(scale log2(e) q . k_j - log2(e) lse): attention's weights again, from its
// log-sums, added up over the rows instead of the keys.  Matrix instructions
// compute Q K^T with the keys as columns, so that a key's weights are in one lane
// column and add up without leaving it.  A wave keeps its keys in registers and
// takes the rows in blocks.
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
  int32_t tiles;  // of a request's keys, that the launch is laid out for
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

// Tokens [lo, hi) of which each may see a key of k0 .. k1 - 1.
__device__ __forceinline__ Range tokens_of(const Args &a, const Seq &s, int32_t k0, int32_t k1) {
  const int64_t old = (int64_t)s.m - s.n;  // the first token's position
  Range r = {0, s.n};
  if (a.causal) r.lo = (int32_t)min((int64_t)s.n, max((int64_t)0, k0 - old));
  if (a.window)
    r.hi = (int32_t)min((int64_t)s.n, max((int64_t)0, (int64_t)k1 - 1 + a.window - old));
  return r;
}

constexpr int kFewKeys = 64;  // of a wave

// Up to 16 rows at a time against 64 keys a wave.
template <int TYPE, bool BF, int D>
__global__ void __launch_bounds__(256, 2) few_kernel(Args a) {
  constexpr int esz = kCodes<TYPE> ? 1 : 2;
  constexpr int steps = D / 32, kloads = D * esz / 64, tiles = kFewKeys / 16;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n16 = lane & 15, g = lane >> 4;
  const int32_t tile = blockIdx.x % a.tiles, pair = blockIdx.x / a.tiles;
  const int32_t h = pair % a.kv_heads, b = pair / a.kv_heads;
  const Seq s = get_seq(a, b);
  const int32_t end = min(s.m, a.capacity);
  for (int32_t k0 = (tile * 4 + wave) * kFewKeys; k0 < end; k0 += a.tiles * 4 * kFewKeys) {
    const int32_t key = k0 + lane;
    const int32_t row_at = cache_row(a, page_entry(a, b, key, end), h, key, end);
    const Range tokens = tokens_of(a, s, k0, min(k0 + kFewKeys, end));
    const bool fresh = !a.accumulate || key >= s.m - s.n;
    if (tokens.lo >= tokens.hi && !__any(fresh)) continue;
    u32x4 kreg[tiles][kloads];
#pragma unroll
    for (int t = 0; t < tiles; ++t) {
      const int64_t r = max(__shfl(row_at, 16 * t + n16), 0);
      const char *p = a.k + r * (D * esz) + 16 * g;
#pragma unroll
      for (int i = 0; i < kloads; ++i) kreg[t][i] = *reinterpret_cast<const u32x4 *>(p + 64 * i);
    }
    float by = a.scale;
    if constexpr (kCodes<TYPE>) by *= a.ks[max(row_at, 0)];
    float weight = 0.0f;
    if (!fresh && row_at != kNoRow) weight = a.weights[row_at];
    float sum[tiles] = {};
    const int32_t last = tokens.hi * a.group;
    for (int32_t r0 = tokens.lo * a.group; r0 < last; r0 += 16) {
      const int32_t row = r0 + n16;
      const bool live = row < last;
      const int32_t token = live ? row / a.group : 0;
      const int32_t head = h * a.group + (live ? row - token * a.group : 0);
      const int64_t at = s.q0 + token;
      const uint16_t *p = a.q + at * a.qt + head * a.qh;
      const bool wide = ((a.qt | a.qh) & 7) == 0 && ((uintptr_t)a.q & 15) == 0;
      u32x4 q[steps];
#pragma unroll
      for (int i = 0; i < steps; ++i) {
        const int d = kCodes<TYPE> ? 64 * (i / 2) + 16 * g + 8 * (i % 2) : 32 * i + 8 * g;
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
      const float mine = live ? row_log(a.lse[at * a.heads + head]) : INFINITY;
      Range see = token_range(a, s, token);
      if (!live) see = {0, 0};
      // every row sees all of the keys: no masks
      const bool all =
          __all(!live || (see.lo <= k0 && see.hi >= k0 + kFewKeys));
      float log[4];
      Range range[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        log[r] = __shfl(mine, 4 * g + r);
        range[r] = {__shfl(see.lo, 4 * g + r), __shfl(see.hi, 4 * g + r)};
      }
#pragma unroll
      for (int t = 0; t < tiles; ++t) {
        f32x4 z = {0, 0, 0, 0};
        if constexpr (kCodes<TYPE>) {
#pragma unroll
          for (int i = 0; i < kloads; ++i) {
            u32x4 lo, hi;
            codes_to_16<TYPE, BF>(kreg[t][i], lo, hi);
            z = mfma16<BF>(q[2 * i], lo, z);
            z = mfma16<BF>(q[2 * i + 1], hi, z);
          }
        } else {
#pragma unroll
          for (int i = 0; i < kloads; ++i) z = mfma16<BF>(q[i], kreg[t][i], z);
        }
        const float factor = kCodes<TYPE> ? __shfl(by, 16 * t + n16) : by;
        const int32_t j = k0 + 16 * t + n16;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float p = exp2_of(__builtin_fmaf(z[r], factor, -log[r]));
          if (!all) p = j >= range[r].lo && j < range[r].hi ? p : 0.0f;
          sum[t] += p;
        }
      }
    }
    float mine = 0.0f;
#pragma unroll
    for (int t = 0; t < tiles; ++t) {
      sum[t] += __shfl_xor(sum[t], 16);
      sum[t] += __shfl_xor(sum[t], 32);
      if (g == t) mine = sum[t];
    }
    if (row_at != kNoRow) a.weights[row_at] = weight + mine;
  }
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

template <int TYPE, bool BF, int D>
int weigh_launch(const Args &a, hipStream_t stream) {
  const int64_t blocks = (int64_t)a.n_seq * a.kv_heads * a.tiles;
  if (blocks * 256 >= (int64_t)1 << 32)
    return ws_record_failure(WS_EUNSUPPORTED, "weigh: too many workgroups");
  few_kernel<TYPE, BF, D><<<dim3((uint32_t)blocks), 256, 0, stream>>>(a);
  return launched();
}

template <int TYPE, bool BF>
int weigh_dim(int dim, const Args &a, hipStream_t stream) {
  if (dim == 64) return weigh_launch<TYPE, BF, 64>(a, stream);
  if (dim == 128) return weigh_launch<TYPE, BF, 128>(a, stream);
  return weigh_launch<TYPE, BF, 256>(a, stream);
}

// Whether byte ranges meet.
bool meet(const void *a, int64_t na, const void *b, int64_t nb) {
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
    *bytes = 0;
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
    if (meet(weights, cells * 4, lse, (int64_t)b.n_tokens * b.heads * 4) ||
        meet(weights, cells * 4, cache->k, cells * cache->dim * type_bytes(cache->type)) ||
        (cache->k_scale && meet(weights, cells * 4, cache->k_scale, cells * 4)))
      return invalid("weigh: the weights must not overlap the log-sums or the keys");
    const int64_t capacity = (int64_t)b.table_cols * cache->page_size;
    if (capacity == 0) return WS_OK;
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
    a.tiles = (int32_t)ceil_div(longest, 4 * kFewKeys);
    hipStream_t s = (hipStream_t)hip_stream;
    const bool bf = q->type == WS_KV_BF16;
    switch (cache->type) {
      case WS_KV_BF16: return weigh_dim<WS_KV_BF16, true>(cache->dim, a, s);
      case WS_KV_FP16: return weigh_dim<WS_KV_FP16, false>(cache->dim, a, s);
      case WS_KV_FP8:
        return bf ? weigh_dim<WS_KV_FP8, true>(cache->dim, a, s)
                  : weigh_dim<WS_KV_FP8, false>(cache->dim, a, s);
      default:
        return bf ? weigh_dim<WS_KV_INT8, true>(cache->dim, a, s)
                  : weigh_dim<WS_KV_INT8, false>(cache->dim, a, s);
    }
  });
}

}  // extern "C"

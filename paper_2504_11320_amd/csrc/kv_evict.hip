// Eviction from a cache by accumulated weights.
//
// One kernel finds the kept keys of each request and KV head: with weights as
// whole numbers of the same order, the smallest kept one is found digit by digit
// (a histogram of the next digit of those that share the digits so far), and the
// kept indices are written in order.  A second one moves their rows.
#include <cmath>

#include "kv_common.h"
#include "wait_kv_budget.h"

namespace {

using namespace kv;

struct Args {
  char *k, *v;
  float *ks, *vs, *weights;
  const int32_t *table, *to;
  int64_t table_stride, to_stride;
  const int32_t *lens;
  int32_t *kept, *new_lens;
  int32_t capacity;  // keys that the table's columns hold
  int32_t kv_heads, pages, page_shift;
  int32_t keep, recent;
  int32_t blocks;    // of a request and head, that move rows
};

__device__ __forceinline__ int32_t length_of(const Args &a, int32_t b) {
  return min(max(a.lens[b], 0), a.capacity);
}
// The row of the cache at a position of a list of pages, for KV head h.
__device__ __forceinline__ int32_t row_of(const Args &a, const int32_t *list, int32_t h, int32_t j) {
  const int32_t page = list[j >> a.page_shift];
  const int32_t row = ((page * a.kv_heads + h) << a.page_shift) + (j & ((1 << a.page_shift) - 1));
  return (uint32_t)page < (uint32_t)a.pages ? row : kNoRow;
}

// Whole numbers that order as the weights do: zeros of both signs are equal, NaN
// is the largest; 0 is less than all of them.
__device__ __forceinline__ uint32_t order_of(float w) {
  const uint32_t bits = __float_as_uint(w + 0.0f);
  const uint32_t up = bits & 0x80000000u ? ~bits : bits | 0x80000000u;
  return w != w ? 0xffffffffu : up;
}

template <int THREADS>
constexpr int kHeld = THREADS == 256 ? 4096 : 32768;  // weights in shared memory

template <int THREADS>
struct Shared {
  uint32_t order[kHeld<THREADS>];
  int32_t count[256];
  int32_t above[THREADS / 64], equal[THREADS / 64];
  uint32_t digit;
  int32_t left;
};

// The kept ones of the keys 0 .. n - 1, `need` of them, 0 < need < n; order(j)
// gives key j's.
template <int THREADS, class F>
__device__ __forceinline__ void pick(Shared<THREADS> &sh, int32_t *kept, int32_t n, int32_t need,
                                     F &&order) {
  constexpr int waves = THREADS / 64;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t least = 0;   // digits of the smallest kept one
  int32_t left = need;  // of those that share them, so many stay
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < 256; i += THREADS) sh.count[i] = 0;
    __syncthreads();
    for (int32_t j = threadIdx.x; j < n; j += THREADS) {
      const uint32_t x = order(j);
      if (shift == 24 || (x ^ least) >> (shift + 8) == 0) atomicAdd(&sh.count[x >> shift & 255], 1);
    }
    __syncthreads();
    if (wave == 0) {  // four digits a lane, the largest in lane 0
      int32_t c[4], mine = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) mine += c[i] = sh.count[255 - 4 * lane - i];
      int32_t upto = mine;
      for (int m = 1; m < 64; m *= 2) {
        const int32_t other = __shfl_up(upto, m);
        if (lane >= m) upto += other;
      }
      int32_t before = upto - mine;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (before < left && before + c[i] >= left) {
          sh.digit = 255 - 4 * lane - i;
          sh.left = left - before;
        }
        before += c[i];
      }
    }
    __syncthreads();
    least |= sh.digit << shift;
    left = sh.left;
    __syncthreads();
  }
  // each wave takes keys that follow one another
  const int32_t each = ((n + waves - 1) / waves + 63) / 64 * 64;
  const int32_t from = min(wave * each, n), to = min(from + each, n);
  int32_t above = 0, equal = 0;
  for (int32_t j0 = from; j0 < to; j0 += 64) {
    const int32_t j = j0 + lane;
    const uint32_t x = j < to ? order(j) : 0;
    above += __popcll(__ballot(j < to && x > least));
    equal += __popcll(__ballot(j < to && x == least));
  }
  if (lane == 0) {
    sh.above[wave] = above;
    sh.equal[wave] = equal;
  }
  __syncthreads();
  above = equal = 0;
  for (int w = 0; w < wave; ++w) {
    above += sh.above[w];
    equal += sh.equal[w];
  }
  int32_t at = above + min(equal, left);
  const uint64_t below = (1ull << lane) - 1;
  for (int32_t j0 = from; j0 < to; j0 += 64) {
    const int32_t j = j0 + lane;
    const uint32_t x = j < to ? order(j) : 0;
    const uint64_t same = __ballot(j < to && x == least);
    const bool stays = j < to && (x > least || (x == least && equal + __popcll(same & below) < left));
    const uint64_t all = __ballot(stays);
    if (stays) kept[at + __popcll(all & below)] = j;
    at += __popcll(all);
    equal += __popcll(same);
  }
}

template <int THREADS>
__global__ void __launch_bounds__(THREADS) pick_kernel(Args a) {
  __shared__ Shared<THREADS> sh;
  const int32_t h = blockIdx.x % a.kv_heads, b = blockIdx.x / a.kv_heads;
  const int32_t m = length_of(a, b);
  int32_t *kept = a.kept + (int64_t)blockIdx.x * a.keep;
  if (h == 0 && threadIdx.x == 0) a.new_lens[b] = min(m, a.keep);
  const int32_t n = m - a.recent, need = a.keep - a.recent;
  if (m <= a.keep || need == 0) {
    const int32_t first = m <= a.keep ? 0 : n;
    for (int32_t d = threadIdx.x; d < a.keep; d += THREADS) kept[d] = d < m ? first + d : -1;
    return;
  }
  const int32_t *pages = a.table + b * a.table_stride;
  auto order = [&](int32_t j) {
    const int32_t row = row_of(a, pages, h, j);
    return row == kNoRow ? 0u : order_of(a.weights[row]);
  };
  if (n <= kHeld<THREADS>) {
    for (int32_t j = threadIdx.x; j < n; j += THREADS) sh.order[j] = order(j);
    __syncthreads();
    pick(sh, kept, n, need, [&](int32_t j) { return sh.order[j]; });
  } else {
    pick(sh, kept, n, need, order);
  }
  for (int32_t d = threadIdx.x; d < a.recent; d += THREADS) kept[need + d] = n + d;
}

// ------------------------------------------------------------- rows ------

constexpr int kRows = 4;  // of a thread

// Rows to other pages: each of C lanes takes 16 bytes of the two rows of a key.
template <int C>
__global__ void __launch_bounds__(256) move_kernel(Args a) {
  constexpr int groups = 256 / C;
  const int lane = threadIdx.x % C;
  const int32_t pair = blockIdx.x / a.blocks, block = blockIdx.x % a.blocks;
  const int32_t h = pair % a.kv_heads, b = pair / a.kv_heads;
  const int32_t count = min(length_of(a, b), a.keep);
  const int32_t *pages = a.table + b * a.table_stride, *to = a.to + b * a.to_stride;
  const int32_t *kept = a.kept + (int64_t)pair * a.keep;
  int32_t from[kRows], at[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int32_t d = (block * kRows + i) * groups + threadIdx.x / C;
    from[i] = at[i] = kNoRow;
    if (d < count) {
      from[i] = row_of(a, pages, h, kept[d]);
      at[i] = row_of(a, to, h, d);
    }
  }
  u32x4 x[kRows], y[kRows];
  float s[kRows], t[kRows], w[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    if (from[i] == kNoRow || at[i] == kNoRow) continue;
    x[i] = *reinterpret_cast<const u32x4 *>(a.k + ((int64_t)from[i] * C + lane) * 16);
    y[i] = *reinterpret_cast<const u32x4 *>(a.v + ((int64_t)from[i] * C + lane) * 16);
    if (lane == 0) {
      w[i] = a.weights[from[i]];
      if (a.ks) {
        s[i] = a.ks[from[i]];
        t[i] = a.vs[from[i]];
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    if (from[i] == kNoRow || at[i] == kNoRow) continue;
    *reinterpret_cast<u32x4 *>(a.k + ((int64_t)at[i] * C + lane) * 16) = x[i];
    *reinterpret_cast<u32x4 *>(a.v + ((int64_t)at[i] * C + lane) * 16) = y[i];
    if (lane == 0) {
      a.weights[at[i]] = w[i];
      if (a.ks) {
        a.ks[at[i]] = s[i];
        a.vs[at[i]] = t[i];
      }
    }
  }
}

// Rows within a request's own pages: one workgroup takes the keys or the values
// of a request and head from the front on.  A row never goes behind its place,
// so what a step writes lies before what later steps read; within a step
// everything is read before anything is written.
template <int C>
__global__ void __launch_bounds__(256) close_up_kernel(Args a) {
  constexpr int groups = 256 / C, step = groups * kRows;
  const int lane = threadIdx.x % C;
  const bool values = blockIdx.x & 1;
  const int32_t pair = blockIdx.x / 2;
  const int32_t h = pair % a.kv_heads, b = pair / a.kv_heads;
  if (length_of(a, b) <= a.keep) return;
  const int32_t *pages = a.table + b * a.table_stride;
  const int32_t *kept = a.kept + (int64_t)pair * a.keep;
  char *rows = values ? a.v : a.k;
  float *scales = values ? a.vs : a.ks, *weights = values ? nullptr : a.weights;
  for (int32_t d0 = 0; d0 < a.keep; d0 += step) {
    const int32_t last = min(d0 + step, a.keep) - 1;
    if (kept[last] == last) continue;  // nothing before it moves
    int32_t from[kRows], at[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int32_t d = d0 + i * groups + threadIdx.x / C;
      from[i] = at[i] = kNoRow;
      if (d <= last) {
        from[i] = row_of(a, pages, h, kept[d]);
        at[i] = row_of(a, pages, h, d);
      }
    }
    u32x4 x[kRows];
    float s[kRows], w[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      x[i] = u32x4{0, 0, 0, 0};
      s[i] = w[i] = 0.0f;
      if (from[i] == kNoRow) continue;
      x[i] = *reinterpret_cast<const u32x4 *>(rows + ((int64_t)from[i] * C + lane) * 16);
      if (lane == 0) {
        if (scales) s[i] = scales[from[i]];
        if (weights) w[i] = weights[from[i]];
      }
    }
    // all of it has arrived, in every wave, before any of it is overwritten
#pragma unroll
    for (int i = 0; i < kRows; ++i) asm volatile("" : "+v"(x[i]), "+v"(s[i]), "+v"(w[i])::"memory");
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      if (from[i] == kNoRow || at[i] == kNoRow) continue;
      *reinterpret_cast<u32x4 *>(rows + ((int64_t)at[i] * C + lane) * 16) = x[i];
      if (lane == 0) {
        if (scales) scales[at[i]] = s[i];
        if (weights) weights[at[i]] = w[i];
      }
    }
  }
}

// -------------------------------------------------------------- host -----

template <int C>
int move_rows(Args a, int64_t pairs, hipStream_t stream) {
  if (!a.to) {
    if (pairs * 2 * 256 >= (int64_t)1 << 32)
      return ws_record_failure(WS_EUNSUPPORTED, "evict: too many workgroups");
    close_up_kernel<C><<<dim3((uint32_t)(pairs * 2)), 256, 0, stream>>>(a);
    return launched();
  }
  constexpr int each = 256 / C * kRows;
  a.blocks = (a.keep + each - 1) / each;
  if (pairs * a.blocks * 256 >= (int64_t)1 << 32)
    return ws_record_failure(WS_EUNSUPPORTED, "evict: too many workgroups");
  move_kernel<C><<<dim3((uint32_t)(pairs * a.blocks)), 256, 0, stream>>>(a);
  return launched();
}

}  // namespace

extern "C" {

int wait_kv_evict(const ws_kv_cache *cache, const ws_kv_eviction *eviction, float *weights,
                  int32_t *kept, int32_t *new_lens, void *hip_stream) {
  return guarded([&]() -> int {
    if (int rc = check_cache(cache)) return rc;
    if (!eviction) return invalid("evict: the eviction must be non-NULL");
    const ws_kv_eviction &e = *eviction;
    if (e.n_seq < 0 || e.table_cols < 0 || e.table_stride < 0) return invalid("evict: bad sizes");
    if (e.keep < 1) return invalid("evict: at least one key must be kept");
    if (e.recent < 0 || e.recent > e.keep) return invalid("evict: recent must be 0 to keep");
    if (e.max_kv_len < 0) return invalid("evict: bad length bound");
    if ((int64_t)e.table_cols * cache->page_size >= (int64_t)1 << 30 || e.keep >= 1 << 30)
      return ws_record_failure(WS_EUNSUPPORTED, "evict: 2^30 keys a request or more");
    if (e.to && (e.to_stride < 0 || (int64_t)e.to_cols * cache->page_size < e.keep))
      return invalid("evict: the kept rows need pages to go to");
    if (e.n_seq == 0) return WS_OK;
    if (!e.kv_lens || !weights || !kept || !new_lens || (e.table_cols > 0 && !e.table))
      return invalid("evict: the page table, lengths, weights and outputs must be non-NULL");
    if ((uintptr_t)e.table % 4 || (uintptr_t)e.to % 4 || (uintptr_t)e.kv_lens % 4 ||
        (uintptr_t)weights % 4 || (uintptr_t)kept % 4 || (uintptr_t)new_lens % 4)
      return invalid("evict: tables, lengths, weights and outputs must be aligned to 4 bytes");
    const int64_t pairs = (int64_t)e.n_seq * cache->kv_heads;
    if (e.kv_lens < new_lens + e.n_seq && new_lens < e.kv_lens + e.n_seq)
      return invalid("evict: the new lengths need memory of their own");
    Args a{};
    a.k = (char *)cache->k;
    a.v = (char *)cache->v;
    a.ks = cache->k_scale;
    a.vs = cache->v_scale;
    a.weights = weights;
    a.table = e.table;
    a.to = e.to;
    a.table_stride = e.table_stride;
    a.to_stride = e.to_stride;
    a.lens = e.kv_lens;
    a.kept = kept;
    a.new_lens = new_lens;
    a.capacity = e.table_cols * cache->page_size;
    a.kv_heads = cache->kv_heads;
    a.pages = cache->pages;
    a.page_shift = log2_of(cache->page_size);
    a.keep = e.keep;
    a.recent = e.recent;
    if (pairs * 1024 >= (int64_t)1 << 32)
      return ws_record_failure(WS_EUNSUPPORTED, "evict: too many requests times heads");
    hipStream_t s = (hipStream_t)hip_stream;
    if (e.max_kv_len <= kHeld<256>)
      pick_kernel<256><<<dim3((uint32_t)pairs), 256, 0, s>>>(a);
    else
      pick_kernel<1024><<<dim3((uint32_t)pairs), 1024, 0, s>>>(a);
    if (int rc = launched()) return rc;
    switch (cache->dim * type_bytes(cache->type) / 16) {
      case 4: return move_rows<4>(a, pairs, s);
      case 8: return move_rows<8>(a, pairs, s);
      case 16: return move_rows<16>(a, pairs, s);
      default: return move_rows<32>(a, pairs, s);
    }
  });
}

}  // extern "C"

// Eviction from a cache by accumulated weights: the kept keys of each request and
// KV head are found, then their rows move.
//
// Weights are compared as whole numbers of the same order.  Up to 2048 keys, a
// wave holds them in registers and halves the range that the smallest kept one
// lies in until as many are above as may stay.  More keys are split over
// workgroups, and that number is found digit by digit: a histogram of the next
// digit of those that share the digits so far, one launch each.
#include <algorithm>
#include <cmath>

#include "kv_common.h"
#include "wait_kv_budget.h"

namespace {

using namespace kv;

// What a part of the keys knows of the smallest kept weight.
struct Found {
  uint32_t least;  // its digits so far
  int32_t left;    // of those that share them, so many stay
  int32_t above;   // of the parts before, so many are larger
  int32_t unused;
};

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
  int32_t parts;     // of a request's keys, that are counted
  int32_t *counts;   // [digit][request][KV head][part][256]
  Found *found;      // [request][KV head][part]
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

// A request and KV head: its keys, those among which the heaviest stay, and how
// many do.
struct Pair {
  const int32_t *pages;
  int32_t h, m, n, need;
  __device__ __forceinline__ Pair(const Args &a, int32_t pair) {
    h = pair % a.kv_heads;
    const int32_t b = pair / a.kv_heads;
    pages = a.table + b * a.table_stride;
    m = length_of(a, b);
    n = m - a.recent;
    need = a.keep - a.recent;
  }
  // Which keys stay does not depend on weights: the first, or the last, so many.
  __device__ __forceinline__ bool simple(const Args &a) const { return m <= a.keep || need == 0; }
  __device__ __forceinline__ int32_t simply(const Args &a, int32_t d) const {
    return d >= m ? -1 : m <= a.keep ? d : n + d;
  }
  __device__ __forceinline__ uint32_t order(const Args &a, int32_t j) const {
    const int32_t row = row_of(a, pages, h, j);
    return row == kNoRow ? 0u : order_of(a.weights[row]);
  }
};

// ------------------------------------------------- up to 2048 keys ------

constexpr int kHeld = 32;  // keys of a lane, at most

// The kept ones of n keys, 0 < need < n <= 64 R: `kept` gets their indices.
template <int R, class F>
__device__ __forceinline__ void pick_held(int32_t n, int32_t need, F &&order, int32_t *kept) {
  const int lane = threadIdx.x & 63;
  uint32_t x[R];
#pragma unroll
  for (int i = 0; i < R; ++i) x[i] = order(min(64 * i + lane, n - 1));
  uint32_t low = 0xffffffffu, high = 0;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    low = min(low, x[i]);
    high = max(high, x[i]);
    // Behind the last key 0, which is not more than any: it is not counted, and
    // where it equals the smallest kept number it comes behind all that do.
    if (64 * i + lane >= n) x[i] = 0;
  }
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    low = min(low, (uint32_t)__shfl_xor((int)low, m));
    high = max(high, (uint32_t)__shfl_xor((int)high, m));
  }
  // More than `need` numbers are lo or more, up to that many are above hi: the
  // smallest kept one is in lo .. hi.
  uint32_t lo = __builtin_amdgcn_readfirstlane(low), hi = __builtin_amdgcn_readfirstlane(high);
  int32_t left = need;  // of those that equal hi, once that is lo
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo) / 2 + 1;  // lo < mid <= hi
    int32_t c = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) c += __popcll(__ballot(x[i] >= mid));
    if (c > need) {
      lo = mid;
    } else {
      hi = mid - 1;
      left = need - c;
      if (left == 0) break;  // those above hi are the kept ones
    }
  }
  int32_t at = 0;
  const uint64_t below = (1ull << lane) - 1;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const uint64_t same = __ballot(x[i] == hi);
    const bool stays = x[i] > hi || (x[i] == hi && (int32_t)__popcll(same & below) < left);
    left = max(0, left - (int32_t)__popcll(same));
    const uint64_t all = __ballot(stays);
    if (stays) kept[at + __popcll(all & below)] = 64 * i + lane;
    at += __popcll(all);
  }
}
template <class F>
__device__ __forceinline__ void pick_held(int32_t n, int32_t need, F &&order, int32_t *kept) {
  if (n <= 64 * 8)
    pick_held<8>(n, need, order, kept);
  else if (n <= 64 * 16)
    pick_held<16>(n, need, order, kept);
  else if (n <= 64 * 24)
    pick_held<24>(n, need, order, kept);
  else
    pick_held<kHeld>(n, need, order, kept);
}

// ------------------------------------------- any number, a workgroup ----

struct Scan {
  int32_t count[4][256];
  int32_t above[4], equal[4];
  uint32_t digit;
  int32_t left;
};

// Of the counts of 256 digits, the digit that the left-th largest has, and how many
// of those with it stay: sh.digit, sh.left.
__device__ __forceinline__ void find_digit(Scan &sh, int32_t left) {
  if (threadIdx.x < 64) {  // four digits a lane, the largest in lane 0
    const int lane = threadIdx.x;
    int32_t c[4], mine = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) mine += c[i] = sh.count[0][255 - 4 * lane - i];
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
}

// Counts of a digit of the keys from .. to - 1 that share the digits above it, one
// array a wave, added up in the first.
template <class F>
__device__ __forceinline__ void count_digits(Scan &sh, int32_t from, int32_t to, uint32_t least,
                                             int shift, F &&order) {
  const int wave = threadIdx.x >> 6;
  for (int i = threadIdx.x; i < 1024; i += 256) sh.count[0][i] = 0;
  __syncthreads();
  constexpr int ahead = 4;
  for (int32_t j0 = from; j0 < to; j0 += 256 * ahead) {
    uint32_t x[ahead];
#pragma unroll
    for (int i = 0; i < ahead; ++i) x[i] = order(min(j0 + i * 256 + (int32_t)threadIdx.x, to - 1));
#pragma unroll
    for (int i = 0; i < ahead; ++i) {
      const bool is = j0 + i * 256 + (int32_t)threadIdx.x < to;
      if (is && (shift == 24 || (x[i] ^ least) >> (shift + 8) == 0))
        atomicAdd(&sh.count[wave][x[i] >> shift & 255], 1);
    }
  }
  __syncthreads();
  const int t = threadIdx.x;
  sh.count[0][t] += sh.count[1][t] + sh.count[2][t] + sh.count[3][t];
  __syncthreads();
}

// The kept ones of the keys from .. to - 1 go to kept[above + min(equal, left)] and
// on: larger than least, or among the first `left` that equal it, `equal` of
// which lie before.
template <class F>
__device__ __forceinline__ void write_kept(Scan &sh, int32_t from, int32_t to, uint32_t least,
                                           int32_t left, int32_t above, int32_t equal, F &&order,
                                           int32_t *kept) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // each wave takes keys that follow one another
  const int32_t each = ((to - from + 3) / 4 + 63) / 64 * 64;
  const int32_t first = min(from + wave * each, to), last = min(first + each, to);
  int32_t more = 0, same = 0;
  for (int32_t j0 = first; j0 < last; j0 += 64) {
    const int32_t j = j0 + lane;
    const uint32_t x = order(min(j, to - 1));
    more += __popcll(__ballot(j < last && x > least));
    same += __popcll(__ballot(j < last && x == least));
  }
  if (lane == 0) {
    sh.above[wave] = more;
    sh.equal[wave] = same;
  }
  __syncthreads();
  for (int w = 0; w < wave; ++w) {
    above += sh.above[w];
    equal += sh.equal[w];
  }
  int32_t at = above + min(equal, left);
  const uint64_t below = (1ull << lane) - 1;
  for (int32_t j0 = first; j0 < last; j0 += 64) {
    const int32_t j = j0 + lane;
    const uint32_t x = order(min(j, to - 1));
    const uint64_t ties = __ballot(j < last && x == least);
    const bool stays =
        j < last && (x > least || (x == least && equal + (int32_t)__popcll(ties & below) < left));
    const uint64_t all = __ballot(stays);
    if (stays) kept[at + __popcll(all & below)] = j;
    at += __popcll(all);
    equal += __popcll(ties);
  }
}

// The kept ones of a request longer than its launch was laid out for, by one
// workgroup.
template <class F>
__device__ __forceinline__ void pick_any(Scan &sh, int32_t n, int32_t need, F &&order, int32_t *kept) {
  uint32_t least = 0;
  int32_t left = need;
  for (int shift = 24; shift >= 0; shift -= 8) {
    count_digits(sh, 0, n, least, shift, order);
    find_digit(sh, left);
    least |= sh.digit << shift;
    left = sh.left;
    __syncthreads();
  }
  write_kept(sh, 0, n, least, left, 0, 0, order, kept);
}

// ------------------------------------------------------ many keys -------

struct Range {
  int32_t lo, hi;
};
__device__ __forceinline__ Range part_of(const Args &a, int32_t part, int32_t n) {
  const int64_t each = ((int64_t)(n + a.parts - 1) / a.parts + 63) / 64 * 64;
  return {(int32_t)min((int64_t)n, part * each), (int32_t)min((int64_t)n, (part + 1) * each)};
}

// The digit that the counts of all parts give; what this part knows behind it;
// `equal` gets how many of the parts before share it.
__device__ __forceinline__ Found next_digit(Scan &sh, const Args &a, int32_t pair, int32_t part,
                                            int digit, Found f, int32_t *equal) {
  const int t = threadIdx.x;
  const int32_t *c = a.counts + (((int64_t)digit * (gridDim.x / a.parts) + pair) * a.parts) * 256 + t;
  int32_t all = 0, before = 0;
#pragma unroll 8
  for (int32_t q = 0; q < a.parts; ++q) {
    const int32_t x = c[q * 256];
    all += x;
    before += q < part ? x : 0;
  }
  sh.count[0][t] = all;
  sh.count[1][t] = before;
  __syncthreads();
  find_digit(sh, f.left);
  const uint32_t d = sh.digit;
  int32_t above = (uint32_t)t > d ? before : 0;
  for (int m = 1; m < 64; m *= 2) above += __shfl_xor(above, m);
  if ((t & 63) == 0) sh.above[t >> 6] = above;
  __syncthreads();
  f.above += sh.above[0] + sh.above[1] + sh.above[2] + sh.above[3];
  f.least |= d << (24 - 8 * digit);
  f.left = sh.left;
  *equal = sh.count[1][d];
  __syncthreads();
  return f;
}

// Launch number `digit` counts that digit, once the ones before are known; the one
// behind the last digit writes the kept keys.  131,072 keys of 8 heads: five
// launches of 2 to 4 us, 310 us by one workgroup a head.
__global__ void __launch_bounds__(256) count_kernel(Args a, int digit) {
  __shared__ Scan sh;
  const int32_t part = blockIdx.x % a.parts, pair = blockIdx.x / a.parts;
  const Pair p(a, pair);
  int32_t *kept = a.kept + (int64_t)pair * a.keep;
  if (digit == 4 && p.h == 0 && part == 0 && threadIdx.x == 0)
    a.new_lens[pair / a.kv_heads] = min(p.m, a.keep);
  if (p.simple(a)) {
    if (digit == 4)
      for (int32_t d = part * 256 + threadIdx.x; d < a.keep; d += a.parts * 256)
        kept[d] = p.simply(a, d);
    return;
  }
  Found f = {0, p.need, 0, 0};
  int32_t equal = 0;
  if (digit > 0) {
    if (digit > 1) f = a.found[blockIdx.x];
    f = next_digit(sh, a, pair, part, digit - 1, f, &equal);
  }
  const Range r = part_of(a, part, p.n);
  auto order = [&](int32_t j) { return p.order(a, j); };
  if (digit < 4) {
    if (digit > 0 && threadIdx.x == 0) a.found[blockIdx.x] = f;
    count_digits(sh, r.lo, r.hi, f.least, 24 - 8 * digit, order);
    a.counts[((int64_t)digit * gridDim.x + blockIdx.x) * 256 + threadIdx.x] =
        sh.count[0][threadIdx.x];
    return;
  }
  if (r.lo < r.hi) write_kept(sh, r.lo, r.hi, f.least, f.left, f.above, equal, order, kept);
  for (int32_t d = part * 256 + threadIdx.x; d < a.recent; d += a.parts * 256)
    kept[p.need + d] = p.n + d;
}

// ------------------------------------------------------------- rows ------

constexpr int kRows = 4;  // of a thread

// Kept rows d, d + step, ... to other pages: each of C lanes takes 16 bytes of the
// two rows of a key; key_of(d) is the kept key.
template <int C, class F>
__device__ __forceinline__ void move_rows(const Args &a, const Pair &p, const int32_t *to,
                                          int32_t d0, int32_t step, int32_t count, F &&key_of) {
  const int lane = threadIdx.x % C;
  int32_t from[kRows], at[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int32_t d = d0 + i * step;
    from[i] = at[i] = kNoRow;
    if (d < count) {
      from[i] = row_of(a, p.pages, p.h, key_of(d));
      at[i] = row_of(a, to, p.h, d);
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

// Behind count_kernel.
template <int C>
__global__ void __launch_bounds__(256) move_kernel(Args a) {
  constexpr int groups = 256 / C;
  const int32_t pair = blockIdx.x / a.blocks, block = blockIdx.x % a.blocks;
  const Pair p(a, pair);
  const int32_t *kept = a.kept + (int64_t)pair * a.keep;
  move_rows<C>(a, p, a.to + pair / a.kv_heads * a.to_stride, block * kRows * groups + threadIdx.x / C,
               groups, min(p.m, a.keep), [&](int32_t d) { return kept[d]; });
}

// The kept keys of a request and head that has up to 2048 and, where C is not 0,
// their rows to other pages: the workgroups that share the rows find the keys each
// for itself, which takes less than another launch.
template <int C>
__global__ void __launch_bounds__(256) pick_kernel(Args a) {
  __shared__ Scan sh;
  __shared__ int32_t list[64 * kHeld];
  const int32_t pair = blockIdx.x / a.blocks, block = blockIdx.x % a.blocks;
  const Pair p(a, pair);
  int32_t *kept = a.kept + (int64_t)pair * a.keep;
  if (p.h == 0 && block == 0 && threadIdx.x == 0) a.new_lens[pair / a.kv_heads] = min(p.m, a.keep);
  const bool simple = p.simple(a), held = p.n <= 64 * kHeld;
  auto order = [&](int32_t j) { return p.order(a, j); };
  if (!simple) {
    if (!held)  // the same list by each of the workgroups
      pick_any(sh, p.n, p.need, order, kept);
    else if (threadIdx.x < 64)
      pick_held(p.n, p.need, order, list);
    __syncthreads();
  }
  auto key_of = [&](int32_t d) {
    if (simple) return p.simply(a, d);
    return d >= p.need ? p.n + d - p.need : held ? list[d] : kept[d];
  };
  const int32_t from = simple || held ? 0 : p.need;  // the others are written
  if (block == 0)
    for (int32_t d = from + threadIdx.x; d < a.keep; d += 256) kept[d] = key_of(d);
  if constexpr (C != 0) {
    constexpr int groups = 256 / C;
    const int32_t count = min(p.m, a.keep);
    const int32_t *to = a.to + pair / a.kv_heads * a.to_stride;
    for (int32_t d = block * kRows * groups; d < count; d += a.blocks * kRows * groups)
      move_rows<C>(a, p, to, d + threadIdx.x / C, groups, count, key_of);
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

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

constexpr int64_t kPart = 4096;  // keys that a workgroup counts

// The parts that a request's keys are counted in; 0 where they are not.
int32_t parts_of(const ws_kv_cache &c, const ws_kv_eviction &e) {
  const int64_t longest = std::min<int64_t>(e.max_kv_len, (int64_t)e.table_cols * c.page_size);
  return longest <= 64 * kHeld ? 0 : (int32_t)ceil_div(longest, kPart);
}
int64_t bytes_of(const ws_kv_cache &c, const ws_kv_eviction &e) {
  return (int64_t)e.n_seq * c.kv_heads * parts_of(c, e) * (4 * 256 * 4 + (int64_t)sizeof(Found));
}

int check_eviction(const ws_kv_cache *c, const ws_kv_eviction *e) {
  if (int rc = check_cache(c)) return rc;
  if (!e) return invalid("evict: the eviction must be non-NULL");
  if (e->n_seq < 0 || e->table_cols < 0 || e->table_stride < 0) return invalid("evict: bad sizes");
  if (e->keep < 1) return invalid("evict: at least one key must be kept");
  if (e->recent < 0 || e->recent > e->keep) return invalid("evict: recent must be 0 to keep");
  if (e->max_kv_len < 0) return invalid("evict: bad length bound");
  if ((int64_t)e->table_cols * c->page_size >= (int64_t)1 << 30 || e->keep >= 1 << 30)
    return ws_record_failure(WS_EUNSUPPORTED, "evict: 2^30 keys a request or more");
  if (e->to && (e->to_stride < 0 || (int64_t)e->to_cols * c->page_size < e->keep))
    return invalid("evict: the kept rows need pages to go to");
  return WS_OK;
}

template <int C>
int evict_launch(Args a, int64_t pairs, hipStream_t stream) {
  auto fits = [](int64_t blocks) { return blocks * 256 < (int64_t)1 << 32; };
  auto many = [] { return ws_record_failure(WS_EUNSUPPORTED, "evict: too many workgroups"); };
  const int64_t blocks = ceil_div(a.keep, 256 / C * kRows);
  if (a.parts) {
    if (!fits(pairs * a.parts) || !fits(pairs * blocks)) return many();
    for (int digit = 0; digit <= 4; ++digit)
      count_kernel<<<dim3((uint32_t)(pairs * a.parts)), 256, 0, stream>>>(a, digit);
    if (int rc = launched()) return rc;
    if (a.to) {
      a.blocks = (int32_t)blocks;
      move_kernel<C><<<dim3((uint32_t)(pairs * blocks)), 256, 0, stream>>>(a);
    }
  } else {
    // as many as fill the card, if there are rows for them
    a.blocks = a.to ? (int32_t)std::min(blocks, ceil_div(1024, pairs)) : 1;
    if (!fits(pairs * a.blocks)) return many();
    if (a.to)
      pick_kernel<C><<<dim3((uint32_t)(pairs * a.blocks)), 256, 0, stream>>>(a);
    else
      pick_kernel<0><<<dim3((uint32_t)pairs), 256, 0, stream>>>(a);
  }
  if (int rc = launched()) return rc;
  if (!a.to) {
    if (!fits(pairs * 2)) return many();
    close_up_kernel<C><<<dim3((uint32_t)(pairs * 2)), 256, 0, stream>>>(a);
    return launched();
  }
  return WS_OK;
}

}  // namespace

extern "C" {

int wait_kv_evict_workspace_bytes(const ws_kv_cache *cache, const ws_kv_eviction *eviction,
                                  size_t *bytes) {
  return guarded([&]() -> int {
    if (!bytes) return invalid("bytes must be non-NULL");
    if (int rc = check_eviction(cache, eviction)) return rc;
    *bytes = (size_t)bytes_of(*cache, *eviction);
    return WS_OK;
  });
}

int wait_kv_evict(const ws_kv_cache *cache, const ws_kv_eviction *eviction, float *weights,
                  int32_t *kept, int32_t *new_lens, void *d_workspace, size_t ws_bytes,
                  void *hip_stream) {
  return guarded([&]() -> int {
    if (int rc = check_eviction(cache, eviction)) return rc;
    const ws_kv_eviction &e = *eviction;
    if (e.n_seq == 0) return WS_OK;
    if (!e.kv_lens || !weights || !kept || !new_lens || (e.table_cols > 0 && !e.table))
      return invalid("evict: the page table, lengths, weights and outputs must be non-NULL");
    if ((uintptr_t)e.table % 4 || (uintptr_t)e.to % 4 || (uintptr_t)e.kv_lens % 4 ||
        (uintptr_t)weights % 4 || (uintptr_t)kept % 4 || (uintptr_t)new_lens % 4)
      return invalid("evict: tables, lengths, weights and outputs must be aligned to 4 bytes");
    const int64_t pairs = (int64_t)e.n_seq * cache->kv_heads;
    if (e.kv_lens < new_lens + e.n_seq && new_lens < e.kv_lens + e.n_seq)
      return invalid("evict: the new lengths need memory of their own");
    const int64_t bytes = bytes_of(*cache, e);
    if (bytes && (!d_workspace || ws_bytes < (size_t)bytes))
      return ws_record_failure(WS_EWORKSPACE, "evict: the workspace is too small");
    if ((uintptr_t)d_workspace % 16) return invalid("evict: the workspace must be 16-byte aligned");
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
    a.parts = parts_of(*cache, e);
    a.blocks = 1;
    if (bytes) {
      a.found = (Found *)d_workspace;
      a.counts = (int32_t *)(a.found + pairs * a.parts);
    }
    hipStream_t s = (hipStream_t)hip_stream;
    switch (cache->dim * type_bytes(cache->type) / 16) {
      case 4: return evict_launch<4>(a, pairs, s);
      case 8: return evict_launch<8>(a, pairs, s);
      case 16: return evict_launch<16>(a, pairs, s);
      default: return evict_launch<32>(a, pairs, s);
    }
  });
}

}  // extern "C"

// Eviction from a cache by accumulated weights: the kept keys of each request and
// KV head are found, then their rows move.
//
// Weights are compared as whole numbers of the same order.  Up to 2048 keys, a
// workgroup holds them in registers and narrows the range that the smallest kept
// one lies in until as many are above as may stay.  More keys are split over
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
  uint32_t *orders;  // [request][KV head][part][kPart]: the weights as whole numbers; or NULL
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
    const uint32_t x = order_of(a.weights[max(row, 0)]);  // without a branch, which would wait
    return row == kNoRow ? 0u : x;
  }
};

// ----------------------------------------------------- a workgroup ------
//
// Four waves hold up to 4096 keys: lane l of wave w the keys w 64 R + 64 i + l, R at
// most 16, in registers.

constexpr int kCopies = 4;  // of the counts, one a wave

struct Shared {
  int32_t count[kCopies][256];
  int32_t among[2][4][4];  // [turn][wave]
  uint32_t digit;
  int32_t left;
};

template <int R>
struct Held {
  uint32_t x[R];
  // The keys from .. to - 1, of up to 256 R; what lies behind them is 0.
  template <class F>
  __device__ __forceinline__ void load(int32_t from, int32_t to, F &&order) {
#pragma unroll
    for (int i = 0; i < R; ++i) x[i] = order(min(from + key(i), to - 1));
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (from + key(i) >= to) x[i] = 0;
  }
  // Those that an earlier launch left, and what lies behind them.
  __device__ __forceinline__ void load_left(const uint32_t *p) {
#pragma unroll
    for (int i = 0; i < R; ++i) x[i] = p[key(i)];
  }
  __device__ __forceinline__ void leave(uint32_t *p) const {
#pragma unroll
    for (int i = 0; i < R; ++i) p[key(i)] = x[i];
  }
  static __device__ __forceinline__ int32_t key(int i) {
    return (threadIdx.x >> 6) * 64 * R + 64 * i + (threadIdx.x & 63);
  }
};

// Writes the kept ones of keys from .. to - 1 behind kept[0 .. at - 1]: larger than
// `least`, or among the first `left` that equal it.  at and left are then what the
// keys behind find.
template <int R>
__device__ __forceinline__ void write_kept(Shared &sh, const Held<R> &k, int32_t from, int32_t to,
                                           uint32_t least, int32_t *left, int32_t *at,
                                           int32_t *kept) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int32_t more = 0, same = 0;
  auto there = [&](int i) { return from + k.key(i) < to; };
#pragma unroll
  for (int i = 0; i < R; ++i) {
    more += (int32_t)__popcll(__ballot(there(i) && k.x[i] > least));
    same += (int32_t)__popcll(__ballot(there(i) && k.x[i] == least));
  }
  __syncthreads();
  if (lane == 0) {
    sh.among[0][wave][0] = more;
    sh.among[0][wave][1] = same;
  }
  __syncthreads();
  int32_t my_left = *left, my_at = *at, all_more = 0, all_same = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w == wave) {
      my_at += all_more + min(all_same, *left);
      my_left = max(0, *left - all_same);
    }
    all_more += sh.among[0][w][0];
    all_same += sh.among[0][w][1];
  }
  *at += all_more + min(all_same, *left);
  *left = max(0, *left - all_same);
  const uint64_t below = (1ull << lane) - 1;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const uint64_t ties = __ballot(there(i) && k.x[i] == least);
    const bool stays = there(i) && (k.x[i] > least || (k.x[i] == least &&
                                                       (int32_t)__popcll(ties & below) < my_left));
    my_left = max(0, my_left - (int32_t)__popcll(ties));
    const uint64_t all = __ballot(stays);
    if (stays) kept[my_at + (int32_t)__popcll(all & below)] = from + k.key(i);
    my_at += (int32_t)__popcll(all);
  }
}

// The kept ones of n <= 256 R keys, 0 < need < n.  More than `need` numbers are lo
// or more, up to that many are above hi: the smallest kept one is in lo .. hi, of
// which each turn leaves a quarter.
template <int R, class F>
__device__ __forceinline__ void pick_held(Shared &sh, int32_t n, int32_t need, F &&order,
                                          int32_t *kept) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Held<R> k;
  k.load(0, n, order);
  uint32_t lo = 0, hi = 0xffffffffu;
  int32_t left = need;  // of those that equal hi, once that is lo
  for (int turn = 0; lo < hi && left > 0; turn ^= 1) {
    const uint32_t quarter = (hi - lo) / 4;
    uint32_t mid[3];  // lo < mid <= hi
    int32_t c[3] = {0, 0, 0};
#pragma unroll
    for (int m = 0; m < 3; ++m) {
      mid[m] = lo + 1 + (m + 1) * quarter;
#pragma unroll
      for (int i = 0; i < R; ++i) c[m] += (int32_t)__popcll(__ballot(k.x[i] >= mid[m]));
    }
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int m = 0; m < 3; ++m) sh.among[turn][wave][m] = c[m];
    }
    __syncthreads();
#pragma unroll
    for (int m = 0; m < 3; ++m)
      c[m] = __builtin_amdgcn_readfirstlane(sh.among[turn][0][m] + sh.among[turn][1][m] +
                                            sh.among[turn][2][m] + sh.among[turn][3][m]);
#pragma unroll
    for (int m = 2; m >= 0; --m)
      if (c[m] <= need) {
        hi = mid[m] - 1;
        left = need - c[m];
      }
#pragma unroll
    for (int m = 0; m < 3; ++m)
      if (c[m] > need) lo = mid[m];
  }
  int32_t at = 0;
  write_kept(sh, k, 0, n, hi, &left, &at, kept);
}
template <class F>
__device__ __forceinline__ void pick_held(Shared &sh, int32_t n, int32_t need, F &&order,
                                          int32_t *kept) {
  if (n <= 512)
    pick_held<2>(sh, n, need, order, kept);
  else if (n <= 1024)
    pick_held<4>(sh, n, need, order, kept);
  else if (n <= 1536)
    pick_held<6>(sh, n, need, order, kept);
  else
    pick_held<8>(sh, n, need, order, kept);
}

constexpr int kHeld = 2048;  // keys of pick_held, at most
constexpr int kPart = 4096;  // keys that are counted at a time

// Of the counts of 256 digits, the digit that the left-th largest has, and how many
// of those with it stay: sh.digit, sh.left.
__device__ __forceinline__ void find_digit(Shared &sh, int32_t left) {
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

// Adds to the counts of a digit those of the keys that share the
// digits above it.
__device__ __forceinline__ void count_held(Shared &sh, const Held<16> &k, int32_t from, int32_t to,
                                           uint32_t least, int shift) {
  const int copy = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (from + k.key(i) < to && (shift == 24 || (k.x[i] ^ least) >> (shift + 8) == 0))
      atomicAdd(&sh.count[copy][k.x[i] >> shift & 255], 1);
}
__device__ __forceinline__ void clear_counts(Shared &sh) {
  for (int i = threadIdx.x; i < 256 * kCopies; i += 256) sh.count[0][i] = 0;
  __syncthreads();
}
// All of them in the first array.
__device__ __forceinline__ void add_counts(Shared &sh) {
  __syncthreads();
  const int t = threadIdx.x;
  int32_t sum = 0;
#pragma unroll
  for (int i = 0; i < kCopies; ++i) sum += sh.count[i][t];
  sh.count[0][t] = sum;
  __syncthreads();
}

// The kept ones of a request longer than its launch was laid out for, by one
// workgroup.
template <class F>
__device__ __forceinline__ void pick_any(Shared &sh, int32_t n, int32_t need, F &&order,
                                         int32_t *kept) {
  uint32_t least = 0;
  int32_t left = need, at = 0;
  Held<16> k;
  for (int shift = 24; shift >= 0; shift -= 8) {
    clear_counts(sh);
    for (int32_t from = 0; from < n; from += kPart) {
      k.load(from, n, order);
      count_held(sh, k, from, n, least, shift);
    }
    add_counts(sh);
    find_digit(sh, left);
    least |= sh.digit << shift;
    left = sh.left;
    __syncthreads();
  }
  for (int32_t from = 0; from < n; from += kPart) {
    k.load(from, n, order);
    write_kept(sh, k, from, n, least, &left, &at, kept);
  }
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
__device__ __forceinline__ Found next_digit(Shared &sh, const Args &a, int32_t pair, int32_t part,
                                            int digit, Found f, int32_t *equal) {
  const int t = threadIdx.x;
  const int32_t *c = a.counts + (((int64_t)digit * (gridDim.x / a.parts) + pair) * a.parts) * 256 + t;
  int32_t all = 0, before = 0;
#pragma unroll 16
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
  if ((t & 63) == 0) sh.among[0][t >> 6][0] = above;
  __syncthreads();
  f.above += sh.among[0][0][0] + sh.among[0][1][0] + sh.among[0][2][0] + sh.among[0][3][0];
  f.least |= d << (24 - 8 * digit);
  f.left = sh.left;
  *equal = sh.count[1][d];
  __syncthreads();
  return f;
}

// Launch number `digit` counts that digit, once the ones before are known; the one
// behind the last digit writes the kept keys.  131,072 keys of 8 heads: five
// launches of 6 to 8 us, each a chain of loads, counts and barriers; by one
// workgroup a head 310 us.
__global__ void __launch_bounds__(256) count_kernel(Args a, int digit) {
  __shared__ Shared sh;
  const int32_t part = blockIdx.x % a.parts, pair = blockIdx.x / a.parts;
  // asked for before anything is known; the first launch leaves the numbers where
  // they need no page table, if there is room
  const bool room = a.orders != nullptr;
  uint32_t *left_here = a.orders + (room ? (int64_t)blockIdx.x * kPart : 0);
  Held<16> k;
  if (digit > 0 && room) k.load_left(left_here);
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
  const Range r = part_of(a, part, p.n);
  auto order = [&](int32_t j) { return p.order(a, j); };
  const bool whole = room && r.hi - r.lo <= kPart;  // the numbers of all of its keys
  if (r.lo < r.hi && (digit == 0 || !whole)) {
    k.load(r.lo, min(r.hi, r.lo + kPart), order);
    if (digit == 0 && whole) k.leave(left_here);
  }
  Found f = {0, p.need, 0, 0};
  int32_t equal = 0;
  if (digit > 0) {
    if (digit > 1) f = a.found[blockIdx.x];
    f = next_digit(sh, a, pair, part, digit - 1, f, &equal);
  }
  if (digit < 4) {
    if (digit > 0 && threadIdx.x == 0) a.found[blockIdx.x] = f;
    clear_counts(sh);
    for (int32_t from = r.lo; from < r.hi; from += kPart) {
      const int32_t to = min(r.hi, from + kPart);
      if (from > r.lo) k.load(from, to, order);
      count_held(sh, k, from, to, f.least, 24 - 8 * digit);
    }
    add_counts(sh);
    a.counts[((int64_t)digit * gridDim.x + blockIdx.x) * 256 + threadIdx.x] =
        sh.count[0][threadIdx.x];
    return;
  }
  int32_t left = max(0, f.left - equal), at = f.above + min(equal, f.left);
  for (int32_t from = r.lo; from < r.hi; from += kPart) {
    const int32_t to = min(r.hi, from + kPart);
    if (from > r.lo) k.load(from, to, order);
    write_kept(sh, k, from, to, f.least, &left, &at, kept);
  }
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
  if (count <= 0) return;
  // all without branches, in which each load would be waited for
  int32_t from[kRows], at[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int32_t d = min(d0 + i * step, count - 1);
    from[i] = row_of(a, p.pages, p.h, key_of(d));
    at[i] = row_of(a, to, p.h, d);
  }
  u32x4 x[kRows], y[kRows];
  float s[kRows], t[kRows], w[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    if (d0 + i * step >= count || from[i] == kNoRow) at[i] = kNoRow;
    const int32_t row = max(from[i], 0);
    x[i] = *reinterpret_cast<const u32x4 *>(a.k + ((int64_t)row * C + lane) * 16);
    y[i] = *reinterpret_cast<const u32x4 *>(a.v + ((int64_t)row * C + lane) * 16);
    w[i] = a.weights[row];
    if (a.ks) {
      s[i] = a.ks[row];
      t[i] = a.vs[row];
    }
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    if (at[i] == kNoRow) continue;
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
// for itself, which takes less than another launch.  One request of 777 keys to 512,
// 32 heads of 128 bf16: 9.6 us, against 8.0 and 5.3 in two launches; 128 requests of
// 513 to 1512 keys to 512, fp8 (1.14 GB moved), 268 us (4.3 TB/s).
template <int C>
__global__ void __launch_bounds__(256) pick_kernel(Args a) {
  __shared__ Shared sh;
  __shared__ int32_t list[kHeld];
  const int32_t pair = blockIdx.x / a.blocks, block = blockIdx.x % a.blocks;
  const Pair p(a, pair);
  int32_t *kept = a.kept + (int64_t)pair * a.keep;
  if (p.h == 0 && block == 0 && threadIdx.x == 0) a.new_lens[pair / a.kv_heads] = min(p.m, a.keep);
  const bool simple = p.simple(a), held = p.n <= kHeld;
  auto order = [&](int32_t j) { return p.order(a, j); };
  if (!simple) {
    if (!held)  // the same list by each of the workgroups
      pick_any(sh, p.n, p.need, order, kept);
    else
      pick_held(sh, p.n, p.need, order, list);
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

// Rows within a request's own pages: one workgroup takes W of the C 16-byte columns
// of the keys, or of the values, of a request and head from the front on.  A row
// never goes behind its place, so what a step writes lies before what later steps
// read; within a step everything is read before anything is written.  Columns do
// not meet, so that few requests can have a workgroup for each four of them: one of
// 131,072 keys to 16,384, 8 heads of 128 bf16, takes 155 us, 474 with whole rows.
template <int C, int W>
__global__ void __launch_bounds__(256) close_up_kernel(Args a) {
  constexpr int groups = 256 / W, step = groups * kRows;
  const int32_t slice = blockIdx.x % (C / W), id = blockIdx.x / (C / W);
  const int lane = slice * W + threadIdx.x % W;
  const bool values = id & 1;
  const int32_t pair = id / 2;
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
      const int32_t d = min(d0 + i * groups + (int32_t)threadIdx.x / W, last);
      from[i] = row_of(a, pages, h, kept[d]);
      at[i] = row_of(a, pages, h, d);
    }
    u32x4 x[kRows];
    float s[kRows], w[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      if (d0 + i * groups + (int32_t)threadIdx.x / W > last || from[i] == kNoRow) at[i] = kNoRow;
      const int32_t row = max(from[i], 0);
      x[i] = *reinterpret_cast<const u32x4 *>(rows + ((int64_t)row * C + lane) * 16);
      s[i] = scales ? scales[row] : 0.0f;
      w[i] = weights ? weights[row] : 0.0f;
    }
    // all of it has arrived, in every wave, before any of it is overwritten
#pragma unroll
    for (int i = 0; i < kRows; ++i) asm volatile("" : "+v"(x[i]), "+v"(s[i]), "+v"(w[i])::"memory");
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      if (at[i] == kNoRow) continue;
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

// How the keys are counted.
struct Layout {
  int32_t parts;  // of a request's keys; 0 where they are not counted
  bool orders;    // their numbers are kept
  int64_t bytes;
};
constexpr int64_t kMost = (int64_t)256 << 20;  // bytes of workspace

// A part has 4096 keys, unless their counts would take more than 256 MB: then there
// are fewer and longer ones, or a workgroup alone finds a request's and head's keys.
// The numbers are kept where they fit beside the counts: 64 requests of 32,768 keys,
// 32 heads of 64 fp8, 1028 us with them (336 MB), 1090 without; 128 of 131,072, 8
// heads, 1196 (840 MB) and 1378.
Layout layout_of(const ws_kv_cache &c, const ws_kv_eviction &e) {
  Layout L{};
  const int64_t longest = std::min<int64_t>(e.max_kv_len, (int64_t)e.table_cols * c.page_size);
  const int64_t pairs = (int64_t)e.n_seq * c.kv_heads;
  if (longest <= kHeld || e.keep == e.recent || pairs == 0) return L;
  const int64_t counts = pairs * (4 * 256 * 4 + (int64_t)sizeof(Found)), orders = pairs * kPart * 4;
  const int64_t parts = ceil_div(longest, kPart);
  L.orders = parts <= kMost / (counts + orders);
  L.parts = (int32_t)std::min(parts, kMost / counts);
  L.bytes = L.parts * (counts + (L.orders ? orders : 0));
  return L;
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
  if ((int64_t)e->n_seq * c->kv_heads >= (int64_t)1 << 24)  // a workgroup each
    return ws_record_failure(WS_EUNSUPPORTED, "evict: 2^24 requests times heads or more");
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
    // whole rows where there are two workgroups a CU of them
    if (pairs * 2 >= 512)
      close_up_kernel<C, C><<<dim3((uint32_t)(pairs * 2)), 256, 0, stream>>>(a);
    else
      close_up_kernel<C, 4><<<dim3((uint32_t)(pairs * 2 * (C / 4))), 256, 0, stream>>>(a);
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
    *bytes = (size_t)layout_of(*cache, *eviction).bytes;
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
    const Layout L = layout_of(*cache, e);
    const int64_t bytes = L.bytes;
    if (bytes && (!d_workspace || ws_bytes < (size_t)bytes))
      return ws_record_failure(WS_EWORKSPACE, "evict: the workspace is too small");
    if ((uintptr_t)d_workspace % 16) return invalid("evict: the workspace must be 16-byte aligned");
    const CacheSpans in_cache(*cache);
    const Span w = span(weights, (__int128)cache->pages * cache->kv_heads * cache->page_size * 4);
    const Span list = span(kept, (__int128)pairs * e.keep * 4), lens = span(new_lens, (__int128)e.n_seq * 4);
    const Span space = span(d_workspace, bytes);
    const Span read[3] = {table_span(e.table, e.n_seq, e.table_stride, e.table_cols),
                          table_span(e.to, e.n_seq, e.to_stride, e.to_cols),
                          span(e.kv_lens, (__int128)e.n_seq * 4)};
    for (const Span &in : read)
      if (shares(in, in_cache) || shares(in, {w, list, lens}))
        return invalid("evict: weights, outputs and cache must not overlap the lengths or the pages");
    if (shares(w, in_cache) || shares(list, in_cache) || shares(lens, in_cache) || shares(w, {list, lens}) ||
        shares(list, lens))
      return invalid("evict: weights and outputs must not overlap the cache or one another");
    if (shares(space, in_cache) || shares(space, {w, list, lens, read[0], read[1], read[2]}))
      return invalid("evict: the workspace must be its own memory");
    if (e.to && e.to == e.table) return invalid("evict: the requests' own pages are no others: leave `to` out");
    if (!e.to && (shares(in_cache.k, in_cache.v) || shares(in_cache.ks, in_cache.vs)))
      return invalid("evict: keys and values that move in place must not overlap");
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
    a.parts = L.parts;
    a.blocks = 1;
    if (bytes) {
      a.found = (Found *)d_workspace;
      a.counts = (int32_t *)(a.found + pairs * a.parts);
      if (L.orders) a.orders = (uint32_t *)(a.counts + pairs * a.parts * 4 * 256);
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

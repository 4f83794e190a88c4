// Norms of queries and keys with the rotation in the same pass, and a batch's
// rows on their way into a layer: one pass over the data each, bound by memory.
//
// y = x r w with r = (mean x^2 + eps)^(-1/2), then pairs of y turned.  A group of
// lanes holds a whole vector: each lane two chunks of VEC elements, which are
// partners in the rotation, so that norm and rotation need no more than one sum
// over the lanes; an 8-bit cache takes one more, the row's largest magnitude.
#include <algorithm>
#include <type_traits>

#include "kv_rows.h"
#include "wait_kv_norm.h"

namespace {

using namespace kv;

// One kind of row: queries, keys or values.
struct Side {
  const void *x;
  int64_t xt, xh;
  const void *w;  // NULL: ones
  int64_t wh;
  int32_t w_type, normed;
  float eps;
};

struct Args {
  Side q, k, v;
  void *out;  // of the queries
  int64_t ot, oh;
  void *ck, *cv;
  float *ks, *vs;
  const int64_t *slots;
  int64_t n, n_slots;
  int32_t heads, kv_heads, dim, page_shift;
  int32_t q_groups, kv_groups;  // groups of HPT heads
  int32_t lane_bits;            // a vector takes 2^lane_bits lanes,
  int32_t items;                // so many of which have chunks
  int32_t interleaved;
  TurnArgs turn;
};

constexpr int kNone = -1;  // no cache: queries alone

template <class T>
constexpr int kWide = 16 / sizeof(typename T::raw);  // elements of 16 bytes

// VEC weights from element d of head h on.
template <int VEC>
__device__ __forceinline__ void load_weights(const Side &s, int32_t h, int32_t d, float (&w)[VEC]) {
  const int64_t at = h * s.wh + d;
  if (!s.w) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) w[i] = 1.0f;
  } else if (s.w_type == WS_KV_FP32) {
    load_n<Fp32, VEC, (VEC < 4 ? VEC : 4)>((const uint32_t *)s.w + at, w);
  } else if (s.w_type == WS_KV_BF16) {
    load_n<Bf16, VEC, VEC>((const uint16_t *)s.w + at, w);
  } else {
    load_n<Fp16, VEC, VEC>((const uint16_t *)s.w + at, w);
  }
}

// Weights asked for and not yet waited for: VEC of 32 bits, or of 16 in the first
// half of the words.  (As vectors: arrays end in memory here.)
template <int VEC>
struct AskedWeights {
  u32x4 a, b;
  __device__ __forceinline__ AskedWeights(const void *w, int64_t at, bool wide) {
    const uint32_t *p = (const uint32_t *)w + at;
    const uint16_t *q = (const uint16_t *)w + at;
    a = b = u32x4{0, 0, 0, 0};
    if constexpr (VEC == 8) {
      a = *reinterpret_cast<const u32x4 *>(wide ? (const void *)p : q);
      if (wide) b = *reinterpret_cast<const u32x4 *>(p + 4);
    } else if constexpr (VEC == 4) {
      if (wide) {
        a = *reinterpret_cast<const u32x4 *>(p);
      } else {
        const u32x2 x = *reinterpret_cast<const u32x2 *>(q);
        a = u32x4{x[0], x[1], 0, 0};
      }
    } else {
      if (wide) {
        const u32x2 x = *reinterpret_cast<const u32x2 *>(p);
        a = u32x4{x[0], x[1], 0, 0};
      } else {
        a[0] = *reinterpret_cast<const uint32_t *>(q);
      }
    }
  }
  __device__ __forceinline__ void get(int type, float (&w)[VEC]) const {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const uint32_t full = i < 4 ? a[i & 3] : b[i & 3];
      const uint16_t half = (uint16_t)(a[i / 2] >> (16 * (i & 1)));
      const float x = type == WS_KV_BF16 ? Bf16::get(half) : Fp16::get(half);
      w[i] = type == WS_KV_FP32 ? __uint_as_float(full) : x;
    }
  }
};

// f over the lanes of a group, up to 16 without leaving the registers: neighbours,
// pairs, then mirrored halves, whose lanes hold the same by then.
template <class F>
__device__ __forceinline__ uint32_t over_lanes(uint32_t x, int lanes, F &&f) {
  auto with = [&](auto control) {
    x = f(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, decltype(control)::value, 0xf, 0xf, true));
  };
  if (lanes > 1) with(std::integral_constant<int, 0xb1>{});    // 1 0 3 2
  if (lanes > 2) with(std::integral_constant<int, 0x4e>{});    // 2 3 0 1
  if (lanes > 4) with(std::integral_constant<int, 0x141>{});   // 7 .. 0
  if (lanes > 8) with(std::integral_constant<int, 0x140>{});   // 15 .. 0
  for (int m = 16; m < lanes; m *= 2) x = f(x, (uint32_t)__shfl_xor((int)x, m));
  return x;
}
__device__ __forceinline__ float sum_over(float x, int lanes) {
  return __uint_as_float(over_lanes(__float_as_uint(x), lanes, [](uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}
__device__ __forceinline__ uint32_t max_over(uint32_t x, int lanes) {
  return over_lanes(x, lanes, [](uint32_t a, uint32_t b) { return max(a, b); });
}

// Of a pair of chunks.
template <int VEC>
struct Pair {
  float u[VEC], w[VEC];
};

// HPT heads of a token for each group of lanes.  Everything is asked for before the
// first use of any of it, the position first, which the angles wait for.
//
// Bound by memory: 8192 x 32 vectors of 128 bf16 (138 MB) 22.5 us (6.2 TB/s), where
// the rotation alone takes 21.5; weights turned into floats as they were asked for
// made that 27, since the angles were asked for behind them.  Four heads a thread
// share angles and weights once there is enough for that: one 41 us, two 30, eight
// 24.  8191 tokens of 32 + 2 x 8 heads, fp16 into int8 (185 MB), 33.6 us (5.5 TB/s);
// with all kinds of rows in a wave 45.
template <class T, int TYPE, int VEC, bool INTER, int HPT, bool STREAM>
__global__ void __launch_bounds__(256) norm_kernel(Args a) {
  using raw = typename T::raw;
  constexpr int acc = VEC < kWide<T> ? VEC : kWide<T>;
  const int lanes = 1 << a.lane_bits, lane = threadIdx.x & (lanes - 1);
  const uint32_t id = blockIdx.x * (256u >> a.lane_bits) + (threadIdx.x >> a.lane_bits);
  // all queries, then all keys, then all values: a wave has rows of one kind
  const uint32_t queries = (uint32_t)a.n * (uint32_t)a.q_groups;
  const uint32_t keys = TYPE == kNone ? 0 : (uint32_t)a.n * (uint32_t)a.kv_groups;
  if (id >= queries + 2 * keys) return;  // the lanes of a group end together
  const bool is_k = TYPE != kNone && id >= queries && id < queries + keys;
  const bool is_v = TYPE != kNone && id >= queries + keys;
  const uint32_t nth = id - (is_v ? queries + keys : is_k ? queries : 0);
  const uint32_t groups = is_k || is_v ? a.kv_groups : a.q_groups;
  const uint32_t token = nth / groups;
  const int32_t unit = (int32_t)(nth - token * groups);
  Side s = a.q;  // by value: the arguments are not read through a pointer
  if (is_k) s = a.k;
  if (is_v) s = a.v;
  const int32_t heads = is_k || is_v ? a.kv_heads : a.heads;
  const int32_t h0 = unit * HPT;
  const int32_t part = a.turn.part, half = part / 2;
  const bool live = lane < a.items;
  const int32_t item = min(lane, a.items - 1);
  // the two chunks, and whether they are turned
  const int32_t turned = half / VEC;
  int32_t d0, d1;
  bool turn0, turn1;
  if (INTER || item >= turned) {
    d0 = INTER ? item * 2 * VEC : part + (item - turned) * 2 * VEC;
    d1 = d0 + VEC;
    turn0 = INTER && d0 < part;
    turn1 = INTER && d1 < part;
  } else {
    d0 = item * VEC;
    d1 = half + d0;
    turn0 = turn1 = true;
  }
  if (is_v) turn0 = turn1 = false;

  Position position = {};
  if (part) position = ask_position(a.turn, token);
  int64_t slot = 0;
  if constexpr (TYPE != kNone) slot = a.slots[token];
  raw x0[HPT][VEC], x1[HPT][VEC];
  const raw *x = (const raw *)s.x + (int64_t)token * s.xt;
#pragma unroll
  for (int i = 0; i < HPT; ++i) {
    const int32_t h = min(h0 + i, heads - 1);
    load_raw<T, VEC, acc>(x + h * s.xh + d0, x0[i]);
    load_raw<T, VEC, acc>(x + h * s.xh + d1, x1[i]);
  }
  // (of a side without weights something that is there, and is not used)
  const void *weights = s.w ? s.w : s.x;
  const bool wide = s.w && s.w_type == WS_KV_FP32;
  const AskedWeights<VEC> w0(weights, s.w ? h0 * s.wh + d0 : 0, wide);
  const AskedWeights<VEC> w1(weights, s.w ? h0 * s.wh + d1 : 0, wide);
  all_asked(position);
  // angles of the chunks: the same ones where they are partners
  constexpr int NC = INTER ? (VEC + 1) / 2 : VEC;
  float c0[NC], s0[NC], c1[INTER ? NC : 1], s1[INTER ? NC : 1];
  const float *row = turn0 ? turn_row(a.turn, position) : nullptr;
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    c0[i] = s0[i] = NAN;
    if constexpr (INTER) c1[i] = s1[i] = NAN;
  }
  if (row) {
    const float *p = row + (INTER ? d0 / 2 : d0);
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      c0[i] = p[i];
      s0[i] = p[half + i];
    }
    if (INTER && turn1) {
      p = row + d1 / 2;
#pragma unroll
      for (int i = 0; i < (INTER ? NC : 1); ++i) {
        c1[i] = p[i];
        s1[i] = p[half + i];
      }
    }
  }
  const bool stored = TYPE == kNone || !(is_k || is_v) || (slot >= 0 && slot < a.n_slots);
  if (!stored) return;
  // the heads' sums, one beside the other
  float r[HPT];
  Pair<VEC> w;
  if (s.normed) {
#pragma unroll
    for (int i = 0; i < HPT; ++i) {
      float sum = 0.0f;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float u = T::get(x0[i][e]), v = T::get(x1[i][e]);
        sum = __builtin_fmaf(u, u, sum);
        sum = __builtin_fmaf(v, v, sum);
      }
      r[i] = live ? sum : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < HPT; ++i) r[i] = sum_over(r[i], lanes);
#pragma unroll
    for (int i = 0; i < HPT; ++i) r[i] = rsqrtf(r[i] / (float)a.dim + s.eps);
    w0.get(s.w_type, w.u);
    w1.get(s.w_type, w.w);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      w.u[e] = s.w ? w.u[e] : 1.0f;
      w.w[e] = s.w ? w.w[e] : 1.0f;
    }
  }
#pragma unroll
  for (int i = 0; i < HPT; ++i) {
    const int32_t h = h0 + i;
    Pair<VEC> y;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      y.u[e] = T::get(x0[i][e]);
      y.w[e] = T::get(x1[i][e]);
    }
    if (s.normed) {
      if (i > 0 && s.wh) {
        load_weights<VEC>(s, min(h, heads - 1), d0, w.u);
        load_weights<VEC>(s, min(h, heads - 1), d1, w.w);
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        y.u[e] = y.u[e] * r[i] * w.u[e];
        y.w[e] = y.w[e] * r[i] * w.w[e];
      }
    }
    if constexpr (INTER) {
      if (turn0) {
#pragma unroll
        for (int e = 0; e < VEC / 2; ++e) {
          const float p = y.u[2 * e], q = y.u[2 * e + 1];
          y.u[2 * e] = p * c0[e] - q * s0[e];
          y.u[2 * e + 1] = q * c0[e] + p * s0[e];
        }
      }
      if (turn1) {
#pragma unroll
        for (int e = 0; e < VEC / 2; ++e) {
          const float p = y.w[2 * e], q = y.w[2 * e + 1];
          y.w[2 * e] = p * c1[e] - q * s1[e];
          y.w[2 * e + 1] = q * c1[e] + p * s1[e];
        }
      }
    } else if (turn0) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float p = y.u[e], q = y.w[e];
        y.u[e] = p * c0[e] - q * s0[e];
        y.w[e] = q * c0[e] + p * s0[e];
      }
    }
    if (TYPE == kNone || !(is_k || is_v)) {
      if (!live || h >= heads) continue;
      raw *o = (raw *)a.out + (int64_t)token * a.ot + h * a.oh;
      store_n<T, VEC, acc, STREAM>(o + d0, y.u);
      store_n<T, VEC, acc, STREAM>(o + d1, y.w);
    } else if constexpr (TYPE != kNone) {
      if (h >= heads) continue;
      const int64_t page = slot >> a.page_shift, off = slot & ((1 << a.page_shift) - 1);
      const int64_t row = ((page * a.kv_heads + h) << a.page_shift) + off;
      void *base = is_k ? a.ck : a.cv;
      if constexpr (TYPE == WS_KV_BF16) {
        store_n<Bf16, VEC, VEC>((uint16_t *)base + row * a.dim + d0, y.u);
        store_n<Bf16, VEC, VEC>((uint16_t *)base + row * a.dim + d1, y.w);
      } else if constexpr (TYPE == WS_KV_FP16) {
        store_n<Fp16, VEC, VEC>((uint16_t *)base + row * a.dim + d0, y.u);
        store_n<Fp16, VEC, VEC>((uint16_t *)base + row * a.dim + d1, y.w);
      } else {
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < VEC; ++e) top = max(top, max(magnitude(y.u[e]), magnitude(y.w[e])));
        top = max_over(top, lanes);
        const Coding<TYPE> code(top);
        uint8_t *to = (uint8_t *)base + row * a.dim;
        *reinterpret_cast<u32x2 *>(to + d0) = code.codes(y.u);
        *reinterpret_cast<u32x2 *>(to + d1) = code.codes(y.w);
        if (lane == 0) (is_k ? a.ks : a.vs)[row] = code.scale;
      }
    }
  }
}

// Any alignment, any even part: a wave takes one vector, a lane its pairs, one at
// a time, each element in one lane only, so that out may be x.  Bound by instructions,
// an element a load and the vector read twice: 8192 x 32 vectors of 128 bf16 at odd
// addresses 109 us (22 with aligned ones), with 66 elements turned 134; 8191 tokens of
// 32 + 2 x 8 heads at odd addresses, fp16 into int8, 236 (34).
template <class T, int TYPE>
__global__ void __launch_bounds__(256) norm_single_kernel(Args a) {
  using raw = typename T::raw;
  const int lane = threadIdx.x & 63;
  const uint32_t id = blockIdx.x * 4u + (threadIdx.x >> 6);
  const uint32_t units = (uint32_t)a.heads + (TYPE == kNone ? 0 : 2 * a.kv_heads);
  const uint32_t token = id / units;
  int32_t h = (int32_t)(id - token * units);
  if (token >= a.n) return;
  bool is_k = false, is_v = false;
  if (TYPE != kNone && h >= a.heads) {
    h -= a.heads;
    is_v = h >= a.kv_heads;
    is_k = !is_v;
    if (is_v) h -= a.kv_heads;
  }
  const Side &s = is_k ? a.k : is_v ? a.v : a.q;
  const raw *x = (const raw *)s.x + (int64_t)token * s.xt + h * s.xh;
  const int32_t part = is_v ? 0 : a.turn.part, half = part / 2;
  const float *row = part ? turn_row(a.turn, ask_position(a.turn, token)) : nullptr;
  float r = 1.0f;
  if (s.normed) {
    float sum = 0.0f;
    for (int32_t d = lane; d < a.dim; d += 64) {
      const float u = T::get(x[d]);
      sum += u * u;
    }
    for (int m = 1; m < 64; m *= 2) sum += __shfl_xor(sum, m);
    r = rsqrtf(sum / (float)a.dim + s.eps);
  }
  auto value = [&](int32_t d) {
    const float u = T::get(x[d]);
    if (!s.normed) return u;
    float w[1];
    load_weights<1>(s, h, d, w);
    return u * r * w[0];
  };
  // put(d, element d of the result) for this lane's elements
  auto each = [&](auto &&put) {
    for (int32_t i = lane; i < half + a.dim - part; i += 64) {
      if (i >= half) {
        put(part + i - half, value(part + i - half));
        continue;
      }
      const int32_t d0 = a.interleaved ? 2 * i : i, d1 = a.interleaved ? d0 + 1 : i + half;
      const float c = row ? row[i] : NAN, sn = row ? row[half + i] : NAN;
      const float p = value(d0), q = value(d1);
      put(d0, p * c - q * sn);
      put(d1, q * c + p * sn);
    }
  };
  if (TYPE == kNone || !(is_k || is_v)) {
    raw *o = (raw *)a.out + (int64_t)token * a.ot + h * a.oh;
    each([&](int32_t d, float y) { o[d] = T::put(y); });
  } else if constexpr (TYPE != kNone) {
    const int64_t slot = a.slots[token];
    if (slot < 0 || slot >= a.n_slots) return;
    const int64_t page = slot >> a.page_shift, off = slot & ((1 << a.page_shift) - 1);
    const int64_t at = ((page * a.kv_heads + h) << a.page_shift) + off;
    void *base = is_k ? a.ck : a.cv;
    if constexpr (TYPE == WS_KV_BF16) {
      each([&](int32_t d, float y) { ((uint16_t *)base)[at * a.dim + d] = Bf16::put(y); });
    } else if constexpr (TYPE == WS_KV_FP16) {
      each([&](int32_t d, float y) { ((uint16_t *)base)[at * a.dim + d] = Fp16::put(y); });
    } else {
      uint32_t top = 0;
      each([&](int32_t, float y) { top = max(top, magnitude(y)); });
      for (int m = 1; m < 64; m *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, m));
      const Coding<TYPE> code(top);
      each([&](int32_t d, float y) {
        const float eight[8] = {y, y, y, y, y, y, y, y};
        ((uint8_t *)base)[at * a.dim + d] = (uint8_t)code.codes(eight)[0];
      });
      if (lane == 0) (is_k ? a.ks : a.vs)[at] = code.scale;
    }
  }
}

// -------------------------------------------------------------- host -----

template <class T>
void skip(Args &a, int64_t from) {
  for (Side *s : {&a.q, &a.k, &a.v})
    if (s->x) s->x = (const typename T::raw *)s->x + from * s->xt;
  a.out = (typename T::raw *)a.out + from * a.ot;
  if (a.slots) a.slots += from;
  skip_positions(a.turn, from);
}

template <class T, int TYPE, int VEC, bool INTER>
int launch_vec(Args a, hipStream_t stream) {
  a.items = a.dim / (2 * VEC);
  a.lane_bits = 0;
  while (1 << a.lane_bits < a.items) ++a.lane_bits;
  const bool many =
      a.n * ((int64_t)a.heads + (TYPE == kNone ? 0 : 2 * a.kv_heads)) * a.dim * (int64_t)sizeof(typename T::raw) >=
      kStreamBytes;
  const int per = many ? 4 : 1;
  a.q_groups = (a.heads + per - 1) / per;
  a.kv_groups = TYPE == kNone ? 0 : (a.kv_heads + per - 1) / per;
  const int64_t threads = ((int64_t)a.q_groups + 2 * a.kv_groups) << a.lane_bits;
  return token_ranges(a.n, threads, 1, [&](int64_t from, int64_t n) {
    Args r = a;
    r.n = n;
    skip<T>(r, from);
    const dim3 blocks((uint32_t)((n * threads + 255) / 256));
    if (many)
      norm_kernel<T, TYPE, VEC, INTER, 4, true><<<blocks, 256, 0, stream>>>(r);
    else
      norm_kernel<T, TYPE, VEC, INTER, 1, false><<<blocks, 256, 0, stream>>>(r);
  });
}

template <class T, int TYPE>
int launch_single(const Args &a, hipStream_t stream) {
  const int64_t units = (int64_t)a.heads + (TYPE == kNone ? 0 : 2 * a.kv_heads);
  return token_ranges(a.n, units * 64, 1, [&](int64_t from, int64_t n) {
    Args r = a;
    r.n = n;
    skip<T>(r, from);
    norm_single_kernel<T, TYPE><<<dim3((uint32_t)((n * units + 3) / 4)), 256, 0, stream>>>(r);
  });
}

// Whether chunks of v elements fit: in every vector's alignment (`wide` elements
// at least), in the halves, and behind them.
bool fits(const Args &a, int v, int wide, int most) {
  const int32_t part = a.turn.part;
  if ((v < most ? v : most) > wide || a.dim % (2 * v) || a.dim / (2 * v) > 64) return false;
  if (a.interleaved ? part % v : part / 2 % v || (a.dim - part) % (2 * v)) return false;
  for (const Side *s : {&a.q, &a.k}) {
    const int bytes = type_bytes(s->w_type);
    if (s->normed && s->w && ((uintptr_t)s->w % (v * bytes < 16 ? v * bytes : 16) || s->wh % v))
      return false;
  }
  return true;
}

template <class T, int TYPE, int VEC>
int launch_pairs(const Args &a, hipStream_t stream) {
  if (a.interleaved) return launch_vec<T, TYPE, VEC, true>(a, stream);
  return launch_vec<T, TYPE, VEC, false>(a, stream);
}

// The widest chunks that fit, of up to 16 bytes (a row of a cache: 8 elements).
// fp32 vectors in chunks of 8 elements took a quarter longer: 8192 x 32 of 128
// (268 MB) 52.8 us against 40.3, which the rotation alone takes too.
template <class T, int TYPE>
int launch(const Args &a, int wide, hipStream_t stream) {
  constexpr int most = kWide<T>;
  if constexpr (TYPE != kNone || most == 8)
    if (fits(a, 8, wide, most)) return launch_pairs<T, TYPE, 8>(a, stream);
  if constexpr (TYPE == kNone) {
    if (fits(a, 4, wide, most)) return launch_pairs<T, TYPE, 4>(a, stream);
    if (fits(a, 2, wide, most)) return launch_pairs<T, TYPE, 2>(a, stream);
  }
  return launch_single<T, TYPE>(a, stream);
}

int check_norm(const ws_kv_norm *n) {
  if (!n) return WS_OK;
  if (!is_wide(n->type)) return invalid("a norm's weights must be bf16, fp16 or fp32");
  if ((uintptr_t)n->weight % type_bytes(n->type)) return invalid("a norm's weights must be aligned to their type");
  if (!(n->eps >= 0.0f) || !std::isfinite(n->eps)) return invalid("a norm's eps must be finite and not negative");
  return WS_OK;
}

Side side(const ws_kv_rows &r, const ws_kv_norm *n) {
  Side s{};
  s.x = r.data;
  s.xt = r.token_stride;
  s.xh = r.head_stride;
  if (n) {
    s.normed = 1;
    s.w = n->weight;
    s.wh = n->head_stride;
    s.w_type = n->type;
    s.eps = n->eps;
  }
  return s;
}

void set_turn(Args &a, const ws_kv_turn *t) {
  if (!t) return;
  a.turn = {t->table, t->positions, t->positions_32, t->n_table, t->part};
  a.interleaved = t->interleaved != 0;
}

template <class T>
int enter_type(const Args &a, int type, int wide, hipStream_t s) {
  switch (type) {
    case WS_KV_BF16: return launch<T, WS_KV_BF16>(a, wide, s);
    case WS_KV_FP16: return launch<T, WS_KV_FP16>(a, wide, s);
    case WS_KV_FP8: return launch<T, WS_KV_FP8>(a, wide, s);
    default: return launch<T, WS_KV_INT8>(a, wide, s);
  }
}

}  // namespace

extern "C" {

int wait_kv_norm_rotary(const ws_kv_rows *x, const ws_kv_rows *out, int64_t n, int32_t heads,
                        int32_t dim, const ws_kv_norm *norm, const ws_kv_turn *turn,
                        void *hip_stream) {
  return guarded([&]() -> int {
    if (n < 0 || heads < 1 || dim < 1 || dim > 65536) return invalid("norm: bad sizes");
    if (n >= (int64_t)1 << 31) return ws_record_failure(WS_EUNSUPPORTED, "2^31 tokens or more");
    if (int rc = check_rows(x, n, "norm: x must be non-NULL")) return rc;
    if (int rc = check_rows(out, n, "norm: out must be non-NULL")) return rc;
    if (x->type != out->type) return invalid("norm: x and out must have one type");
    if (int rc = check_norm(norm)) return rc;
    if (turn)
      if (int rc = check_turn(turn, n, dim)) return rc;
    if (!one_place(*x, *out) && overlap(*x, *out, n, heads, dim))
      return invalid("norm: out must be x or not overlap it");
    if (n == 0) return WS_OK;
    Args a{};
    a.q = side(*x, norm);
    a.out = out->data;
    a.ot = out->token_stride;
    a.oh = out->head_stride;
    a.n = n;
    a.heads = heads;
    a.dim = dim;
    set_turn(a, turn);
    const int wide = widest(*x, *out);
    hipStream_t s = (hipStream_t)hip_stream;
    if (x->type == WS_KV_BF16) return launch<Bf16, kNone>(a, wide, s);
    if (x->type == WS_KV_FP16) return launch<Fp16, kNone>(a, wide, s);
    return launch<Fp32, kNone>(a, wide, s);
  });
}

int wait_kv_enter(const ws_kv_cache *cache, const ws_kv_rows *q, const ws_kv_rows *q_out,
                  int32_t heads, const ws_kv_rows *k, const ws_kv_rows *v, const int64_t *slots,
                  int64_t n, const ws_kv_norm *q_norm, const ws_kv_norm *k_norm,
                  const ws_kv_turn *turn, void *hip_stream) {
  return guarded([&]() -> int {
    if (int rc = check_cache(cache)) return rc;
    if (n < 0 || heads < 1) return invalid("enter: bad sizes");
    const int64_t rows = (int64_t)heads + 2 * (int64_t)cache->kv_heads;
    if (rows >= (int64_t)1 << 31 || n >= ((int64_t)1 << 31) / rows)
      return ws_record_failure(WS_EUNSUPPORTED, "2^31 rows or more");
    if (int rc = check_rows(q, n, "enter: q must be non-NULL")) return rc;
    if (int rc = check_rows(q_out, n, "enter: q's output must be non-NULL")) return rc;
    if (int rc = check_rows(k, n, "enter: k must be non-NULL")) return rc;
    if (int rc = check_rows(v, n, "enter: v must be non-NULL")) return rc;
    if (q->type != q_out->type || q->type != k->type || q->type != v->type)
      return invalid("enter: q, its output, k and v must have one type");
    if (n > 0 && !slots) return invalid("enter: slots must be non-NULL");
    if ((uintptr_t)slots % 8) return invalid("enter: slots must be aligned to 8 bytes");
    if (int rc = check_norm(q_norm)) return rc;
    if (int rc = check_norm(k_norm)) return rc;
    if (turn)
      if (int rc = check_turn(turn, n, cache->dim)) return rc;
    if (!one_place(*q, *q_out) && overlap(*q, *q_out, n, heads, cache->dim))
      return invalid("enter: q's output must be q or not overlap it");
    for (const ws_kv_rows *r : {k, v})
      if (overlap(*q_out, *r, n, heads, cache->kv_heads, cache->dim))
        return invalid("enter: q's output must not overlap k or v");
    if (shares(span(*q_out, n, heads, cache->dim), CacheSpans(*cache)))
      return invalid("enter: q's output must not overlap the cache");
    if (n == 0) return WS_OK;
    Args a{};
    a.q = side(*q, q_norm);
    a.k = side(*k, k_norm);
    a.v = side(*v, nullptr);
    a.out = q_out->data;
    a.ot = q_out->token_stride;
    a.oh = q_out->head_stride;
    a.ck = cache->k;
    a.cv = cache->v;
    a.ks = cache->k_scale;
    a.vs = cache->v_scale;
    a.slots = slots;
    a.n = n;
    a.n_slots = (int64_t)cache->pages * cache->page_size;
    a.heads = heads;
    a.kv_heads = cache->kv_heads;
    a.dim = cache->dim;
    a.page_shift = log2_of(cache->page_size);
    set_turn(a, turn);
    const int wide = std::min(widest(*q, *q_out), widest(*k, *v));
    hipStream_t s = (hipStream_t)hip_stream;
    if (q->type == WS_KV_BF16) return enter_type<Bf16>(a, cache->type, wide, s);
    if (q->type == WS_KV_FP16) return enter_type<Fp16>(a, cache->type, wide, s);
    return enter_type<Fp32>(a, cache->type, wide, s);
  });
}

}  // extern "C"

// Rotary positions, quantised writes into a paged cache and reads from it:
// one pass over the data each, bound by memory.
#include "kv_rows.h"

namespace {

using namespace kv;

// ------------------------------------------------------------ rotary -----

struct RotaryArgs {
  const void *x;
  void *out;
  int64_t xt, xh, ot, oh;
  int64_t n;
  int32_t heads, dim, inverse;
  int32_t items;        // work items of a vector: pairs of chunks, then chunks that are copied
  int32_t turned;       // of them pairs
  int32_t head_groups;  // groups of HPT heads
  TurnArgs turn;
};

// A thread takes one work item of HPT heads of a token: VEC elements and their
// partners (INTER: VEC elements that hold VEC / 2 pairs), or VEC elements
// behind the turned part.  The angles' row is read once for the HPT heads.
// Both halves are read before either is written, so out may be x.
template <class T, int VEC, bool INTER, int HPT, bool STREAM>
__global__ void __launch_bounds__(256) rotary_kernel(RotaryArgs a) {
  using raw = typename T::raw;
  const uint32_t id = blockIdx.x * 256u + threadIdx.x;
  const uint32_t rest = id / (uint32_t)a.items;
  const int32_t item = (int32_t)(id - rest * a.items);
  const uint32_t at = rest / (uint32_t)a.head_groups;
  const int32_t h0 = (int32_t)(rest - at * a.head_groups) * HPT;
  const int64_t token = at;
  if (token >= a.n) return;
  const raw *x = (const raw *)a.x + token * a.xt;
  raw *out = (raw *)a.out + token * a.ot;
  const int32_t part = a.turn.part, half = part / 2;
  const bool copy = item >= a.turned;
  const int32_t d = copy ? part + (item - a.turned) * VEC : item * VEC;
  constexpr int NC = INTER ? (VEC + 1) / 2 : VEC;
  // the position first, which the angles wait for, then the vectors; a value is
  // used only behind the last request, because using it is waiting for it
  Position position = ask_position(a.turn, token);
  raw u0[HPT][VEC], w0[HPT][VEC];
#pragma unroll
  for (int k = 0; k < HPT; ++k) {
    const int32_t h = min(h0 + k, a.heads - 1);
    load_raw<T, VEC, VEC>(x + h * a.xh + d, u0[k]);
    if constexpr (!INTER) load_raw<T, VEC, VEC>(x + h * a.xh + (copy ? d : half + d), w0[k]);
  }
  all_asked(position);
  float c[NC], s[NC];
  if (!copy) {
    const float *row = turn_row(a.turn, position);
    const int32_t i0 = INTER ? d / 2 : d;
    if (row) {
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        c[i] = row[i0 + i];
        s[i] = a.inverse ? -row[half + i0 + i] : row[half + i0 + i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < NC; ++i) c[i] = s[i] = NAN;
    }
  }
#pragma unroll
  for (int k = 0; k < HPT; ++k) {
    const int32_t h = h0 + k;
    if (h >= a.heads) continue;
    raw *o = out + h * a.oh + d;
    float u[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) u[i] = T::get(u0[k][i]);
    if (copy) {
      store_n<T, VEC, VEC, STREAM>(o, u);
    } else if constexpr (INTER) {
      float y[VEC];
#pragma unroll
      for (int i = 0; i < VEC / 2; ++i) {
        y[2 * i] = u[2 * i] * c[i] - u[2 * i + 1] * s[i];
        y[2 * i + 1] = u[2 * i + 1] * c[i] + u[2 * i] * s[i];
      }
      store_n<T, VEC, VEC, STREAM>(o, y);
    } else {
      float y[VEC], z[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float w = T::get(w0[k][i]);
        y[i] = u[i] * c[i] - w * s[i];
        z[i] = w * c[i] + u[i] * s[i];
      }
      store_n<T, VEC, VEC, STREAM>(o, y);
      store_n<T, VEC, VEC, STREAM>(o + half, z);
    }
  }
}

template <class T, class F>
int in_ranges(const RotaryArgs &all, int64_t threads_a_token, F &&launch) {
  return token_ranges(all.n, threads_a_token, 1, [&](int64_t from, int64_t n) {
    RotaryArgs a = all;
    a.n = n;
    a.x = (const typename T::raw *)a.x + from * a.xt;
    a.out = (typename T::raw *)a.out + from * a.ot;
    skip_positions(a.turn, from);
    launch(a, (uint32_t)((n * threads_a_token + 255) / 256));
  });
}

template <class T, int VEC, bool INTER>
int rotary_launch(RotaryArgs a, hipStream_t stream) {
  const int32_t half = a.turn.part / 2;
  a.turned = INTER ? a.turn.part / VEC : half / VEC;
  a.items = a.turned + (a.dim - a.turn.part) / VEC;
  // four heads a thread share the row of angles once there are threads to spare
  const bool many = a.n * a.heads * a.dim * (int64_t)sizeof(typename T::raw) >= kStreamBytes;
  a.head_groups = many ? (a.heads + 3) / 4 : a.heads;
  return in_ranges<T>(a, (int64_t)a.head_groups * a.items, [&](const RotaryArgs &r, uint32_t blocks) {
    if (many)
      rotary_kernel<T, VEC, INTER, 4, true><<<dim3(blocks), 256, 0, stream>>>(r);
    else
      rotary_kernel<T, VEC, INTER, 1, false><<<dim3(blocks), 256, 0, stream>>>(r);
  });
}

// The widest access that alignment and the parts' sizes allow.
template <class T, bool INTER>
int rotary_vec(const RotaryArgs &a, int max_vec, hipStream_t stream) {
  const int32_t unit = INTER ? a.turn.part : a.turn.part / 2;
  auto fits = [&](int v) { return v <= max_vec && unit % v == 0 && (a.dim - a.turn.part) % v == 0; };
  if constexpr (sizeof(typename T::raw) == 2)
    if (fits(8)) return rotary_launch<T, 8, INTER>(a, stream);
  if (fits(4)) return rotary_launch<T, 4, INTER>(a, stream);
  if (fits(2)) return rotary_launch<T, 2, INTER>(a, stream);
  return ws_record_failure(WS_EINTERNAL, "no access width fits");
}

// One element (a pair, where interleaved) at a time, for any alignment.
template <class T, bool INTER>
__global__ void __launch_bounds__(256) rotary_single_kernel(RotaryArgs a) {
  using raw = typename T::raw;
  const uint32_t id = blockIdx.x * 256u + threadIdx.x;
  const uint32_t rest = id / (uint32_t)a.items;
  const int32_t item = (int32_t)(id - rest * a.items);
  const int64_t token = rest / (uint32_t)a.heads;
  const int32_t h = (int32_t)(rest % (uint32_t)a.heads);
  if (token >= a.n) return;
  const raw *x = (const raw *)a.x + token * a.xt + h * a.xh;
  raw *out = (raw *)a.out + token * a.ot + h * a.oh;
  const int32_t part = a.turn.part, half = part / 2;
  if (item >= half) {
    out[part + item - half] = x[part + item - half];
    return;
  }
  const float *row = turn_row(a.turn, ask_position(a.turn, token));
  const float c = row ? row[item] : NAN;
  float s = row ? row[half + item] : NAN;
  if (a.inverse) s = -s;
  const int32_t i = INTER ? 2 * item : item, j = INTER ? i + 1 : i + half;
  const float u = T::get(x[i]), w = T::get(x[j]);
  out[i] = T::put(u * c - w * s);
  out[j] = T::put(w * c + u * s);
}

template <class T>
int rotary_type(RotaryArgs a, int max_vec, bool inter, hipStream_t stream) {
  const int32_t unit = inter ? a.turn.part : a.turn.part / 2;
  if (max_vec >= 2 && unit % 2 == 0 && (a.dim - a.turn.part) % 2 == 0)
    return inter ? rotary_vec<T, true>(a, max_vec, stream) : rotary_vec<T, false>(a, max_vec, stream);
  a.items = a.turn.part / 2 + a.dim - a.turn.part;
  return in_ranges<T>(a, (int64_t)a.heads * a.items, [&](const RotaryArgs &r, uint32_t blocks) {
    if (inter)
      rotary_single_kernel<T, true><<<dim3(blocks), 256, 0, stream>>>(r);
    else
      rotary_single_kernel<T, false><<<dim3(blocks), 256, 0, stream>>>(r);
  });
}

// ------------------------------------------------------------ append -----

struct AppendArgs {
  const void *k, *v;
  int64_t kt, kh, vt, vh;
  void *ck, *cv;
  float *ks, *vs;
  const int64_t *slots;
  int64_t n, n_slots;
  int32_t heads, page_shift;
  int32_t head_groups;  // groups of H heads
  int32_t interleaved;
  TurnArgs turn;
};

// Beyond the threads that the card holds at once, a thread takes two heads.
// 8191 x 8 rows of 128, fp16 into int8: 12.5 us against 13.6 with one head a
// thread, 14.0 with four, 16.7 with eight; 1024 x 32 rows, bf16 into fp8, which it
// holds: 8.6 against 7.9.
constexpr int kHeads = 2;
constexpr int64_t kResidentThreads = 256 * 2048;

// A row's eight elements u, d .. d+7, of this lane turned by the angles of
// `row`, element by element: neighbours, or halves that do not fill lanes.
template <class T>
__device__ __forceinline__ void turn_any(const typename T::raw *x, int d, const AppendArgs &a,
                                         const float *row, float (&u)[8]) {
  const int part = a.turn.part, half = part / 2;
  if (d >= part) return;
  if (a.interleaved) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      if (d + i >= part) break;
      const float c = row ? row[(d + i) / 2] : NAN, s = row ? row[half + (d + i) / 2] : NAN;
      const float p = u[i], q = u[i + 1];
      u[i] = p * c - q * s;
      u[i + 1] = q * c + p * s;
    }
    return;
  }
  for (int i = 0; i < 8 && d + i < part; ++i) {
    const bool low = d + i < half;
    const int j = low ? d + i : d + i - half;
    const float c = row ? row[j] : NAN, s = row ? row[half + j] : NAN;
    const float other = T::get(x[low ? d + i + half : d + i - half]);
    u[i] = low ? u[i] * c - other * s : u[i] * c + other * s;
  }
}

// G = dim / 8 lanes take the two rows of H heads of a token, which are read and
// written once, whole lines each; slot, position and angles are read once for
// the H.  LANES: nothing is turned, or halves of whole lanes.
// 8191 x 8 rows of 128, fp16 into int8, the keys turned (50 MB): 12.5 us (4.0
// TB/s), 17.1 with a wait at each request for what is converted there.
template <class T, int TYPE, int G, int VEC, int H, bool LANES>
__global__ void __launch_bounds__(256) append_kernel(AppendArgs a) {
  using raw = typename T::raw;
  constexpr int dim = 8 * G;
  const int lane = threadIdx.x % G;
  const uint32_t id = blockIdx.x * (256u / G) + threadIdx.x / G;
  const int64_t token = id / (uint32_t)a.head_groups;
  const int32_t h0 = (int32_t)(id - (uint32_t)token * (uint32_t)a.head_groups) * H;
  if (token >= a.n) return;  // the G lanes of a row end together
  const raw *k = (const raw *)a.k + token * a.kt;
  const raw *v = (const raw *)a.v + token * a.vt;
  const int d = lane * 8;
  // Everything is asked for before the first use of any of it, the position
  // first, which the angles wait for; partners in a rotation come by a second
  // read, which the first level cache answers.
  const bool turn = a.turn.positions != nullptr;
  const int half = a.turn.part / 2;
  const bool low = d < half, turned = LANES && turn && d < a.turn.part;
  const int partner = !turned ? d : low ? d + half : d - half;
  Position position = {};
  if (turn) position = ask_position(a.turn, token);
  const int64_t slot = a.slots[token];
  raw x[H][8], y[H][8], w[H][8];
#pragma unroll
  for (int i = 0; i < H; ++i) {
    const int32_t h = min(h0 + i, a.heads - 1);
    load_raw<T, 8, VEC>(k + h * a.kh + d, x[i]);
    load_raw<T, 8, VEC>(v + h * a.vh + d, y[i]);
    if constexpr (LANES) load_raw<T, 8, VEC>(k + h * a.kh + partner, w[i]);
  }
  all_asked(position);
  const float *angles = turn ? turn_row(a.turn, position) : nullptr;
  float c[8], s[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) c[e] = s[e] = NAN;
  if (turned && angles) {
    const float *p = angles + (low ? d : d - half);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      c[e] = p[e];
      s[e] = p[half + e];
    }
  }
  if (slot < 0 || slot >= a.n_slots) return;
  const int64_t page = slot >> a.page_shift, off = slot & ((1 << a.page_shift) - 1);
#pragma unroll
  for (int i = 0; i < H; ++i) {
    const int32_t h = h0 + i;
    if (h >= a.heads) break;
    const int64_t row = ((page * a.heads + h) << a.page_shift) + off;
    float u[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = T::get(x[i][e]);
    if constexpr (LANES) {
      if (turned) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float other = T::get(w[i][e]);
          u[e] = u[e] * c[e] + (low ? -other : other) * s[e];
        }
      }
    } else if (turn) {
      turn_any<T>(k + h * a.kh, d, a, angles, u);
    }
    put_row<TYPE, G>(a.ck, a.ks, row, lane, dim, u);
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = T::get(y[i][e]);
    put_row<TYPE, G>(a.cv, a.vs, row, lane, dim, u);
  }
}

template <class T, int TYPE, int G>
int append_launch(AppendArgs a, int vec, hipStream_t stream) {
  constexpr int wide = 16 / sizeof(typename T::raw);
  const bool lanes = vec >= wide && !a.interleaved && a.turn.part % 16 == 0;
  const bool many = lanes && a.heads >= kHeads && a.n * a.heads * G > kResidentThreads;
  a.head_groups = many ? (a.heads + kHeads - 1) / kHeads : a.heads;
  return token_ranges(a.n, (int64_t)a.head_groups * G, 1, [&](int64_t from, int64_t n) {
    AppendArgs r = a;
    r.n = n;
    r.k = (const typename T::raw *)a.k + from * a.kt;
    r.v = (const typename T::raw *)a.v + from * a.vt;
    r.slots = a.slots + from;
    skip_positions(r.turn, from);
    const dim3 blocks((uint32_t)((n * a.head_groups + 256 / G - 1) / (256 / G)));
    if (many)
      append_kernel<T, TYPE, G, wide, kHeads, true><<<blocks, 256, 0, stream>>>(r);
    else if (lanes)
      append_kernel<T, TYPE, G, wide, 1, true><<<blocks, 256, 0, stream>>>(r);
    else if (vec >= wide)
      append_kernel<T, TYPE, G, wide, 1, false><<<blocks, 256, 0, stream>>>(r);
    else
      append_kernel<T, TYPE, G, 1, 1, false><<<blocks, 256, 0, stream>>>(r);
  });
}

template <class T, int TYPE>
int append_dim(const AppendArgs &a, int dim, int vec, hipStream_t stream) {
  if (dim == 64) return append_launch<T, TYPE, 8>(a, vec, stream);
  if (dim == 128) return append_launch<T, TYPE, 16>(a, vec, stream);
  return append_launch<T, TYPE, 32>(a, vec, stream);
}

template <class T>
int append_type(const AppendArgs &a, int type, int dim, int vec, hipStream_t stream) {
  switch (type) {
    case WS_KV_BF16: return append_dim<T, WS_KV_BF16>(a, dim, vec, stream);
    case WS_KV_FP16: return append_dim<T, WS_KV_FP16>(a, dim, vec, stream);
    case WS_KV_FP8: return append_dim<T, WS_KV_FP8>(a, dim, vec, stream);
    default: return append_dim<T, WS_KV_INT8>(a, dim, vec, stream);
  }
}

// -------------------------------------------------------------- read -----

struct ReadArgs {
  const void *ck, *cv;
  const float *ks, *vs;
  const int64_t *slots;
  void *k, *v;
  int64_t kt, kh, vt, vh;
  int64_t n, n_slots;
  int32_t heads, page_shift;
};

template <int TYPE>
__device__ __forceinline__ void get_row(const void *base, const float *scales, int64_t row, int lane,
                                        int dim, float (&u)[8]) {
  if constexpr (TYPE == WS_KV_BF16) {
    load_n<Bf16, 8, 8>((const uint16_t *)base + row * dim + lane * 8, u);
  } else if constexpr (TYPE == WS_KV_FP16) {
    load_n<Fp16, 8, 8>((const uint16_t *)base + row * dim + lane * 8, u);
  } else {
    const u32x2 code = *reinterpret_cast<const u32x2 *>((const uint8_t *)base + row * dim + lane * 8);
    const float scale = scales[row];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x2 w = codes_to_half<TYPE>(code[i]);
      const half2v lo = __builtin_bit_cast(half2v, (uint32_t)w.x);
      const half2v hi = __builtin_bit_cast(half2v, (uint32_t)w.y);
      u[4 * i] = (float)lo.x * scale;
      u[4 * i + 1] = (float)lo.y * scale;
      u[4 * i + 2] = (float)hi.x * scale;
      u[4 * i + 3] = (float)hi.y * scale;
    }
  }
}

// As append, but a head's rows of 16 tokens follow one another, as they do in a
// page: 32,768 x 32 rows of 128, fp8 to fp32 (1.3 GB), 268 us (5.0 TB/s) against
// 286 with the heads of a token together.
template <class T, int TYPE, int G, int VEC>
__global__ void __launch_bounds__(256) read_kernel(ReadArgs a) {
  using raw = typename T::raw;
  constexpr int dim = 8 * G;
  const int lane = threadIdx.x % G;
  const uint32_t id = blockIdx.x * (256u / G) + threadIdx.x / G;
  const uint32_t sixteen = id / (16u * a.heads), in = id - sixteen * (16u * a.heads);
  const int64_t token = (int64_t)sixteen * 16 + in % 16;
  const int32_t h = (int32_t)(in / 16);
  if (token >= a.n) return;
  const int64_t slot = a.slots[token];
  float x[8] = {}, y[8] = {};
  if (slot >= 0 && slot < a.n_slots) {
    const int64_t page = slot >> a.page_shift, off = slot & ((1 << a.page_shift) - 1);
    const int64_t row = ((page * a.heads + h) << a.page_shift) + off;
    get_row<TYPE>(a.ck, a.ks, row, lane, dim, x);
    get_row<TYPE>(a.cv, a.vs, row, lane, dim, y);
  }
  store_n<T, 8, VEC>((raw *)a.k + token * a.kt + h * a.kh + lane * 8, x);
  store_n<T, 8, VEC>((raw *)a.v + token * a.vt + h * a.vh + lane * 8, y);
}

template <class T, int TYPE, int G>
int read_launch(const ReadArgs &a, int vec, hipStream_t stream) {
  constexpr int wide = 16 / sizeof(typename T::raw);
  return token_ranges(a.n, (int64_t)a.heads * G, 16, [&](int64_t from, int64_t n) {
    ReadArgs r = a;
    r.n = n;
    r.k = (typename T::raw *)a.k + from * a.kt;
    r.v = (typename T::raw *)a.v + from * a.vt;
    r.slots = a.slots + from;
    const int64_t rows = (n + 15) / 16 * 16 * a.heads;
    const dim3 blocks((uint32_t)((rows + 256 / G - 1) / (256 / G)));
    if (vec >= wide)
      read_kernel<T, TYPE, G, wide><<<blocks, 256, 0, stream>>>(r);
    else
      read_kernel<T, TYPE, G, 1><<<blocks, 256, 0, stream>>>(r);
  });
}

template <class T, int TYPE>
int read_dim(const ReadArgs &a, int dim, int vec, hipStream_t stream) {
  if (dim == 64) return read_launch<T, TYPE, 8>(a, vec, stream);
  if (dim == 128) return read_launch<T, TYPE, 16>(a, vec, stream);
  return read_launch<T, TYPE, 32>(a, vec, stream);
}

template <class T>
int read_type(const ReadArgs &a, int type, int dim, int vec, hipStream_t stream) {
  switch (type) {
    case WS_KV_BF16: return read_dim<T, WS_KV_BF16>(a, dim, vec, stream);
    case WS_KV_FP16: return read_dim<T, WS_KV_FP16>(a, dim, vec, stream);
    case WS_KV_FP8: return read_dim<T, WS_KV_FP8>(a, dim, vec, stream);
    default: return read_dim<T, WS_KV_INT8>(a, dim, vec, stream);
  }
}

}  // namespace

extern "C" {

int wait_kv_rotary(const ws_kv_rows *x, const ws_kv_rows *out, int64_t n, int32_t heads,
                   int32_t dim, const ws_kv_turn *turn, int32_t inverse, void *hip_stream) {
  return guarded([&]() -> int {
    if (n < 0 || heads < 1 || dim < 2 || dim > 65536) return invalid("rotary: bad sizes");
    if (n >= (int64_t)1 << 31) return ws_record_failure(WS_EUNSUPPORTED, "2^31 tokens or more");
    if (int rc = check_rows(x, n, "rotary: x must be non-NULL")) return rc;
    if (int rc = check_rows(out, n, "rotary: out must be non-NULL")) return rc;
    if (x->type != out->type) return invalid("rotary: x and out must have one type");
    if (int rc = check_turn(turn, n, dim)) return rc;
    if (x->data == out->data &&
        (x->token_stride != out->token_stride || x->head_stride != out->head_stride))
      return invalid("rotary: in place, the strides must be the same");
    if (!one_place(*x, *out) && overlap(*x, *out, n, heads, dim))
      return invalid("rotary: out must be x or not overlap it");
    if (n == 0) return WS_OK;
    RotaryArgs a{};
    a.x = x->data;
    a.out = out->data;
    a.xt = x->token_stride;
    a.xh = x->head_stride;
    a.ot = out->token_stride;
    a.oh = out->head_stride;
    a.n = n;
    a.heads = heads;
    a.dim = dim;
    a.inverse = inverse != 0;
    a.turn = {turn->table, turn->positions, turn->positions_32, turn->n_table, turn->part};
    const int vec = widest(*x, *out);
    const bool inter = turn->interleaved != 0;
    hipStream_t s = (hipStream_t)hip_stream;
    if (x->type == WS_KV_BF16) return rotary_type<Bf16>(a, vec, inter, s);
    if (x->type == WS_KV_FP16) return rotary_type<Fp16>(a, vec, inter, s);
    return rotary_type<Fp32>(a, vec, inter, s);
  });
}

int wait_kv_append(const ws_kv_cache *cache, const ws_kv_rows *k, const ws_kv_rows *v,
                   const int64_t *slots, int64_t n, const ws_kv_turn *turn, void *hip_stream) {
  return guarded([&]() -> int {
    if (int rc = check_cache(cache)) return rc;
    if (n < 0) return invalid("append: bad sizes");
    if (n + 16 >= ((int64_t)1 << 31) / cache->kv_heads)
      return ws_record_failure(WS_EUNSUPPORTED, "2^31 rows or more");
    if (int rc = check_rows(k, n, "append: k must be non-NULL")) return rc;
    if (int rc = check_rows(v, n, "append: v must be non-NULL")) return rc;
    if (k->type != v->type) return invalid("append: k and v must have one type");
    if (n > 0 && !slots) return invalid("append: slots must be non-NULL");
    if ((uintptr_t)slots % 8) return invalid("append: slots must be aligned to 8 bytes");
    if (turn)
      if (int rc = check_turn(turn, n, cache->dim)) return rc;
    if (n == 0) return WS_OK;
    AppendArgs a{};
    a.k = k->data;
    a.v = v->data;
    a.kt = k->token_stride;
    a.kh = k->head_stride;
    a.vt = v->token_stride;
    a.vh = v->head_stride;
    a.ck = cache->k;
    a.cv = cache->v;
    a.ks = cache->k_scale;
    a.vs = cache->v_scale;
    a.slots = slots;
    a.n = n;
    a.n_slots = (int64_t)cache->pages * cache->page_size;
    a.heads = cache->kv_heads;
    a.page_shift = log2_of(cache->page_size);
    if (turn) {
      a.interleaved = turn->interleaved != 0;
      a.turn = {turn->table, turn->positions, turn->positions_32, turn->n_table, turn->part};
    }
    const int vec = widest(*k, *v);
    hipStream_t s = (hipStream_t)hip_stream;
    if (k->type == WS_KV_BF16) return append_type<Bf16>(a, cache->type, cache->dim, vec, s);
    if (k->type == WS_KV_FP16) return append_type<Fp16>(a, cache->type, cache->dim, vec, s);
    return append_type<Fp32>(a, cache->type, cache->dim, vec, s);
  });
}

int wait_kv_read(const ws_kv_cache *cache, const int64_t *slots, int64_t n, const ws_kv_rows *k,
                 const ws_kv_rows *v, void *hip_stream) {
  return guarded([&]() -> int {
    if (int rc = check_cache(cache)) return rc;
    if (n < 0) return invalid("read: bad sizes");
    if (n + 16 >= ((int64_t)1 << 31) / cache->kv_heads)
      return ws_record_failure(WS_EUNSUPPORTED, "2^31 rows or more");
    if (int rc = check_rows(k, n, "read: k must be non-NULL")) return rc;
    if (int rc = check_rows(v, n, "read: v must be non-NULL")) return rc;
    if (k->type != v->type) return invalid("read: k and v must have one type");
    if (overlap(*k, *v, n, cache->kv_heads, cache->dim))
      return invalid("read: k and v must not overlap");
    if (n > 0 && !slots) return invalid("read: slots must be non-NULL");
    if ((uintptr_t)slots % 8) return invalid("read: slots must be aligned to 8 bytes");
    if (n == 0) return WS_OK;
    ReadArgs a{};
    a.ck = cache->k;
    a.cv = cache->v;
    a.ks = cache->k_scale;
    a.vs = cache->v_scale;
    a.slots = slots;
    a.k = k->data;
    a.v = v->data;
    a.kt = k->token_stride;
    a.kh = k->head_stride;
    a.vt = v->token_stride;
    a.vh = v->head_stride;
    a.n = n;
    a.n_slots = (int64_t)cache->pages * cache->page_size;
    a.heads = cache->kv_heads;
    a.page_shift = log2_of(cache->page_size);
    const int vec = widest(*k, *v);
    hipStream_t s = (hipStream_t)hip_stream;
    if (k->type == WS_KV_BF16) return read_type<Bf16>(a, cache->type, cache->dim, vec, s);
    if (k->type == WS_KV_FP16) return read_type<Fp16>(a, cache->type, cache->dim, vec, s);
    return read_type<Fp32>(a, cache->type, cache->dim, vec, s);
  });
}

}  // extern "C"

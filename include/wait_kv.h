/*
 * wait_kv.h -- C ABI of the KV-path operators (MI355X / gfx950).
 *
 * What one iteration of the simulated server does with its KV cache, so that
 * the iteration time d0 + d1 * tokens and the budget C of wait_sim.h can be
 * measured on the card:
 *
 *   - wait_kv_rotary: vectors turned by their positions,
 *   - wait_kv_append: new keys and values into the pages of a cache, as 16-bit
 *     values or quantised to 8 bits, the keys turned on the way,
 *   - wait_kv_read: rows of a cache back as values,
 *   - wait_kv_attention: every token's softmax-weighted mean of the values of
 *     its request's keys, over the pages.
 *
 * All pointers are device pointers unless said otherwise.  Calls are
 * asynchronous on hip_stream, allocate nothing, and can be captured into a
 * graph.  They return WS_OK or an error code of wait_sim.h, with a message in
 * wait_sim_last_error().  Strides are in elements; a vector's own elements lie
 * one after another.  Vectors whose base or strides are not multiples of 16
 * bytes take slower loads, with the same results.  Output rows must not
 * overlap one another, nor an input's rows; those of wait_kv_rotary and
 * wait_kv_attention may be the input itself.
 */
#ifndef WAIT_KV_H
#define WAIT_KV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Types of elements.  WS_KV_FP8 is the 8-bit float with 4 exponent and 3
 * fraction bits, no infinities, largest value 448. */
enum { WS_KV_BF16 = 0, WS_KV_FP16 = 1, WS_KV_FP32 = 2, WS_KV_FP8 = 3, WS_KV_INT8 = 4 };

/* [n][heads] vectors of dim elements: element d of vector (i, h) is at
 * data[i * token_stride + h * head_stride + d]. */
typedef struct {
  void *data;
  int64_t token_stride, head_stride;
  int32_t type; /* WS_KV_BF16, WS_KV_FP16 or WS_KV_FP32 */
} ws_kv_rows;

/* Rotation of the first `part` elements of a vector by its position p.
 * table [positions][part], fp32, contiguous: row p has the cosines of the
 * part / 2 angles, then their sines (both times whatever factor the scaling to
 * long contexts asks for).  Pair i is the elements (i, i + part / 2), or
 * (2 i, 2 i + 1) where interleaved.  A position outside the table makes the
 * vector's first `part` elements NaN. */
typedef struct {
  const float *table;
  const void *positions; /* [n], int64 or int32 */
  int32_t positions_32;  /* 1: int32 */
  int32_t n_table;       /* rows of the table */
  int32_t part;          /* even, 2 .. dim */
  int32_t interleaved;
} ws_kv_turn;

/* A cache of one layer: k and v [pages][kv_heads][page_size][dim], contiguous,
 * 16-byte aligned; page_size a power of two up to 1024, dim 64, 128 or 256,
 * pages * kv_heads * page_size < 2^31.
 * 8-bit types have fp32 scales [pages][kv_heads][page_size]: an element stands
 * for code * scale.  Slot page * page_size + offset names a token's rows. */
typedef struct {
  void *k, *v;
  float *k_scale, *v_scale; /* NULL for 16-bit types */
  int32_t pages, page_size, kv_heads, dim, type;
} ws_kv_cache;

/* out = x turned; inverse: turned back (the gradient of a rotation).  n tokens
 * of `heads` vectors of dim elements; out may be x itself, and shares no memory
 * with it otherwise (rows within the range of the other's need the same token
 * stride).  Angles and products are in fp32, rounded once to x's type. */
int wait_kv_rotary(const ws_kv_rows *x, const ws_kv_rows *out, int64_t n, int32_t heads,
                   int32_t dim, const ws_kv_turn *turn, int32_t inverse, void *hip_stream);

/* Rows i = 0 .. n-1 of k and v into slots[i] (int64); a row whose slot is
 * outside the cache is left out.  Slots within the cache must differ: what two
 * rows with one slot leave there is made of both, codes of one under the scale
 * of the other among it.
 * turn (NULL: none) rotates k.  8-bit types: with t the row's largest
 * magnitude and M the largest code (448, 127), scale = t / M and
 * code = x * ((1 / t) * M) in fp32, rounded to nearest, ties to even.  Rows
 * with t < 2^-100 are stored as zeros with scale 0, rows that hold an infinity
 * or a NaN as zeros with scale NaN, which read back as NaN. */
int wait_kv_append(const ws_kv_cache *cache, const ws_kv_rows *k, const ws_kv_rows *v,
                   const int64_t *slots, int64_t n, const ws_kv_turn *turn, void *hip_stream);

/* Rows i = 0 .. n-1 of k and v from slots[i], as values, rounded once to the
 * outputs' type; zeros for a slot outside the cache. */
int wait_kv_read(const ws_kv_cache *cache, const int64_t *slots, int64_t n, const ws_kv_rows *k,
                 const ws_kv_rows *v, void *hip_stream);

/* Attention of n_tokens queries of n_seq requests.  Request b has the queries
 * starts[b] .. starts[b + 1] - 1 and kv_lens[b] keys, key j in the cache at
 * offset j % page_size of page table[b * table_stride + j / page_size].  Query
 * i of its n sits at position p = kv_len - n + i and sees the keys j with
 *   j < kv_len, j <= p (causal), j > p - window (window > 0).
 * out = sum_j softmax_j(scale q . k_j) v_j over those; head h reads KV head
 * h / (heads / kv_heads).  A query that sees nothing gets zeros, and
 * lse = -infinity.  Keys whose page is outside 0 .. pages-1, or behind the
 * table's table_cols columns, are not there.  Queries outside every request
 * leave out as it is. */
typedef struct {
  const int32_t *table;
  int64_t table_stride;
  int32_t table_cols;
  const int32_t *starts;  /* [n_seq + 1], not decreasing, within 0 .. n_tokens */
  const int32_t *kv_lens; /* [n_seq] */
  int32_t n_seq;
  int32_t n_tokens;
  int32_t heads;          /* a multiple of kv_heads */
  float scale;            /* > 0 */
  int32_t causal;
  int32_t window;         /* 0: none */
  /* Upper bounds that the launch is laid out for.  Requests that are longer
   * are computed all the same, only slower; bounds far above the lengths cost
   * time and workspace. */
  int32_t max_q_len, max_kv_len;
} ws_kv_batch;

/* Bytes of workspace that wait_kv_attention takes for this batch (0 where no
 * request is split over its keys). */
int wait_kv_attention_workspace_bytes(const ws_kv_cache *cache, const ws_kv_batch *batch,
                                      size_t *bytes);

/* q and out: bf16 or fp16, the cache's type where that is a 16-bit one; out may
 * be q itself, and shares no memory with it otherwise (as in wait_kv_rotary).
 * lse (NULL: none): [n_tokens][heads] fp32, the natural logarithm of the
 * softmax's denominator, sum_j exp(scale q . k_j).  Products, softmax and sums
 * are in fp32; the weights are rounded to 16 bits before they meet the
 * values.  The workspace holds nothing between calls; calls that overlap need
 * one each. */
int wait_kv_attention(const ws_kv_cache *cache, const ws_kv_batch *batch, const ws_kv_rows *q,
                      const ws_kv_rows *out, float *lse, void *d_workspace, size_t ws_bytes,
                      void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif

/*
 * wait_kv_norm.h -- C ABI of the norms of queries and keys (MI355X / gfx950).
 *
 * Models that norm each head's query and key vectors do so between the product
 * that makes them and their rotation.  Here norm and rotation are one pass:
 *
 *   - wait_kv_norm_rotary: vectors normed, then turned by their positions,
 *   - wait_kv_enter: a batch's queries, keys and values on their way into a
 *     layer: queries normed and turned, keys normed and turned into the cache,
 *     values into the cache, in one launch.
 *
 * Pointers, strides, streams, errors and what must not overlap are as in
 * wait_kv.h.
 */
#ifndef WAIT_KV_NORM_H
#define WAIT_KV_NORM_H

#include "wait_kv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* y_d = x_d * r * w_d with r = 1 / sqrt(mean_d x_d^2 + eps), each vector by
 * itself, in fp32.  w: dim weights one after another, of head h at
 * weight[h * head_stride]; head_stride 0 where the heads share them; NULL: ones.
 * Nothing is rounded between the norm and a rotation. */
typedef struct {
  const void *weight;
  int64_t head_stride; /* in elements */
  int32_t type;        /* of the weights: WS_KV_BF16, WS_KV_FP16 or WS_KV_FP32 */
  float eps;           /* >= 0, finite */
} ws_kv_norm;

/* out = x normed (NULL: as it is), then turned (NULL: not), rounded once to x's
 * type.  n tokens of `heads` vectors of dim elements; out may be x itself. */
int wait_kv_norm_rotary(const ws_kv_rows *x, const ws_kv_rows *out, int64_t n, int32_t heads,
                        int32_t dim, const ws_kv_norm *norm, const ws_kv_turn *turn,
                        void *hip_stream);

/* Rows i = 0 .. n-1 of a batch: q [n][heads] by q_norm and turn into q_out; k and
 * v [n][kv_heads] of the cache into slots[i], as wait_kv_append puts them there,
 * k by k_norm and turn.  One turn for both; either norm and the turn may be
 * NULL.  q, q_out, k and v have one type.  q_out may be q itself and shares no
 * memory with k, v or the cache.  A row whose slot is outside the cache gives its queries
 * all the same. */
int wait_kv_enter(const ws_kv_cache *cache, const ws_kv_rows *q, const ws_kv_rows *q_out,
                  int32_t heads, const ws_kv_rows *k, const ws_kv_rows *v, const int64_t *slots,
                  int64_t n, const ws_kv_norm *q_norm, const ws_kv_norm *k_norm,
                  const ws_kv_turn *turn, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif

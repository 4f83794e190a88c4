/*
 * wait_kv_budget.h -- C ABI of the operators that hold a request's cached tokens
 * within a budget (MI355X / gfx950).
 *
 *   - wait_kv_weigh: how much attention every cached key received,
 *   - wait_kv_evict: of a request that holds more keys than it may keep, the
 *     last ones stay and, of the others, those that received most.
 *
 * Pointers, streams, errors and graphs are as in wait_kv.h.  Weights are
 * [pages][kv_heads][page_size] fp32, contiguous, one for each row of a cache.
 */
#ifndef WAIT_KV_BUDGET_H
#define WAIT_KV_BUDGET_H

#include "wait_kv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of workspace that wait_kv_weigh takes for this batch (0 where no
 * request's tokens are split). */
int wait_kv_weigh_workspace_bytes(const ws_kv_cache *cache, const ws_kv_batch *batch,
                                  size_t *bytes);

/* The batch is one of wait_kv_attention, q its queries (bf16 or fp16, the
 * cache's type where that is a 16-bit one) and lse [n_tokens][heads] fp32 the
 * log-sums that it returned.  For key j of request b and KV head h
 *   S = sum over the tokens i of b that see j, and the heads g that read h, of
 *       exp(scale q_ig . k_j - lse_ig),
 * in fp32, and the weight of j's row becomes S, plus what it was if `accumulate`
 * and j < kv_len - n: the batch's own n tokens are new, and start from zero
 * whatever their rows held.  Rows whose log-sum is -infinity saw nothing and
 * count nothing.  Keys that are not there (wait_kv.h) have no weight.  Two
 * requests must not share pages, nor the weights memory with the cache or another
 * input.  Sums are taken in a fixed order: the same call gives the same bits.  The
 * workspace is memory of its own, and holds nothing between calls; calls that
 * overlap need one each. */
int wait_kv_weigh(const ws_kv_cache *cache, const ws_kv_batch *batch, const ws_kv_rows *q,
                  const float *lse, float *weights, int32_t accumulate, void *d_workspace,
                  size_t ws_bytes, void *hip_stream);

/* A batch of requests that go back to `keep` keys each.  Key j of request b is
 * at offset j % page_size of page table[b * table_stride + j / page_size].  A
 * request of m = kv_lens[b] > keep keys keeps its last `recent` and, of the
 * others, the keep - recent with the largest weights, KV head by KV head (equal
 * ones: the lower index; NaN is larger than all else), in their order; one of
 * up to keep keys keeps all.  Kept rows d = 0, 1, ... of k, v, their scales and
 * weights go to offset d % page_size of page to[b * to_stride + d / page_size],
 * or of the request's own pages where `to` is NULL.  Rows behind them stay as
 * they are.
 * Requests share no pages, and pages of `to` are no request's (`to` is not `table`).
 * Pages are there: of a row whose page is outside 0 .. pages-1 nothing is read, its
 * weight is less than all others, and nothing is written in its place; keys behind
 * the table's columns do not count. */
typedef struct {
  const int32_t *table;
  int64_t table_stride;
  int32_t table_cols;
  const int32_t *kv_lens; /* [n_seq] */
  int32_t n_seq;
  int32_t keep;   /* >= 1 */
  int32_t recent; /* 0 .. keep */
  const int32_t *to; /* NULL: in place */
  int64_t to_stride;
  int32_t to_cols;    /* at least keep / page_size, rounded up */
  /* Upper bound that the launch is laid out for.  Requests that are longer are
   * right all the same, only slower. */
  int32_t max_kv_len;
} ws_kv_eviction;

/* Bytes of workspace that wait_kv_evict takes: 0 where requests are short, at most
 * 256 MB. */
int wait_kv_evict_workspace_bytes(const ws_kv_cache *cache, const ws_kv_eviction *eviction,
                                  size_t *bytes);

/* kept [n_seq][kv_heads][keep] int32: the kept keys' indices, -1 behind them;
 * new_lens [n_seq]: min(kv_lens, keep).  Weights, outputs and workspace have memory
 * of their own, apart from one another, the cache, its page tables and the lengths;
 * so have keys and values that move in place.  The workspace holds nothing between
 * calls; calls that overlap need one each. */
int wait_kv_evict(const ws_kv_cache *cache, const ws_kv_eviction *eviction, float *weights,
                  int32_t *kept, int32_t *new_lens, void *d_workspace, size_t ws_bytes,
                  void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif

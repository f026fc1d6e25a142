/*
 * flasheval_packed.h -- a paged cache that holds keys and values in 4 bits: its append, reading rows back, the
 * attention of a request's lists over it, the attention weight that every cached row received, and eviction by it.
 *
 *   fe_packed_page_bytes      bytes of a page
 *   fe_packed_append          new rows of every sequence into the cache, keys (and queries) turned on the way
 *   fe_packed_read            rows of every sequence as dense tensors
 *   fe_packed_attention       attention over shared rows and the list's own rows, both in such caches
 *   fe_packed_weights         adds to every cached row's weight what the query rows gave it
 *   fe_packed_weights_strided the same with log sums of any strides
 *   fe_packed_evict           keeps the rows of greatest weight, in other pages
 *   fe_packed_workspace_size  workspace bytes of fe_packed_attention or fe_packed_weights
 *
 * Conventions are those of flasheval_prefix.h: device pointers owned by the caller, nothing allocated and
 * nothing waited for, asynchronous on `stream`, host-side validation before any launch, no state between
 * calls, lengths on the device and clamped to their range, rows outside them never used.  One workspace is not used by
 * two streams, or two captured graphs that may run at once, at a time.  No output may overlap an input or another output, but
 * where that is said below.
 *
 * What 4 bits stand for.  The columns of a head are held in blocks of 32: 4-bit floats (from the top bit: sign, two
 * exponent bits, one mantissa bit; magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6) times 2^(e - 127) with one byte e a block.
 * A block is written with the smallest e in [2, 252] for which no magnitude exceeds 6 * 2^(e - 127) (at 252 larger ones
 * become 6), each value rounded to the nearest of the 15, ties to the even code; a block with an
 * infinity or a NaN in it is written with e = 255 and all its columns are NaN.  Every value is exact in bf16.
 *
 * Layout.  A page holds page_rows rows: for every key head, head_bytes =
 *   page_rows * (dh + dh / 16) rounded up to 16 bytes:
 *   key codes [page_rows][dh / 2], value codes [page_rows][dh / 2], key scales [page_rows][dh / 32], value scales
 * with column c of a row in byte c / 2, the low half for even c.  Head g of page p begins at pages + p * page_ld +
 * g * head_bytes.
 */
#ifndef FLASHEVAL_PACKED_H
#define FLASHEVAL_PACKED_H

#include <stddef.h>
#include <stdint.h>

#include "flasheval_prefix.h"

#ifdef __cplusplus
extern "C" {
#endif

/* N sequences in pages of a pool: logical row j of sequence s is row j % page_rows of page table[s][j / page_rows]; a
 * table entry outside [0, n_pages) names no page.  cols * page_rows is a sequence's capacity. */
typedef struct {
  void* pages;                          /* 16-byte aligned */
  int64_t page_ld;                      /* bytes from one page to the next: a multiple of 16, >= n_kv_heads * head_bytes, < 2^31 */
  const int32_t* table;                 /* [N][cols] */
  int32_t* len;                         /* [N] rows in the cache; written by fe_packed_evict's `to` alone */
  int32_t N, cols, page_rows, n_pages;
} fe_packed_cache;

/* Bytes of one page of n_kv_heads heads of width dh; FE_EUNSUPPORTED for dh outside {32, 64, 128}. */
fe_status fe_packed_page_bytes(int32_t page_rows, int32_t n_kv_heads, int32_t dh, size_t* bytes);

/*
 * fe_packed_append: row i < n(s) = new_len[s] of sequence s becomes logical row j = len[s] + i:
 *   keys of that row   = held(rotate(k[s][i], pos0[s] + j))
 *   values of that row = held(v[s][i])
 *   q_out[s][i]        = rotate(q[s][i], pos0[s] + j), rounded to its type     (when q is given)
 *   len_out[s]         = len[s] + n(s)                                         (when len_out is given; may be len)
 * with rotate as in fe_cache_append, in fp64 throughout: what is held, and what q_out gets, is the nearest to the turned row itself.
 * A row whose index reaches the capacity, or whose table entry names no page, is not written (its q_out row is);
 * status[s] is FE_DEV_BAD_PAGE then and 0 otherwise.  Other rows of the pages and rows i >= n(s) of q_out are left as they
 * were.  Two new rows must not share a cache row.
 *
 * Errors: as fe_cache_append's, and FE_EINVAL for q_out = q.
 */
typedef struct {
  fe_packed_cache cache;
  int32_t dtype;                        /* fe_dtype of q, k, v, q_out */
  int32_t S, n_heads, n_kv_heads, dh;   /* n_heads: of q; not read when q is NULL */
  int32_t rot, neighbours;
  int32_t q_ld, k_ld, v_ld, q_out_ld;   /* elements from one row to the next */
  const void *q, *k, *v;                /* [N][S] rows */
  void* q_out;
  const double* freq;                   /* [rot / 2] radians per position */
  const int32_t* new_len;               /* [N], or NULL: S */
  const int32_t* pos0;                  /* [N], or NULL: 0 */
  int32_t* len_out;                     /* [N] or NULL */
  int32_t* status;                      /* [N] or NULL */
} fe_packed_append_args;
fe_status fe_packed_append(const fe_packed_append_args* a, void* stream);

/*
 * fe_packed_read: k[s][i] and v[s][i] = the keys and values of logical row start[s] + i, for i < count[s], at most S
 * and whatever the length says; a row past the capacity or of no page is zeros.  Rows i >= count[s] are left as they were.
 * Without start the rows begin at 0, without count they are those up to the length.  k or v may be NULL.
 *
 * Errors: as fe_packed_append's.
 */
typedef struct {
  fe_packed_cache cache;
  int32_t dtype;                        /* fe_dtype of k and v */
  int32_t S, n_kv_heads, dh;
  int32_t k_ld, v_ld;                   /* elements from one row to the next */
  const int32_t *start, *count;         /* [N] or NULL; below 0 counts as 0 */
  void *k, *v;                          /* [N][S] rows of n_kv_heads * dh */
} fe_packed_read_args;
fe_status fe_packed_read(const fe_packed_read_args* a, void* stream);

/*
 * fe_packed_attention: fe_prefix_attention with both caches in 4 bits.  For query row i < n = q_len[b][k] of list k of
 * request b and head h, with key head g = h / (n_heads / n_kv_heads), the keys are rows t < ctx.len[b] of
 * sequence b of `ctx` and rows j < m = own.len[b K + k] of sequence b K + k of `own`, with `causal` only
 * j <= m - n + i; rows of no page do not count.  out = sum p v with p = softmax(scale * q.k), lse = log sum exp(scale * q.k).
 * A row without keys gives out = 0 and lse = -infinity, and so do the rows i >= n.  ctx.N = B and own.N = B * K, or 0: none.
 *
 * Scores, the softmax's maximum and sum and the output sums are fp32.  FE_BF16: the products of the queries' bf16 values with
 * the held ones are exact, probabilities are rounded to bf16 for the product with the values (where K * S * n_heads /
 * n_kv_heads, the rows of a request and key head, are at most 32: to two bf16, 16 bits).  FE_F32: queries and
 * probabilities in three bf16 parts whose sum they are, the held values whole: no product is rounded.
 * A row with a score of +infinity or NaN is NaN, and so is one whose scores are all -infinity; beside finite ones a score of
 * -infinity weighs nothing.  Scores are fp32 (infinite from 2^128 on).
 * What the own rows of other lists hold, NaN or not, changes no bit of a list's outputs; how many rows the other lists and
 * requests have may change the order of its sums.  The same call has the same bits each time.
 *
 * fe_packed_weights: for every row j < len of `ctx` and of `own` and every key head g
 *   w_out[s][g][j] = w[s][g][j] + sum over the query rows and heads of g that see it of exp(scale * q.k - lse)
 * w, w_out [N][n_kv_heads][cols * page_rows], w_out may be w; entries past the length are left as they were.  Query rows with
 * lse = -infinity add nothing; lse is an input here.  ctx_w or own_w (with its output) may be NULL: not computed.
 * fe_packed_weights_strided reads the log sum of (b, k, i, h) at lse + b lse_ld[0] + k lse_ld[1] + i lse_ld[2] + h lse_ld[3]
 * (elements; lse_ld in host memory, read during the call; a stride of 0 shares log sums).
 *
 * Workspace: fe_packed_workspace_size(a, 0 or 1 for the weights) bytes (may be 0: then ws is not read); for the weights it
 * goes by which of ctx_w and own_w are not NULL.
 *
 * Errors: FE_EINVAL for a NULL or misaligned pointer, sizes below 1, n_heads not a multiple of n_kv_heads, ctx.N or own.N
 * other than said, strides too short or not multiples of 16 bytes, a scale that is not finite, an unknown dtype, a workspace that is
 * too small, a negative stride of the log sums; FE_EUNSUPPORTED for dh outside {32, 64, 128}, a capacity above 4194304,
 * B*K*S*n_heads or N*capacity above 1073741823, more than 16777215 workgroups, or log sums that lie more than 2147483647
 * elements apart in one request or 10^15 from the first request to the last.
 */
typedef struct {
  fe_packed_cache ctx, own;
  int32_t dtype;                        /* fe_dtype of q and out */
  int32_t B, K, S, n_heads, n_kv_heads, dh, causal;
  float scale;
  int32_t q_ld, out_ld;
  const void* q;                        /* [B][K][S] rows of n_heads * dh */
  const int32_t* q_len;                 /* [B][K], or NULL: S */
  void* out;                            /* [B][K][S] rows of n_heads * dh; not read by fe_packed_weights */
  float* lse;                           /* [B][K][S][n_heads], or NULL; input of fe_packed_weights */
  const float *ctx_w, *own_w;           /* fe_packed_weights alone */
  float *ctx_w_out, *own_w_out;
  void* ws;
  size_t ws_bytes;
} fe_packed_args;
fe_status fe_packed_workspace_size(const fe_packed_args* a, int weights, size_t* bytes); /* reads sizes only */
fe_status fe_packed_attention(const fe_packed_args* a, void* stream);
fe_status fe_packed_weights(const fe_packed_args* a, void* stream);
fe_status fe_packed_weights_strided(const fe_packed_args* a, const int64_t lse_ld[4], void* stream);

/*
 * fe_packed_evict: for every sequence s (n = from.len[s] rows) and key head g, m = min(keep, n) rows are kept: the
 * first min(first, m), the last min(recent, m - that), and of the others those of greatest weight[s][g][j]; of equal weights
 * the lower index first, a NaN after every number.  In ascending order they become rows 0 .. m - 1 of head g of sequence s
 * of `to`, bits unchanged, and
 *   kept[s][g][i] = the row's index in `from`, -1 for m <= i < keep;
 *   weight_out[s][g][i] = its weight (when given);  to.len[s] = m.
 * Heads choose by themselves: a row of `to` may hold keys of another position in every head.
 * Pages of `to` must be none that a sequence of `from` names.  A row whose page on either side is none is left out of the
 * copy (kept and weight_out name it all the same); status[s] is FE_DEV_BAD_PAGE where a row in use on either side has
 * none, 0 otherwise.  Entries of weight_out past m are left as they were.
 *
 * Errors: FE_EINVAL for a NULL or misaligned pointer, sizes below 1, first or recent below 0, keep above to's
 * capacity, to.N other than from.N, the same table or lengths on both sides, a weight_out that overlaps weight;
 * FE_EUNSUPPORTED for dh outside {32, 64, 128}, a capacity above 4194304 or more than 16777215 workgroups.
 */
typedef struct {
  fe_packed_cache from, to;
  int32_t n_kv_heads, dh, keep, first, recent;
  const float* weight;                  /* [N][n_kv_heads][from.cols * from.page_rows] */
  float* weight_out;                    /* [N][n_kv_heads][to.cols * to.page_rows] or NULL */
  int32_t* kept;                        /* [N][n_kv_heads][keep] */
  int32_t* status;                      /* [N] or NULL */
} fe_packed_evict_args;
fe_status fe_packed_evict(const fe_packed_evict_args* a, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* FLASHEVAL_PACKED_H */

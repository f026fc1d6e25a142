/*
 * flasheval_prefix.h -- attention of many short lists that share one long context, its gradient, and
 * the paged cache that growing lists keep their keys and values in.
 *
 * A request has one context and K candidate lists (Section 3).  fe_encode_context leaves the
 * context's keys and values, computed once per request, in the cache that the items attend to
 * (Section 4.2).  The calls here let the rows of the lists themselves attend to that cache and, each
 * list, to its own rows, in one softmax: for list models that fuse context and list early, and for
 * hypotheses that grow token by token.  The shared rows are read once for all lists of a request.
 *
 *   fe_cache_append           new rows of every list into a paged cache, keys (and queries) turned
 *                             by their positions on the way
 *   fe_prefix_attention       attention over the shared rows and the list's own rows, dense or paged
 *   fe_prefix_attention_grad  gradients of queries, shared and own keys and values (dense own rows)
 *   fe_prefix_workspace_size  workspace bytes of the two attention calls
 *
 * Conventions are those of flasheval.h: device pointers owned by the caller, nothing allocated and
 * nothing waited for, asynchronous on `stream`, host-side validation before any launch, one workspace not used
 * by two streams (or two captured graphs that may run at once) at a time.  The calls hold no state: they can be
 * captured into a graph and replayed.  Tensors, workspace and stream belong to the current device.
 * Pointers are 16-byte aligned (int32 and double arrays as their type) and row strides are multiples
 * of 16 bytes.  Offsets into the caches are 64-bit.
 *
 * Lengths live on the device and are clamped to their range (a negative length is 0, one past the
 * capacity is the capacity).  What lies outside the lengths is never used: it may hold anything,
 * NaN and infinities included.
 */
#ifndef FLASHEVAL_PREFIX_H
#define FLASHEVAL_PREFIX_H

#include <stddef.h>
#include <stdint.h>

#include "flasheval.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Status bit of fe_cache_append, beside the FE_DEV_* bits of flasheval.h. */
#define FE_DEV_BAD_PAGE 4 /* a new row past the table's capacity, or a table entry outside [0, n_pages) */

/*
 * fe_cache_append: row i < n(s) = new_len[s] of sequence s < N becomes logical row j = len[s] + i of
 * its cache, which is row j % page_rows of page table[s][j / page_rows]:
 *   k_pages[that row] = rotate(k[s][i], pos0[s] + j)
 *   v_pages[that row] = v[s][i]
 *   q_out[s][i]       = rotate(q[s][i], pos0[s] + j)         (when q is given)
 *   len_out[s]        = len[s] + n(s)                        (when len_out is given)
 * Page p row r of a cache starts at (p * page_rows + r) * page_ld elements.  rotate turns, in every head, the
 * pairs of the first `rot` columns: pair c by the angle position * freq[c] (formed in fp64, sine and
 * cosine in fp32), (a, b) -> (a cos - b sin, b cos + a sin), one rounding to the tensor's type.
 * Pair c is columns (c, c + rot/2), or with `neighbours` columns (2c, 2c + 1).  The other columns are
 * copied, as is everything when rot = 0.
 *
 * A row whose logical index reaches table_cols * page_rows, or whose table entry is outside [0, n_pages), is
 * not written to the cache (its q_out row is); status[s] is set to FE_DEV_BAD_PAGE then and to 0 otherwise.
 * Rows of k_pages and v_pages that are not named above, and rows i >= n(s) of q_out, are left as they were.
 * len < 0 counts as 0.  Two new rows must not share a cache row (which one stays is open).
 * q_out may be q itself (same pointer and stride); no other output may overlap an input.
 * len_out may be len itself: it then advances after every row has been placed.
 *
 * Errors: FE_EINVAL for a NULL or misaligned pointer, sizes below 1, strides too short or not
 * multiples of 16 bytes, q without q_out, rot without freq, rot > dh or odd, an unknown dtype, sizes whose
 * products overflow int32; FE_EUNSUPPORTED for dh outside {32, 64, 128}, rot not a multiple of 16 or
 * N*S above 16777215.
 */
typedef struct {
  int32_t dtype;                        /* fe_dtype of q, k, v and the cache */
  int32_t N, S;                         /* sequences, new rows per sequence (capacity of new_len) */
  int32_t n_heads, n_kv_heads, dh;      /* n_heads: of q; not read when q is NULL */
  int32_t rot, neighbours;
  int32_t page_rows, n_pages, table_cols;
  int32_t q_ld, k_ld, v_ld, q_out_ld, page_ld; /* elements from one row to the next */
  const void *q, *k, *v;                /* [N][S] rows of n_heads * dh (q) or n_kv_heads * dh elements */
  void* q_out;                          /* [N][S] rows of n_heads * dh, or NULL */
  const double* freq;                   /* [rot / 2] radians per position */
  const int32_t* table;                 /* [N][table_cols] */
  const int32_t* len;                   /* [N] rows already in the cache */
  const int32_t* new_len;               /* [N], or NULL: S */
  const int32_t* pos0;                  /* [N] position of logical row 0, or NULL: 0 */
  void *k_pages, *v_pages;              /* [n_pages][page_rows] rows of n_kv_heads * dh */
  int32_t* len_out;                     /* [N] or NULL */
  int32_t* status;                      /* [N] or NULL */
} fe_append_args;
fe_status fe_cache_append(const fe_append_args* a, void* stream);

/*
 * fe_prefix_attention: for query row i < n = q_len[b][k] of list k of request b and head h, with
 * key/value head g = h / (n_heads / n_kv_heads), the keys are
 *   the shared rows t < ctx_len[b]                 of ctx_k, ctx_v [B][T], and
 *   the list's own rows j < m = own_len[b][k]      of own_k, own_v,
 *                       with `causal` only j <= m - n + i (the n query rows are the last n own rows),
 * and out = sum p v with p = softmax(scale * q.k) over them; lse = log sum exp(scale * q.k).  A row
 * without keys gives out = 0 and lse = -infinity, and so do the rows i >= n.
 *
 * Own rows are dense, own_k [B][K][L], or with page_rows > 0 paged: own_k [n_pages][page_rows] and
 * logical row j of list (b, k) in page table[b][k][j / page_rows] (L a multiple of page_rows); the
 * keys of a page outside [0, n_pages) do not count.  T = 0 or L = 0 leaves that part out.
 *
 * Scores, the softmax's maximum and sum and the output sums are fp32.  FE_BF16: bf16 products with fp32
 * accumulation, probabilities rounded to bf16 for the product with the values (with out_rest, dense own rows and
 * T + L <= 256: to two bf16, 16 bits).  FE_F32: operands in three bf16 parts whose sum they are, products good to
 * 2^-21; an infinity inside the lengths may give NaN where the fp32 product with it would be infinite.
 * A list's outputs do not depend on the values of other lists, finite or not: they have the same bits.  Results have the
 * same bits from call to call.
 *
 * Workspace: fe_prefix_workspace_size(a, 0) bytes (may be 0: then ws is not read).
 *
 * Errors: FE_EINVAL for a NULL or misaligned pointer, B, K, S, heads below 1, T or L below 0, n_heads not a
 * multiple of n_kv_heads, strides too short or not multiples of 16 bytes, L not a multiple of page_rows, a
 * scale that is not finite, an unknown dtype, a workspace that is too small; FE_EUNSUPPORTED for dh outside
 * {32, 64, 128}, T or L above 4194304, B*K*S*n_heads, B*T or B*K*L above 1073741823, more than 16777215
 * workgroups of 64 rows or keys of one request and key head (the gradient: of partial sums, 1024 each, too), or
 * ctx_ld above 8388608.
 */
typedef struct {
  int32_t dtype;                        /* fe_dtype of q, keys, values and out */
  int32_t B, K, S;                      /* requests, lists per request, query rows per list */
  int32_t n_heads, n_kv_heads, dh;
  int32_t T, L;                         /* shared rows per request, own rows per list (capacities) */
  int32_t page_rows, n_pages;           /* page_rows = 0: dense own rows */
  int32_t causal;
  float scale;
  int32_t q_ld, ctx_ld, own_ld, out_ld; /* elements from one row to the next */
  const void* q;                        /* [B][K][S] rows of n_heads * dh */
  const void *ctx_k, *ctx_v;            /* [B][T] rows of n_kv_heads * dh */
  const void *own_k, *own_v;            /* [B][K][L] or [n_pages][page_rows] rows of n_kv_heads * dh */
  const int32_t* table;                 /* [B][K][L / page_rows] when paged */
  const int32_t* ctx_len;               /* [B], or NULL: T */
  const int32_t* q_len;                 /* [B][K], or NULL: S */
  const int32_t* own_len;               /* [B][K], or NULL: L */
  void* out;                            /* [B][K][S] rows of n_heads * dh */
  float* lse;                           /* [B][K][S][n_heads], or NULL (the gradient needs it) */
  void* out_rest;                       /* FE_BF16: [B][K][S][n_heads * dh] bytes, the eight bits that the rounding of
                                           out cut (16-byte aligned), or NULL */
  void* ws;
  size_t ws_bytes;
} fe_prefix_args;
fe_status fe_prefix_workspace_size(const fe_prefix_args* a, int grad, size_t* bytes); /* reads sizes only */
fe_status fe_prefix_attention(const fe_prefix_args* a, void* stream);

/*
 * Gradients of fe_prefix_attention for d loss / d out = dout.  `a` holds the forward's arguments with its out and
 * lse (and out_rest: without it FE_BF16 takes D from the rounded out) and a workspace of
 * fe_prefix_workspace_size(a, 1) bytes; own rows must be dense (FE_EUNSUPPORTED otherwise).
 * With D = dout.out, dp = dout.v and ds = p (dp - D):
 *   dq = scale sum ds k,   dk = scale sum ds q,   dv = sum p dout,
 * where a key's sums run over every list (shared rows), row and head that reads it.  Every row of dq, of the shared
 * gradients [B][T] and of the own gradients [B][K][L] is written; rows outside the lengths are zero.  dout
 * rows i >= q_len are not read into anything.  Sums are fp32, in a fixed order without atomics, rounded
 * once; FE_BF16 rounds p and ds to bf16 for the products (own keys' gradients:
 * to two bf16, 16 bits).  Values inside the lengths have to be finite: one that is not may reach the gradients
 * of the other lists of its request.
 * dctx_k, dctx_v (own: down_k, down_v) may be NULL only when T (L) is 0.
 */
typedef struct {
  const void* dout; int32_t dout_ld;    /* [B][K][S] rows of n_heads * dh */
  int32_t dq_ld, dctx_ld, down_ld;
  void* dq;                             /* [B][K][S] */
  void *dctx_k, *dctx_v;                /* [B][T] */
  void *down_k, *down_v;                /* [B][K][L] */
} fe_prefix_grads;
fe_status fe_prefix_attention_grad(const fe_prefix_args* a, const fe_prefix_grads* g, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* FLASHEVAL_PREFIX_H */

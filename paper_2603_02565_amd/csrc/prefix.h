// Launch descriptors of the shared-prefix attention and paged-cache kernels (flasheval_prefix.h).
#pragma once

#include "fe_common.h"
#include "flasheval_prefix.h"

constexpr int kPrefixMaxLen = 1 << 22;   // T and L: a tile's packed own rows (256 lists) stay in int32

// One attention call as its kernels see it.  The query rows of a (request, key head) are numbered
// r = (k S + s) G + hg < R with G = n_heads / n_kv_heads, so the rows that share keys are adjacent.
struct PrefixArgs {
  const void *q, *ctx_k, *ctx_v, *own_k, *own_v;
  const int32_t *table, *ctx_len, *q_len, *own_len;
  void* out; float* lse;
  signed char* out_rest;                // bf16: the eight bits below out's, dense rows (or nullptr)
  int B, K, S, Hq, Hkv, dh, T, L, page_rows, n_pages, causal;
  int q_ld, ctx_ld, own_ld, out_ld;
  float scale;
  int G, R;
  int tiles, splits;                    // row tiles per (request, key head); key ranges per tile
  // Forward, splits > 1: B * splits ranges in all; by_length: a request has as many of them as its share of the keys
  // says, its own rows taken as own_chunks chunks of 64.
  int by_length, own_chunks;
  float *part_o, *part_ml;              // splits > 1: [B*splits][K*S*Hq][dh] sums, [..][2] maximum and sum; dq: its sums
};

// The gradient's further tensors.
struct PrefixGradArgs {
  PrefixArgs f;
  const void* dout; int dout_ld;
  void *dq, *dctx_k, *dctx_v, *down_k, *down_v;
  int dq_ld, dctx_ld, down_ld;
  float4* rows;                         // [B][Hkv][R]: what the products need of every row
  int ctx_tiles, own_tiles;             // key tiles of the shared rows / of the own rows per (request, key head)
  int ctx_splits, own_splits;           // row ranges per shared / own key tile
  float *part_ctx, *part_own;           // their partial sums [splits][keys][2][dh]
};

// Row tiles, key ranges and partial-sum bytes of a forward call: functions of the sizes alone.
struct PrefixPlan { int rows, tiles, splits, by_length, own_chunks; size_t part_bytes; };
PrefixPlan prefix_plan(const fe_prefix_args& a);
hipError_t launch_prefix_fwd(PrefixArgs a, int dh, bool bf16_rows, const PrefixPlan& p, hipStream_t s);
// The same of a gradient call: dq's row tiles and key ranges, dk's and dv's key tiles and row ranges, scratch bytes.
struct PrefixGradPlan {
  int tiles, splits, ctx_tiles, own_tiles, ctx_splits, own_splits;
  size_t rows_bytes, dq_bytes, ctx_bytes, own_bytes;
  long long dkv_blocks, sum_blocks;     // workgroups
};
PrefixGradPlan prefix_grad_plan(const fe_prefix_args& a);
hipError_t launch_prefix_grad(const PrefixGradArgs& a, int dh, bool bf16_rows, const PrefixGradPlan& p, hipStream_t s);
hipError_t launch_advance(int32_t* len, const int32_t* new_len, int N, int S, hipStream_t s);   // lengths in place, after an append
hipError_t launch_cache_append(const fe_append_args& a, hipStream_t s);

// Launch descriptors of the 4-bit cache's kernels (flasheval_packed.h), and how a cached row is found.
#pragma once

#include "fe_common.h"
#include "flasheval_packed.h"

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kPackedMaxRows = 1 << 22;  // a sequence's capacity

// Division by a number that a launch does not change, as a multiplication: n magic >> shift, exact for 0 <= n < 2^31.
struct Divisor { unsigned magic; int shift; };
inline Divisor divisor(long long d) {
  int s = 0;
  while ((1LL << s) < d) ++s;
  return {(unsigned)((1ULL << (31 + s)) / d + 1), 31 + s};
}
FE_DEV int quotient(const Divisor& d, int n) { return (int)((unsigned long long)(unsigned)n * d.magic >> d.shift); }

// A cache as the kernels see it.
struct PackedCache {
  char* pages;
  long long page_ld;
  const int32_t *table, *len;
  int cols, page_rows, n_pages, cap, head_bytes;
  Divisor by_rows;                       // by page_rows
};
PackedCache packed_cache(const fe_packed_cache& c, int dh);

FE_DEV int packed_page(const PackedCache& c, int j) { return quotient(c.by_rows, j); }
FE_DEV int packed_len(const PackedCache& c, int s) { return min(max(c.len[s], 0), c.cap); }

// Eight columns from four bytes of codes and the block's power of two.
FE_DEV bf16x8 values8(unsigned w, float unit) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
FE_DEV float unit_of(unsigned scale) { return __uint_as_float(scale << 23); }   // 255: NaN from the conversion

// The attention's and the weights' arguments.  The query rows of a (request, key head) are numbered r = (k S + s) G + hg < R
// with G = Hq / Hkv: rows that share keys are adjacent.
struct PackedArgs {
  PackedCache ctx, own;                  // cap = 0: none
  const void* q;
  const int32_t* q_len;
  void* out;
  float* lse;
  int B, K, S, Hq, Hkv, G, R, causal, q_ld, out_ld;
  float scale;
  Divisor by_sg, by_g;                   // by S G and by G
  int tiles, splits;                     // row tiles per (request, key head); key ranges per tile
  // splits > 1: B * splits ranges in all; by_length: a request has as many of them as its share of the keys says, its own
  // rows taken as own_chunks chunks of 64
  int by_length, own_chunks;
  float *part_o, *part_ml;               // splits > 1: [B * splits][K S Hq][dh] sums, [..][2] maximum and sum
  long long lse_b;                       // the weights' log sum of (b, k, s, h): lse + b lse_b + k lse_k + s lse_s + h lse_h
  unsigned lse_k, lse_s, lse_h;          // a request's less than 2^31 apart
  const float *ctx_w, *own_w;            // weights
  float *ctx_w_out, *own_w_out;
  int ctx_keys, own_keys, ctx_splits, own_splits;     // key ranges, and row ranges, per (sequence, key head)
  int keys_by_length;                    // the shared keys' ranges, as above
  float *part_ctx, *part_own;            // [splits][N][Hkv][cap]
};

struct PackedPlan { int waves, wide, tiles, splits, by_length, own_chunks; size_t part_bytes; };   // waves: those that share a chunk
PackedPlan packed_plan(const fe_packed_args& a);
struct PackedWeighPlan {
  int ctx_keys, own_keys, ctx_splits, own_splits, keys_by_length;
  size_t ctx_bytes, own_bytes;
  long long blocks, sum_blocks;
};
PackedWeighPlan packed_weigh_plan(const fe_packed_args& a);

hipError_t launch_packed_attention(const PackedArgs& a, int dh, bool bf16_rows, const PackedPlan& p, hipStream_t s);
hipError_t launch_packed_weights(const PackedArgs& a, int dh, bool bf16_rows, hipStream_t s);
hipError_t launch_packed_append(const fe_packed_append_args& a, hipStream_t s);
hipError_t launch_packed_read(const fe_packed_read_args& a, hipStream_t s);
hipError_t launch_packed_evict(const fe_packed_evict_args& a, hipStream_t s);

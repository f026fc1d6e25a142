// C ABI of the 4-bit cache: argument checks and launches (flasheval_packed.h).
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "packed.h"

fe_status fe_report(fe_status st, const char* msg);

namespace {

fe_status pfail(fe_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return fe_report(st, buf);
}

bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
constexpr long long kInt32 = 0x7fffffffLL, kMaxGrid = (1 << 24) - 1;
bool stride_ok(int ld, long long width, int dtype) { return ld >= width && ld % (dtype == FE_BF16 ? 8 : 4) == 0; }
long long head_bytes(long long page_rows, int dh) { return (page_rows * (dh + dh / 16) + 15) / 16 * 16; }

fe_status check_head(int dh, int n_kv_heads) {
  if (n_kv_heads < 1) return pfail(FE_EINVAL, "n_kv_heads must be >= 1");
  if (dh != 32 && dh != 64 && dh != 128) return pfail(FE_EUNSUPPORTED, "head width %d not in {32,64,128}", dh);
  return FE_OK;
}
fe_status check_dtype(int dtype) {
  if (dtype != FE_F32 && dtype != FE_BF16) return pfail(FE_EINVAL, "dtype %d is not FE_F32 or FE_BF16", dtype);
  return FE_OK;
}
// Sizes of a cache; its pointers are looked at by check_cache.
fe_status check_cache_sizes(const fe_packed_cache& c, const char* name) {
  if (c.N < 1 || c.cols < 1 || c.page_rows < 1 || c.n_pages < 1)
    return pfail(FE_EINVAL, "%s: sequences, columns, page_rows and n_pages must be >= 1", name);
  if ((long long)c.cols * c.page_rows > kPackedMaxRows)
    return pfail(FE_EUNSUPPORTED, "%s: a capacity of %lld rows above %d", name, (long long)c.cols * c.page_rows, kPackedMaxRows);
  if ((double)c.N * c.cols * c.page_rows > 1073741823.)
    return pfail(FE_EUNSUPPORTED, "%s: batch too large: more than 1073741823 rows", name);
  return FE_OK;
}
fe_status check_cache(const fe_packed_cache& c, int dh, int n_kv_heads, const char* name) {
  const fe_status st = check_cache_sizes(c, name);
  if (st != FE_OK) return st;
  if (!c.pages || !c.table || !c.len) return pfail(FE_EINVAL, "%s: pages, table or len is NULL", name);
  if (!aligned(c.pages, 16) || !aligned(c.table, 4) || !aligned(c.len, 4))
    return pfail(FE_EINVAL, "%s: pages must be 16-byte aligned, table and lengths 4-byte aligned", name);
  if (c.page_ld > kInt32) return pfail(FE_EUNSUPPORTED, "%s: pages of more than %lld bytes", name, kInt32);
  if (c.page_ld % 16 || c.page_ld < n_kv_heads * head_bytes(c.page_rows, dh))
    return pfail(FE_EINVAL, "%s: a page stride of %lld bytes is shorter than the page or not a multiple of 16", name,
                 (long long)c.page_ld);
  return FE_OK;
}

fe_status check_sizes(const fe_packed_args* a) {
  if (!a) return pfail(FE_EINVAL, "arguments are NULL");
  if (check_dtype(a->dtype) != FE_OK) return FE_EINVAL;
  if (a->B < 1 || a->K < 1 || a->S < 1 || a->n_heads < 1) return pfail(FE_EINVAL, "B, K, S and n_heads must be >= 1");
  const fe_status st = check_head(a->dh, a->n_kv_heads);
  if (st != FE_OK) return st;
  if (a->n_heads % a->n_kv_heads)
    return pfail(FE_EINVAL, "n_heads=%d is not a multiple of n_kv_heads=%d", a->n_heads, a->n_kv_heads);
  if ((a->ctx.N != 0 && a->ctx.N != a->B) || (a->own.N != 0 && a->own.N != (long long)a->B * a->K))
    return pfail(FE_EINVAL, "the shared cache has %d sequences for B=%d, the lists' %d for B*K=%lld", a->ctx.N, a->B, a->own.N,
                 (long long)a->B * a->K);
  for (const fe_packed_cache* c : {&a->ctx, &a->own}) {
    const fe_status sc = c->N ? check_cache_sizes(*c, c == &a->ctx ? "ctx" : "own") : FE_OK;
    if (sc != FE_OK) return sc;
  }
  const double rows = (double)a->B * a->K * a->S * a->n_heads;
  if (rows > 1073741823.) return pfail(FE_EUNSUPPORTED, "batch too large: more than 1073741823 rows");
  // the rows of a request in tiles of 32 at least, of 128 where there are more than 64
  const double G = a->n_heads / a->n_kv_heads, R = a->K * (double)a->S * G, pairs = (double)a->B * a->n_kv_heads;
  if (pairs * std::ceil(R / 128) > kMaxGrid || rows * (a->dh / 4) / 256 >= kMaxGrid)
    return pfail(FE_EUNSUPPORTED, "batch too large: more than %lld workgroups", kMaxGrid);
  return FE_OK;
}
fe_status check_call(const fe_packed_args* a) {
  const fe_status st = check_sizes(a);
  if (st != FE_OK) return st;
  if (!std::isfinite(a->scale)) return pfail(FE_EINVAL, "scale is not finite");
  if (!a->q) return pfail(FE_EINVAL, "q is NULL");
  for (const fe_packed_cache* c : {&a->ctx, &a->own}) {
    const fe_status sc = c->N ? check_cache(*c, a->dh, a->n_kv_heads, c == &a->ctx ? "ctx" : "own") : FE_OK;
    if (sc != FE_OK) return sc;
  }
  if (!aligned(a->q, 16) || !aligned(a->ws, 16)) return pfail(FE_EINVAL, "q and the workspace must be 16-byte aligned");
  if (!aligned(a->q_len, 4) || !aligned(a->lse, 4)) return pfail(FE_EINVAL, "q_len and lse must be 4-byte aligned");
  if (!stride_ok(a->q_ld, (long long)a->n_heads * a->dh, a->dtype))
    return pfail(FE_EINVAL, "q's row stride is shorter than its row or not a multiple of 16 bytes");
  return FE_OK;
}
fe_status check_weigh_grid(const PackedWeighPlan& p) {
  if (p.blocks > kMaxGrid || p.sum_blocks > kMaxGrid)
    return pfail(FE_EUNSUPPORTED, "batch too large: more than %lld workgroups", kMaxGrid);
  return FE_OK;
}

size_t up256(size_t n) { return (n + 255) & ~size_t(255); }

PackedArgs kernel_args(const fe_packed_args& a) {
  PackedArgs k{};
  k.ctx = packed_cache(a.ctx, a.dh);
  k.own = packed_cache(a.own, a.dh);
  k.q = a.q; k.q_len = a.q_len; k.out = a.out; k.lse = a.lse;
  k.B = a.B; k.K = a.K; k.S = a.S; k.Hq = a.n_heads; k.Hkv = a.n_kv_heads;
  k.G = a.n_heads / a.n_kv_heads;
  k.R = a.K * a.S * k.G;
  k.by_sg = divisor((long long)a.S * k.G);
  k.by_g = divisor(k.G);
  k.causal = a.causal != 0;
  k.q_ld = a.q_ld; k.out_ld = a.out_ld; k.scale = a.scale;
  k.ctx_w = a.ctx_w; k.own_w = a.own_w; k.ctx_w_out = a.ctx_w_out; k.own_w_out = a.own_w_out;
  return k;
}

// What an append's and a read's arguments have in common.
fe_status check_rows(const fe_packed_cache& c, int dtype, int S, int n_kv_heads, int dh) {
  if (check_dtype(dtype) != FE_OK) return FE_EINVAL;
  if (S < 1) return pfail(FE_EINVAL, "S must be >= 1");
  const fe_status st = check_head(dh, n_kv_heads);
  if (st != FE_OK) return st;
  const fe_status sc = check_cache(c, dh, n_kv_heads, "cache");
  if (sc != FE_OK) return sc;
  if ((long long)c.N * S > kMaxGrid) return pfail(FE_EUNSUPPORTED, "N*S=%lld rows above %lld", (long long)c.N * S, kMaxGrid);
  if ((long long)n_kv_heads * dh > kInt32 / 8) return pfail(FE_EINVAL, "sizes overflow int32");
  return FE_OK;
}

// lse_ld: strides of the log sums, nullptr: dense.
fe_status weigh(const fe_packed_args* a, const int64_t* lse_ld, void* stream) {
  const fe_status st = check_call(a);
  if (st != FE_OK) return st;
  if (!a->lse) return pfail(FE_EINVAL, "lse is NULL");
  if ((a->ctx_w == nullptr) != (a->ctx_w_out == nullptr) || (a->own_w == nullptr) != (a->own_w_out == nullptr))
    return pfail(FE_EINVAL, "weights and their output go together");
  if ((a->ctx_w && !a->ctx.N) || (a->own_w && !a->own.N)) return pfail(FE_EINVAL, "weights without their cache");
  if (!aligned(a->ctx_w, 4) || !aligned(a->own_w, 4) || !aligned(a->ctx_w_out, 4) || !aligned(a->own_w_out, 4))
    return pfail(FE_EINVAL, "weights must be 4-byte aligned");
  const int64_t n[4] = {a->B, a->K, a->S, a->n_heads}, dense[4] = {n[1] * n[2] * n[3], n[2] * n[3], n[3], 1};
  int64_t ld[4];                           // of an axis of one element: 0
  double span = 0;
  for (int i = 0; i < 4; ++i) {
    ld[i] = n[i] == 1 ? 0 : lse_ld ? lse_ld[i] : dense[i];
    if (ld[i] < 0) return pfail(FE_EINVAL, "a stride of lse is negative");
    if (i) span += (double)ld[i] * (n[i] - 1);
  }
  if (span > (double)kInt32 || (double)ld[0] * (n[0] - 1) > 1e15)
    return pfail(FE_EUNSUPPORTED, "log sums of a request lie more than %lld elements apart, or the requests' out of reach", kInt32);
  const PackedWeighPlan p = packed_weigh_plan(*a);
  if (check_weigh_grid(p) != FE_OK) return FE_EUNSUPPORTED;
  const size_t need = up256(p.ctx_bytes) + up256(p.own_bytes);
  if (need && (!a->ws || a->ws_bytes < need))
    return pfail(FE_EINVAL, "workspace of %zu bytes < %zu needed", a->ws ? a->ws_bytes : 0, need);
  PackedArgs k = kernel_args(*a);
  k.lse_b = ld[0];
  k.lse_k = (unsigned)ld[1]; k.lse_s = (unsigned)ld[2]; k.lse_h = (unsigned)ld[3];
  k.ctx_keys = p.ctx_keys; k.own_keys = p.own_keys;
  k.ctx_splits = p.ctx_splits; k.own_splits = p.own_splits;
  k.keys_by_length = p.keys_by_length;
  k.part_ctx = static_cast<float*>(a->ws);
  k.part_own = reinterpret_cast<float*>(static_cast<char*>(a->ws) + up256(p.ctx_bytes));
  const hipError_t e = launch_packed_weights(k, a->dh, a->dtype == FE_BF16, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? FE_OK : pfail(FE_EHIP, "attention weights launch failed: %s", hipGetErrorString(e));
}

}  // namespace

extern "C" {

fe_status fe_packed_page_bytes(int32_t page_rows, int32_t n_kv_heads, int32_t dh, size_t* bytes) {
  const fe_status st = check_head(dh, n_kv_heads);
  if (st != FE_OK) return st;
  if (page_rows < 1 || page_rows > kPackedMaxRows || !bytes) return pfail(FE_EINVAL, "page_rows=%d, or bytes is NULL", page_rows);
  *bytes = (size_t)n_kv_heads * head_bytes(page_rows, dh);
  return FE_OK;
}

fe_status fe_packed_append(const fe_packed_append_args* a, void* stream) {
  if (!a) return pfail(FE_EINVAL, "arguments are NULL");
  const fe_status st = check_rows(a->cache, a->dtype, a->S, a->n_kv_heads, a->dh);
  if (st != FE_OK) return st;
  if (a->q && a->n_heads < 1) return pfail(FE_EINVAL, "n_heads must be >= 1");
  if (a->rot < 0 || a->rot > a->dh || a->rot % 2)
    return pfail(FE_EINVAL, "rot=%d is not an even number in [0, %d]", a->rot, a->dh);
  if (a->rot % 16) return pfail(FE_EUNSUPPORTED, "rot=%d is not a multiple of 16", a->rot);
  if (!a->k || !a->v) return pfail(FE_EINVAL, "k or v is NULL");
  if ((a->q == nullptr) != (a->q_out == nullptr)) return pfail(FE_EINVAL, "q and q_out go together");
  if (a->q && a->q == a->q_out) return pfail(FE_EINVAL, "q_out must not be q");
  if (a->rot > 0 && !a->freq) return pfail(FE_EINVAL, "rot=%d without freq", a->rot);
  if (!aligned(a->k, 16) || !aligned(a->v, 16) || !aligned(a->q, 16) || !aligned(a->q_out, 16))
    return pfail(FE_EINVAL, "pointers must be 16-byte aligned");
  if (!aligned(a->freq, 8) || !aligned(a->new_len, 4) || !aligned(a->pos0, 4) || !aligned(a->len_out, 4) || !aligned(a->status, 4))
    return pfail(FE_EINVAL, "freq must be 8-byte aligned, lengths and status 4-byte aligned");
  const long long wk = (long long)a->n_kv_heads * a->dh, wq = a->q ? (long long)a->n_heads * a->dh : 0;
  if (!stride_ok(a->k_ld, wk, a->dtype) || !stride_ok(a->v_ld, wk, a->dtype) ||
      (a->q && (!stride_ok(a->q_ld, wq, a->dtype) || !stride_ok(a->q_out_ld, wq, a->dtype))))
    return pfail(FE_EINVAL, "a row stride is shorter than its row or not a multiple of 16 bytes");
  if (wq + 2 * wk > kInt32 / 16) return pfail(FE_EINVAL, "sizes overflow int32");
  const hipError_t e = launch_packed_append(*a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? FE_OK : pfail(FE_EHIP, "4-bit append launch failed: %s", hipGetErrorString(e));
}

fe_status fe_packed_read(const fe_packed_read_args* a, void* stream) {
  if (!a) return pfail(FE_EINVAL, "arguments are NULL");
  const fe_status st = check_rows(a->cache, a->dtype, a->S, a->n_kv_heads, a->dh);
  if (st != FE_OK) return st;
  if (!a->k && !a->v) return pfail(FE_EINVAL, "k and v are NULL");
  if (!aligned(a->k, 16) || !aligned(a->v, 16)) return pfail(FE_EINVAL, "pointers must be 16-byte aligned");
  if (!aligned(a->start, 4) || !aligned(a->count, 4)) return pfail(FE_EINVAL, "start and count must be 4-byte aligned");
  const long long wk = (long long)a->n_kv_heads * a->dh;
  if ((a->k && !stride_ok(a->k_ld, wk, a->dtype)) || (a->v && !stride_ok(a->v_ld, wk, a->dtype)))
    return pfail(FE_EINVAL, "a row stride is shorter than its row or not a multiple of 16 bytes");
  const double blocks = std::ceil((double)a->S * wk / 8 / 256) * a->cache.N;
  if (blocks > kMaxGrid) return pfail(FE_EUNSUPPORTED, "batch too large: more than %lld workgroups", kMaxGrid);
  const hipError_t e = launch_packed_read(*a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? FE_OK : pfail(FE_EHIP, "4-bit read launch failed: %s", hipGetErrorString(e));
}

fe_status fe_packed_workspace_size(const fe_packed_args* a, int weights, size_t* bytes) {
  const fe_status st = check_sizes(a);
  if (st != FE_OK) return st;
  if (!bytes) return pfail(FE_EINVAL, "bytes is NULL");
  if (!weights) {
    *bytes = packed_plan(*a).part_bytes;
    return FE_OK;
  }
  const PackedWeighPlan p = packed_weigh_plan(*a);
  *bytes = up256(p.ctx_bytes) + up256(p.own_bytes);
  return check_weigh_grid(p);
}

fe_status fe_packed_attention(const fe_packed_args* a, void* stream) {
  const fe_status st = check_call(a);
  if (st != FE_OK) return st;
  if (!a->out) return pfail(FE_EINVAL, "out is NULL");
  if (!aligned(a->out, 16)) return pfail(FE_EINVAL, "out must be 16-byte aligned");
  if (!stride_ok(a->out_ld, (long long)a->n_heads * a->dh, a->dtype))
    return pfail(FE_EINVAL, "out's row stride is shorter than its row or not a multiple of 16 bytes");
  const PackedPlan p = packed_plan(*a);
  if (p.part_bytes && (!a->ws || a->ws_bytes < p.part_bytes))
    return pfail(FE_EINVAL, "workspace of %zu bytes < %zu needed", a->ws ? a->ws_bytes : 0, p.part_bytes);
  PackedArgs k = kernel_args(*a);
  k.tiles = p.tiles;
  k.splits = p.splits;
  k.by_length = p.by_length;
  k.own_chunks = p.own_chunks;
  if (p.part_bytes) {
    k.part_o = static_cast<float*>(a->ws);
    k.part_ml = k.part_o + (size_t)p.splits * a->B * a->K * a->S * a->n_heads * a->dh;
  }
  const hipError_t e = launch_packed_attention(k, a->dh, a->dtype == FE_BF16, p, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? FE_OK : pfail(FE_EHIP, "4-bit attention launch failed: %s", hipGetErrorString(e));
}

fe_status fe_packed_weights(const fe_packed_args* a, void* stream) { return weigh(a, nullptr, stream); }

fe_status fe_packed_weights_strided(const fe_packed_args* a, const int64_t lse_ld[4], void* stream) {
  if (!lse_ld) return pfail(FE_EINVAL, "lse_ld is NULL");
  return weigh(a, lse_ld, stream);
}

fe_status fe_packed_evict(const fe_packed_evict_args* a, void* stream) {
  if (!a) return pfail(FE_EINVAL, "arguments are NULL");
  fe_status st = check_head(a->dh, a->n_kv_heads);
  if (st == FE_OK) st = check_cache(a->from, a->dh, a->n_kv_heads, "from");
  if (st == FE_OK) st = check_cache(a->to, a->dh, a->n_kv_heads, "to");
  if (st != FE_OK) return st;
  if (a->to.N != a->from.N) return pfail(FE_EINVAL, "caches of %d and %d sequences", a->from.N, a->to.N);
  if (a->from.table == a->to.table || a->from.len == a->to.len)
    return pfail(FE_EINVAL, "`to` needs a table and lengths of its own");
  if (a->keep < 1 || a->first < 0 || a->recent < 0) return pfail(FE_EINVAL, "keep must be >= 1, first and recent >= 0");
  if (a->keep > (long long)a->to.cols * a->to.page_rows)
    return pfail(FE_EINVAL, "keep=%d above the capacity of %lld rows", a->keep, (long long)a->to.cols * a->to.page_rows);
  if (!a->weight || !a->kept) return pfail(FE_EINVAL, "weight or kept is NULL");
  if (!aligned(a->weight, 4) || !aligned(a->weight_out, 4) || !aligned(a->kept, 4) || !aligned(a->status, 4))
    return pfail(FE_EINVAL, "weights, kept and status must be 4-byte aligned");
  if (a->weight_out) {                     // rows move while others are read
    const auto from = reinterpret_cast<uintptr_t>(a->weight), to = reinterpret_cast<uintptr_t>(a->weight_out);
    const uintptr_t heads = 4ull * a->from.N * a->n_kv_heads;
    if (from < to + heads * a->to.cols * a->to.page_rows && to < from + heads * a->from.cols * a->from.page_rows)
      return pfail(FE_EINVAL, "weight_out overlaps weight");
  }
  const double rows = std::ceil((double)a->keep * (a->dh / 32) / 256);
  if ((double)a->from.N * a->n_kv_heads * rows > kMaxGrid || (double)a->from.N * a->n_kv_heads * 1024 > 4294967295.)
    return pfail(FE_EUNSUPPORTED, "batch too large: more than %lld workgroups", kMaxGrid);
  const hipError_t e = launch_packed_evict(*a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? FE_OK : pfail(FE_EHIP, "eviction launch failed: %s", hipGetErrorString(e));
}

}  // extern "C"

// C ABI of the shared-prefix attention, its gradient and the paged-cache append: argument checks and
// launches (flasheval_prefix.h).
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "prefix.h"

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

// A row stride of `ld` elements holds `width` and keeps rows 16-byte aligned.
bool stride_ok(int ld, long long width, int dtype) { return ld >= width && ld % (dtype == FE_BF16 ? 8 : 4) == 0; }
// A chunk of 64 shared rows keeps its byte offsets in 32 bits.
constexpr int kMaxStride = 1 << 23;

fe_status check_sizes(const fe_prefix_args* a) {
  if (!a) return pfail(FE_EINVAL, "arguments are NULL");
  if (a->dtype != FE_F32 && a->dtype != FE_BF16) return pfail(FE_EINVAL, "dtype %d is not FE_F32 or FE_BF16", a->dtype);
  if (a->B < 1 || a->K < 1 || a->S < 1 || a->n_heads < 1 || a->n_kv_heads < 1)
    return pfail(FE_EINVAL, "B, K, S, n_heads and n_kv_heads must be >= 1");
  if (a->T < 0 || a->L < 0) return pfail(FE_EINVAL, "T and L must be >= 0");
  if (a->n_heads % a->n_kv_heads)
    return pfail(FE_EINVAL, "n_heads=%d is not a multiple of n_kv_heads=%d", a->n_heads, a->n_kv_heads);
  if (a->page_rows < 0 || (a->page_rows > 0 && a->n_pages < 1))
    return pfail(FE_EINVAL, "page_rows=%d, n_pages=%d", a->page_rows, a->n_pages);
  if (a->page_rows > 0 && a->L % a->page_rows)
    return pfail(FE_EINVAL, "L=%d is not a multiple of page_rows=%d", a->L, a->page_rows);
  if (a->dh != 32 && a->dh != 64 && a->dh != 128) return pfail(FE_EUNSUPPORTED, "head width %d not in {32,64,128}", a->dh);
  if (a->T > kPrefixMaxLen || a->L > kPrefixMaxLen)
    return pfail(FE_EUNSUPPORTED, "T=%d or L=%d above %d", a->T, a->L, kPrefixMaxLen);
  const double most = 1073741823., lists = (double)a->B * a->K;
  if (lists * a->S * a->n_heads > most || (double)a->B * a->T > most || lists * a->L > most)
    return pfail(FE_EUNSUPPORTED, "batch too large: more than %.0f rows", most);
  // every launch of the forward, and the gradient's unsplit: a grid of 256 threads a workgroup holds 2^24 - 1 of them
  const double pairs = (double)a->B * a->n_kv_heads, G = a->n_heads / a->n_kv_heads;
  const double tiles = std::floor(((double)a->K * a->S * G + 63) / 64);
  const double keys = std::floor((a->T + 63) / 64.) + std::floor(((double)a->K * a->L + 63) / 64);
  if (pairs * tiles > kMaxGrid || pairs * keys > kMaxGrid || lists * a->S * a->n_heads * (a->dh / 4) / 256 >= kMaxGrid)
    return pfail(FE_EUNSUPPORTED, "batch too large: more than %lld workgroups", kMaxGrid);
  return FE_OK;
}

fe_status check_forward(const fe_prefix_args* a) {
  const fe_status st = check_sizes(a);
  if (st != FE_OK) return st;
  const long long wq = (long long)a->n_heads * a->dh, wk = (long long)a->n_kv_heads * a->dh;
  if (!std::isfinite(a->scale)) return pfail(FE_EINVAL, "scale is not finite");
  if (!a->q || !a->out) return pfail(FE_EINVAL, "q or out is NULL");
  if (a->T > 0 && (!a->ctx_k || !a->ctx_v)) return pfail(FE_EINVAL, "ctx_k or ctx_v is NULL");
  if (a->L > 0 && (!a->own_k || !a->own_v)) return pfail(FE_EINVAL, "own_k or own_v is NULL");
  if (a->L > 0 && a->page_rows > 0 && !a->table) return pfail(FE_EINVAL, "page table is NULL");
  if (!aligned(a->q, 16) || !aligned(a->out, 16) || !aligned(a->ctx_k, 16) || !aligned(a->ctx_v, 16) ||
      !aligned(a->own_k, 16) || !aligned(a->own_v, 16) || !aligned(a->out_rest, 16) || !aligned(a->ws, 16))
    return pfail(FE_EINVAL, "pointers must be 16-byte aligned");
  if (!aligned(a->table, 4) || !aligned(a->ctx_len, 4) || !aligned(a->q_len, 4) || !aligned(a->own_len, 4) ||
      !aligned(a->lse, 4))
    return pfail(FE_EINVAL, "tables, lengths and lse must be 4-byte aligned");
  if (!stride_ok(a->q_ld, wq, a->dtype) || !stride_ok(a->out_ld, wq, a->dtype) ||
      (a->T > 0 && !stride_ok(a->ctx_ld, wk, a->dtype)) || (a->L > 0 && !stride_ok(a->own_ld, wk, a->dtype)))
    return pfail(FE_EINVAL, "a row stride is shorter than its row or not a multiple of 16 bytes");
  if (a->T > 0 && a->ctx_ld > kMaxStride) return pfail(FE_EUNSUPPORTED, "ctx_ld=%d above %d", a->ctx_ld, kMaxStride);
  return FE_OK;
}

// The gradient's launches, split.
fe_status check_grid(const PrefixGradPlan& p) {
  if (p.dkv_blocks > kMaxGrid || p.sum_blocks > kMaxGrid)
    return pfail(FE_EUNSUPPORTED, "batch too large for the gradient: more than %lld workgroups", kMaxGrid);
  return FE_OK;
}

size_t up256(size_t n) { return (n + 255) & ~size_t(255); }
size_t grad_bytes(const PrefixGradPlan& p) {
  return up256(p.rows_bytes) + up256(p.dq_bytes) + up256(p.ctx_bytes) + up256(p.own_bytes);
}

PrefixArgs kernel_args(const fe_prefix_args& a) {
  PrefixArgs k{};
  k.q = a.q; k.ctx_k = a.ctx_k; k.ctx_v = a.ctx_v; k.own_k = a.own_k; k.own_v = a.own_v;
  k.table = a.table; k.ctx_len = a.ctx_len; k.q_len = a.q_len; k.own_len = a.own_len;
  k.out = a.out; k.lse = a.lse; k.out_rest = a.dtype == FE_BF16 ? static_cast<signed char*>(a.out_rest) : nullptr;
  k.B = a.B; k.K = a.K; k.S = a.S; k.Hq = a.n_heads; k.Hkv = a.n_kv_heads; k.dh = a.dh; k.T = a.T; k.L = a.L;
  k.page_rows = a.page_rows; k.n_pages = a.n_pages; k.causal = a.causal != 0;
  k.q_ld = a.q_ld; k.ctx_ld = a.ctx_ld; k.own_ld = a.own_ld; k.out_ld = a.out_ld;
  k.scale = a.scale;
  k.G = a.n_heads / a.n_kv_heads;
  k.R = a.K * a.S * k.G;
  k.tiles = k.splits = 1;
  return k;
}

}  // namespace

extern "C" {

fe_status fe_prefix_workspace_size(const fe_prefix_args* a, int grad, size_t* bytes) {
  const fe_status st = check_sizes(a);
  if (st != FE_OK) return st;
  if (!bytes) return pfail(FE_EINVAL, "bytes is NULL");
  if (grad && a->page_rows > 0) return pfail(FE_EUNSUPPORTED, "the gradient takes dense own rows");
  if (!grad) {
    *bytes = prefix_plan(*a).part_bytes;
    return FE_OK;
  }
  const PrefixGradPlan p = prefix_grad_plan(*a);
  *bytes = grad_bytes(p);
  return check_grid(p);
}

fe_status fe_prefix_attention(const fe_prefix_args* a, void* stream) {
  const fe_status st = check_forward(a);
  if (st != FE_OK) return st;
  const PrefixPlan p = prefix_plan(*a);
  if (p.part_bytes && (!a->ws || a->ws_bytes < p.part_bytes))
    return pfail(FE_EINVAL, "workspace of %zu bytes < %zu needed", a->ws ? a->ws_bytes : 0, p.part_bytes);
  PrefixArgs k = kernel_args(*a);
  if (p.part_bytes) {
    k.part_o = static_cast<float*>(a->ws);
    k.part_ml = k.part_o + (size_t)p.splits * a->B * a->K * a->S * a->n_heads * a->dh;
  }
  const hipError_t e = launch_prefix_fwd(k, a->dh, a->dtype == FE_BF16, p, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? FE_OK : pfail(FE_EHIP, "shared-prefix attention launch failed: %s", hipGetErrorString(e));
}

fe_status fe_prefix_attention_grad(const fe_prefix_args* a, const fe_prefix_grads* g, void* stream) {
  const fe_status st = check_forward(a);
  if (st != FE_OK) return st;
  if (!g) return pfail(FE_EINVAL, "gradient arguments are NULL");
  if (a->page_rows > 0) return pfail(FE_EUNSUPPORTED, "the gradient takes dense own rows");
  if (!a->lse || !g->dout || !g->dq) return pfail(FE_EINVAL, "lse, dout or dq is NULL");
  if (a->T > 0 && (!g->dctx_k || !g->dctx_v)) return pfail(FE_EINVAL, "dctx_k or dctx_v is NULL");
  if (a->L > 0 && (!g->down_k || !g->down_v)) return pfail(FE_EINVAL, "down_k or down_v is NULL");
  if (!aligned(g->dout, 16) || !aligned(g->dq, 16) || !aligned(g->dctx_k, 16) || !aligned(g->dctx_v, 16) ||
      !aligned(g->down_k, 16) || !aligned(g->down_v, 16))
    return pfail(FE_EINVAL, "pointers must be 16-byte aligned");
  const long long wq = (long long)a->n_heads * a->dh, wk = (long long)a->n_kv_heads * a->dh;
  if (!stride_ok(g->dout_ld, wq, a->dtype) || !stride_ok(g->dq_ld, wq, a->dtype) ||
      (a->T > 0 && !stride_ok(g->dctx_ld, wk, a->dtype)) || (a->L > 0 && !stride_ok(g->down_ld, wk, a->dtype)))
    return pfail(FE_EINVAL, "a row stride is shorter than its row or not a multiple of 16 bytes");
  const PrefixGradPlan p = prefix_grad_plan(*a);
  if (check_grid(p) != FE_OK) return FE_EUNSUPPORTED;
  const size_t need = grad_bytes(p);
  if (!a->ws || a->ws_bytes < need)
    return pfail(FE_EINVAL, "workspace of %zu bytes < %zu needed", a->ws ? a->ws_bytes : 0, need);
  PrefixGradArgs k{};
  k.f = kernel_args(*a);
  k.dout = g->dout; k.dout_ld = g->dout_ld;
  k.dq = g->dq; k.dctx_k = g->dctx_k; k.dctx_v = g->dctx_v; k.down_k = g->down_k; k.down_v = g->down_v;
  k.dq_ld = g->dq_ld; k.dctx_ld = g->dctx_ld; k.down_ld = g->down_ld;
  char* ws = static_cast<char*>(a->ws);
  auto take = [&](size_t bytes) {
    char* at = ws;
    ws += up256(bytes);
    return reinterpret_cast<float*>(at);
  };
  k.rows = reinterpret_cast<float4*>(take(p.rows_bytes));
  k.f.part_o = take(p.dq_bytes);
  k.part_ctx = take(p.ctx_bytes);
  k.part_own = take(p.own_bytes);
  const hipError_t e = launch_prefix_grad(k, a->dh, a->dtype == FE_BF16, p, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? FE_OK : pfail(FE_EHIP, "shared-prefix gradient launch failed: %s", hipGetErrorString(e));
}

fe_status fe_cache_append(const fe_append_args* a, void* stream) {
  if (!a) return pfail(FE_EINVAL, "arguments are NULL");
  if (a->dtype != FE_F32 && a->dtype != FE_BF16) return pfail(FE_EINVAL, "dtype %d is not FE_F32 or FE_BF16", a->dtype);
  if (a->N < 1 || a->S < 1 || a->n_kv_heads < 1 || a->page_rows < 1 || a->n_pages < 1 || a->table_cols < 1 ||
      (a->q && a->n_heads < 1))
    return pfail(FE_EINVAL, "N, S, heads, page_rows, n_pages and table_cols must be >= 1");
  if (a->dh != 32 && a->dh != 64 && a->dh != 128) return pfail(FE_EUNSUPPORTED, "head width %d not in {32,64,128}", a->dh);
  if (a->rot < 0 || a->rot > a->dh || a->rot % 2)
    return pfail(FE_EINVAL, "rot=%d is not an even number in [0, %d]", a->rot, a->dh);
  if (a->rot % 16) return pfail(FE_EUNSUPPORTED, "rot=%d is not a multiple of 16", a->rot);
  if (!a->k || !a->v || !a->k_pages || !a->v_pages || !a->table || !a->len) return pfail(FE_EINVAL, "NULL pointer argument");
  if ((a->q == nullptr) != (a->q_out == nullptr)) return pfail(FE_EINVAL, "q and q_out go together");
  if (a->rot > 0 && !a->freq) return pfail(FE_EINVAL, "rot=%d without freq", a->rot);
  if (!aligned(a->k, 16) || !aligned(a->v, 16) || !aligned(a->k_pages, 16) || !aligned(a->v_pages, 16) ||
      !aligned(a->q, 16) || !aligned(a->q_out, 16))
    return pfail(FE_EINVAL, "pointers must be 16-byte aligned");
  if (!aligned(a->freq, 8) || !aligned(a->table, 4) || !aligned(a->len, 4) || !aligned(a->new_len, 4) ||
      !aligned(a->pos0, 4) || !aligned(a->len_out, 4) || !aligned(a->status, 4))
    return pfail(FE_EINVAL, "freq must be 8-byte aligned, tables, lengths and status 4-byte aligned");
  const long long wk = (long long)a->n_kv_heads * a->dh, wq = a->q ? (long long)a->n_heads * a->dh : 0;
  if (!stride_ok(a->k_ld, wk, a->dtype) || !stride_ok(a->v_ld, wk, a->dtype) || !stride_ok(a->page_ld, wk, a->dtype) ||
      (a->q && (!stride_ok(a->q_ld, wq, a->dtype) || !stride_ok(a->q_out_ld, wq, a->dtype))))
    return pfail(FE_EINVAL, "a row stride is shorter than its row or not a multiple of 16 bytes");
  if ((long long)a->N * a->S > kInt32 || (long long)a->table_cols * a->page_rows > kInt32 || wq + 2 * wk > kInt32 / 4)
    return pfail(FE_EINVAL, "sizes overflow int32");
  if ((long long)a->N * a->S > kMaxGrid)
    return pfail(FE_EUNSUPPORTED, "N*S=%lld rows above %lld", (long long)a->N * a->S, kMaxGrid);
  const hipError_t e = launch_cache_append(*a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? FE_OK : pfail(FE_EHIP, "cache append launch failed: %s", hipGetErrorString(e));
}

}  // extern "C"

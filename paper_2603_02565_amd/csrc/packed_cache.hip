// The 4-bit cache's own calls: append, read and eviction (flasheval_packed.h).
#include <algorithm>

#include "packed.h"
#include "prefix.h"

namespace {

template <typename T> struct Vec8;
template <> struct Vec8<bf16> { typedef bf16x8 type; };
template <> struct Vec8<float> { typedef f32x8 type; };

constexpr unsigned char kNoNumber = 255;  // the scale of a block of NaN

FE_DEV int quad_max(int v) {              // over the four lanes of a block
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0xb1, 0xf, 0xf, true));
  return max(v, __builtin_amdgcn_update_dpp(0, v, 0x4e, 0xf, 0xf, true));
}

// x in fp32 for a rounding that follows: what does not fit moves to the odd neighbour, which no border between two results
// is, so that both roundings together are one.
FE_DEV float to_odd(double x) {
  const double a = fabs(x);
  const float f = (float)a;
  const double back = (double)f;
  unsigned b = __float_as_uint(f);
  if (back > a) b -= 1;
  if (back != a) b |= 1;
  return copysignf(__uint_as_float(b), (float)x);
}
template <typename T> FE_DEV T rounded(double x);
template <> FE_DEV float rounded<float>(double x) { return (float)x; }
template <> FE_DEV bf16 rounded<bf16>(double x) { return (bf16)to_odd(x); }

// Eight codes of a block that the lanes of a quad share (lane i: columns 8 i ..), and the block's scale.  The magnitudes'
// leading bits as integers order as they do; 1.5 * 2^(E - bias) is the largest whose scale is 2 below its exponent.
FE_DEV unsigned codes8(const float (&f)[8], float unit) {
  unsigned w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[0] * unit, f[1] * unit, 1.f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2] * unit, f[3] * unit, 1.f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4] * unit, f[5] * unit, 1.f, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6] * unit, f[7] * unit, 1.f, 3);
}
FE_DEV unsigned held(const float (&x)[8], unsigned char* scale) {
  int top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, (int)(__float_as_uint(x[i]) & 0x7fffffffu));
  top = quad_max(top);
  if (top >= 0x7f800000) {
    *scale = kNoNumber;
    return 0;
  }
  const int e = min(max((top >> 23) - 1 - ((top & 0x7fffff) <= 0x400000), 2), 252);
  *scale = (unsigned char)e;
  return codes8(x, __uint_as_float((unsigned)(254 - e) << 23));
}
FE_DEV unsigned held(const double (&x)[8], unsigned char* scale) {
  int top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const long long b = __double_as_longlong(x[i]);
    top = max(top, ((int)(b >> 32) & 0x7fffffff) | ((int)b != 0));     // a bit below the 20 kept ones counts as the last
  }
  top = quad_max(top);
  if (top >= 0x7ff00000) {
    *scale = kNoNumber;
    return 0;
  }
  const int e = min(max((top >> 20) - 897 - ((top & 0xfffff) <= 0x80000), 2), 252);
  *scale = (unsigned char)e;
  const double unit = __longlong_as_double((long long)(1150 - e) << 52);
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = to_odd(x[i] * unit);
  return codes8(f, 1.f);
}

constexpr int kTurns = 1024;              // sines and cosines in LDS
constexpr int kAppendRows = 64;           // rows of a workgroup

// One workgroup takes `rows` (a power of two) consecutive new rows of one sequence: sines and cosines of a row are
// formed once, in LDS, for all its heads; then every thread takes units of 8 columns, 4 lanes a block, consecutive
// units along a row, then rows, then heads, as the pages hold them.
// Bound: the vector unit (fp64 and the sines) beside HBM: 24 x 1000 rows of 24 heads of 128, bf16, 246 MB: 68 us, 3.6 TB/s.  The
// queries in fp32 60 us, but then a turned query may go to the number that is not the nearest.  128 rows of 24 heads of 64: 4.8 us,
// launch latency and a trip to memory.
template <typename T>
__global__ __launch_bounds__(256) void k_packed_append(fe_packed_append_args a, PackedCache c, int log_rows, int blocks) {
  typedef typename Vec8<T>::type V8;
  __shared__ double s_cos[kTurns], s_sin[kTurns];
  __shared__ long long s_page[kAppendRows];
  __shared__ int s_row[kAppendRows];
  const int tid = threadIdx.x, s = blockIdx.x / blocks, blk = blockIdx.x % blocks, rows = 1 << log_rows;
  const int n = a.new_len ? min(max(a.new_len[s], 0), a.S) : a.S;
  const int len = max(c.len[s], 0);
  const long long pos0 = (a.pos0 ? a.pos0[s] : 0) + (long long)len;
  const int32_t* tab = c.table + (long long)s * c.cols;
  const int i0 = blk * rows, m = min(rows, n - i0), np = a.rot / 2;

  const int hq = a.q ? a.n_heads : 0, heads = hq + 2 * a.n_kv_heads;
  const int log_units = a.dh == 32 ? 2 : a.dh == 64 ? 3 : 4, units = 1 << log_units;
  // A unit and its pairs' other columns where they lie rot / 2 apart: requested one ahead, the first before the sines.
  V8 own{}, other{};
  auto fetch = [&](int e) __attribute__((always_inline)) {
    const int x = e & (units - 1), r = e >> log_units & (rows - 1), hh = e >> (log_rows + log_units);
    if (r >= m || hh >= heads) return;
    const long long row = (long long)s * a.S + i0 + r;
    const bool is_q = hh < hq, is_v = hh >= hq + a.n_kv_heads;
    const T* src = is_q ? static_cast<const T*>(a.q) + row * a.q_ld : is_v ? static_cast<const T*>(a.v) + row * a.v_ld
                                                                          : static_cast<const T*>(a.k) + row * a.k_ld;
    src += (is_q ? hh : is_v ? hh - hq - a.n_kv_heads : hh - hq) * a.dh;
    own = *reinterpret_cast<const V8*>(src + 8 * x);
    if (!is_v && 8 * x < a.rot && !a.neighbours) other = *reinterpret_cast<const V8*>(src + (8 * x >= np ? 8 * x - np : 8 * x + np));
  };
  fetch(tid);

  if (tid < m) {
    const long long j = (long long)len + i0 + tid;
    long long at = -1;
    int row = 0;
    if (j < c.cap) {
      const int p = packed_page(c, (int)j), page = tab[p];
      row = (int)j - p * c.page_rows;
      if (page >= 0 && page < c.n_pages) at = (long long)page * c.page_ld;
    }
    s_page[tid] = at;
    s_row[tid] = row;
  }
  for (int e = tid; e < m * np; e += 256) {
    const int r = e / np;
    sincos((double)(pos0 + i0 + r) * a.freq[e - r * np], &s_sin[e], &s_cos[e]);
  }
  if (blk == 0 && a.status) {              // uniform over the workgroup: the pages of all n rows
    int bad = (long long)len + n > c.cap && n > 0;
    if (n > 0 && len < c.cap)
      for (int p = packed_page(c, len) + tid; p <= packed_page(c, (int)min((long long)len + n, (long long)c.cap) - 1); p += 256)
        bad |= tab[p] < 0 || tab[p] >= c.n_pages;
    bad = block_any<4>(bad);
    if (tid == 0) a.status[s] = bad ? FE_DEV_BAD_PAGE : 0;
  }
  __syncthreads();
  // every thread has read len[s]; with several workgroups a sequence a second launch advances it in place
  if (tid == 0 && blk == 0 && a.len_out && (a.len_out != c.len || blocks == 1))
    a.len_out[s] = (int)min((long long)len + n, 0x7fffffffLL);
  if (m <= 0) return;

  for (int e = tid; e < heads << (log_rows + log_units); e += 256) {
    const int x = e & (units - 1), r = e >> log_units & (rows - 1), hh = e >> (log_rows + log_units);
    const V8 mine = own, pair = other;
    fetch(e + 256);
    if (r >= m) continue;
    const long long row = (long long)s * a.S + i0 + r;
    const bool is_q = hh < hq, is_v = hh >= hq + a.n_kv_heads;
    const int h = is_q ? hh : is_v ? hh - hq - a.n_kv_heads : hh - hq;
    const long long page = s_page[r];
    if (!is_q && page < 0) continue;       // the same in a quad
    unsigned w;
    unsigned char scale;
    const bool turned = !is_v && 8 * x < a.rot, apart = turned && !a.neighbours;   // apart: the pair's columns lie rot / 2 apart
    const bool second = 8 * x >= np;
    const int c0 = !apart ? 4 * x : second ? 8 * x - np : 8 * x;       // the unit's first pair
    T* q_out = static_cast<T*>(a.q_out) + row * a.q_out_ld + h * a.dh + 8 * x;
    if (is_q && !turned) {
      *reinterpret_cast<V8*>(q_out) = mine;
      continue;
    }
    if (is_v || a.rot == 0) {
      float f[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = to_f32((T)mine[i]);
      w = held(f, &scale);
    } else {
      double y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = (double)to_f32((T)mine[i]);
      if (turned) {
        const double *cs = s_cos + r * np + c0, *sn = s_sin + r * np + c0;
        if (apart) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const double o = (double)to_f32((T)pair[i]);
            y[i] = y[i] * cs[i] + (second ? o * sn[i] : -o * sn[i]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const double u = y[2 * i], v = y[2 * i + 1];
            y[2 * i] = u * cs[i] - v * sn[i];
            y[2 * i + 1] = v * cs[i] + u * sn[i];
          }
        }
      }
      if (is_q) {
        V8 out;
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = rounded<T>(y[i]);
        *reinterpret_cast<V8*>(q_out) = out;
        continue;
      }
      w = held(y, &scale);
    }
    char* head = c.pages + page + (long long)h * c.head_bytes;
    const int at = (is_v ? c.page_rows : 0) + s_row[r];
    *reinterpret_cast<unsigned*>(head + ((long long)at << (log_units + 2)) + 4 * x) = w;
    if ((x & 3) == 0)
      head[(long long)c.page_rows * a.dh + ((long long)at << (log_units - 2)) + (x >> 2)] = (char)scale;
  }
}

FE_DEV void put8(bf16* p, bf16x8 v) { *reinterpret_cast<bf16x8*>(p) = v; }
FE_DEV void put8(float* p, bf16x8 v) {
  f32x8 w;
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = (float)v[i];
  *reinterpret_cast<f32x8*>(p) = w;
}

// A thread takes 8 columns of a row's head, of keys and of values: 4 bytes of codes each in, 16 or 32 bytes out, both in
// order.  Bound: HBM (4 x 8192 rows of 8 heads of 128, 170 MB: 28.5 us, 6.0 TB/s, partly from cache).
template <typename T>
__global__ __launch_bounds__(256) void k_packed_read(fe_packed_read_args a, PackedCache c, int blocks) {
  const int s = blockIdx.x / blocks, blk = blockIdx.x % blocks;
  const int log_units = a.dh == 32 ? 2 : a.dh == 64 ? 3 : 4;
  const int start = a.start ? max(a.start[s], 0) : 0;
  const int n = min(max(a.count ? a.count[s] : packed_len(c, s) - start, 0), a.S);
  const long long e = (long long)blk * 256 + threadIdx.x, per = (long long)a.n_kv_heads << log_units;
  const int i = (int)(e / per), rest = (int)(e - i * per), h = rest >> log_units, x = rest & ((1 << log_units) - 1);
  if (i >= n) return;
  const long long j = (long long)start + i, row = (long long)s * a.S + i;
  bf16x8 k{}, v{};
  if (j < c.cap) {
    const int p = packed_page(c, (int)j), page = c.table[(long long)s * c.cols + p], r = (int)j - p * c.page_rows;
    if (page >= 0 && page < c.n_pages) {
      const char* head = c.pages + page * c.page_ld + (long long)h * c.head_bytes;
      const long long at = ((long long)r << (log_units + 2)) + 4 * x, all = (long long)c.page_rows << (log_units + 2);
      const unsigned char* scale =
          reinterpret_cast<const unsigned char*>(head) + 2 * all + ((long long)r << (log_units - 2)) + (x >> 2);
      const unsigned kw = *reinterpret_cast<const unsigned*>(head + at), vw = *reinterpret_cast<const unsigned*>(head + all + at);
      k = values8(kw, unit_of(scale[0]));
      v = values8(vw, unit_of(scale[(long long)c.page_rows << (log_units - 2)]));
    }
  }
  if (a.k) put8(static_cast<T*>(a.k) + row * a.k_ld + h * a.dh + 8 * x, k);
  if (a.v) put8(static_cast<T*>(a.v) + row * a.v_ld + h * a.dh + 8 * x, v);
}

// The order of weights as that of integers; NaN (1) below every number, both zeros equal.  0 is left for what is no candidate,
// the greatest for what is certain.
FE_DEV unsigned order_of(float w) {
  if (w != w) return 1;
  const unsigned b = __float_as_uint(w == 0.f ? 0.f : w);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// What a sequence's first head writes for it: its length in `to`, whether rows in use have no page.  Uniform over NW waves.
template <int NW>
FE_DEV void evict_state(const fe_packed_evict_args& a, const PackedCache& from, const PackedCache& to, int s, int n, int m) {
  const int tid = threadIdx.x;
  if (tid == 0) const_cast<int32_t*>(to.len)[s] = m;
  if (!a.status) return;
  int bad = 0;
  if (n > 0)
    for (int p = tid; p <= packed_page(from, n - 1); p += NW * 64) {
      const int page = from.table[(long long)s * from.cols + p];
      bad |= page < 0 || page >= from.n_pages;
    }
  if (m > 0)
    for (int p = tid; p <= packed_page(to, m - 1); p += NW * 64) {
      const int page = to.table[(long long)s * to.cols + p];
      bad |= page < 0 || page >= to.n_pages;
    }
  bad = block_any<NW>(bad);
  if (tid == 0) a.status[s] = bad ? FE_DEV_BAD_PAGE : 0;
}

// Block x of kept row i of (sequence, head), row j of `from`: its keys and its values.
FE_DEV void move_block(const PackedCache& from, const PackedCache& to, int s, int h, int log_blocks, int i, int j, int x) {
  const int p = packed_page(from, j), t = packed_page(to, i);
  const int page = from.table[(long long)s * from.cols + p], to_page = to.table[(long long)s * to.cols + t];
  if (page < 0 || page >= from.n_pages || to_page < 0 || to_page >= to.n_pages) return;
  const char* src = from.pages + page * from.page_ld + (long long)h * from.head_bytes;
  char* dst = to.pages + to_page * to.page_ld + (long long)h * to.head_bytes;
  const long long b = ((long long)(j - p * from.page_rows) << log_blocks) + x, d = ((long long)(i - t * to.page_rows) << log_blocks) + x;
  const long long sn = (long long)from.page_rows << log_blocks, dn = (long long)to.page_rows << log_blocks;
  const u32x4 k = *reinterpret_cast<const u32x4*>(src + 16 * b), v = *reinterpret_cast<const u32x4*>(src + 16 * (sn + b));
  const char ks = src[32 * sn + b], vs = src[33 * sn + b];
  *reinterpret_cast<u32x4*>(dst + 16 * d) = k;
  *reinterpret_cast<u32x4*>(dst + 16 * (dn + d)) = v;
  dst[32 * dn + d] = ks;
  dst[33 * dn + d] = vs;
}

// Short sequences (64 E rows at most): one wave selects, all four move.  The m-th greatest order is found bit by bit: a ballot
// counts the candidates at or above a trial.  Bound: three trips to memory (1024 heads of 64 rows, 9 MB: 5.1 us; with the
// histograms below and a launch of its own for the move 48).
template <int E>
__global__ __launch_bounds__(256) void k_packed_evict_short(fe_packed_evict_args a, PackedCache from, PackedCache to) {
  __shared__ int s_kept[64 * E];
  const int tid = threadIdx.x, lane = tid & 63, s = blockIdx.x / a.n_kv_heads, h = blockIdx.x % a.n_kv_heads;
  const int n = packed_len(from, s), m = min(a.keep, n);
  const int first = min(a.first, m), recent = min(a.recent, m - first), lo = first, hi = n - recent;
  int32_t* kept = a.kept + (long long)blockIdx.x * a.keep;
  if (h == 0) evict_state<4>(a, from, to, s, n, m);
  for (int i = m + tid; i < a.keep; i += 256) kept[i] = -1;
  if (tid < 64) {
    const float* w = a.weight + (long long)blockIdx.x * from.cap;
    float v[E];
    unsigned o[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = e * 64 + lane < n ? w[e * 64 + lane] : 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = e * 64 + lane >= lo && e * 64 + lane < hi ? order_of(v[e]) : 0;
    int left = m - first - recent;
    unsigned cut = 0xffffffffu;            // no order is as great
    const bool all = m == n;
    if (!all && left > 0) {
      cut = 0;
      for (int bit = 31; bit >= 0; --bit) {
        const unsigned trial = cut | 1u << bit;
        int c = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) c += __popcll(__ballot(o[e] >= trial));
        if (c >= left) cut = trial;
      }
#pragma unroll
      for (int e = 0; e < E; ++e) left -= __popcll(__ballot(o[e] > cut));
    }
    const unsigned long long below = (1ull << lane) - 1;
    float* out = a.weight_out ? a.weight_out + (long long)blockIdx.x * to.cap : nullptr;
    int at = 0, equal = 0;                 // kept, and candidates equal to the cut, so far: the first `left` of these are kept
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int i = e * 64 + lane;
      const bool inside = i >= lo && i < hi, same = !all && inside && o[e] == cut;
      const unsigned long long eq = __ballot(same);
      const bool take = i < n && (all || !inside || o[e] > cut || (same && equal + __popcll(eq & below) < left));
      const unsigned long long got = __ballot(take);
      if (take) {
        const int d = at + __popcll(got & below);
        s_kept[d] = i;
        kept[d] = i;
        if (out) out[d] = v[e];
      }
      at += __popcll(got);
      equal += __popcll(eq);
    }
  }
  __syncthreads();
  const int log_blocks = a.dh == 32 ? 0 : a.dh == 64 ? 1 : 2;
#pragma unroll 2
  for (int e = tid; e < m << log_blocks; e += 256)
    move_block(from, to, s, h, log_blocks, e >> log_blocks, s_kept[e >> log_blocks], e & ((1 << log_blocks) - 1));
}

// Selects a (sequence, key head)'s rows.  Four passes over 8 bits each find the m-th greatest order among the candidates:
// a histogram in LDS, in 32 copies by lane so that equal digits, the rule among weights, do not meet in one word.  Then
// every wave walks its rows in order and numbers what is kept.  The orders of 1024 E rows stay in registers where they are
// all.  Rows that are kept in any case have the highest order, which no weight has, and what is no row the order 0.
// Bound: instructions of the one compute unit that a head has (32 heads of 32768 rows: 21.6 us, of which the loads take 4 and
// a pass 3; the last pass is left out where the third one ends on a digit that is kept whole, as among weights that
// hardly repeat it does; with it 1.8 more).  Above 32768 rows the weights are read again in every pass: 131072 rows, with the move of
// 32768, 205 us, where 32768 rows and 8192 take 37.
constexpr unsigned kCertain = 0xffffffffu;
template <int E>
__global__ __launch_bounds__(1024) void k_packed_select(fe_packed_evict_args a, PackedCache from, PackedCache to) {
  constexpr int NW = 16, NT = NW * 64, SEG = NT * E;
  __shared__ int s_hist[256 * 32];
  __shared__ int s_sum[256], s_kept[NW], s_equal[NW], s_digit, s_left, s_whole;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int s = blockIdx.x / a.n_kv_heads, h = blockIdx.x % a.n_kv_heads;
  const int n = packed_len(from, s), m = min(a.keep, n);
  const int first = min(a.first, m), recent = min(a.recent, m - first);
  const bool all = m == n;                 // uniform
  const int lo = first, hi = all ? 0 : n - recent, segments = (n + SEG - 1) / SEG;
  const float* w = a.weight + (long long)blockIdx.x * from.cap;
  int32_t* kept = a.kept + (long long)blockIdx.x * a.keep;

  if (h == 0) evict_state<NW>(a, from, to, s, n, m);
  for (int i = m + tid; i < a.keep; i += NT) kept[i] = -1;

  unsigned o[E];
  auto index = [&](int seg, int e) { return seg * SEG + (wave * E + e) * 64 + lane; };
  auto load = [&](int seg) __attribute__((always_inline)) {
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = w[min(index(seg, e), n - 1)];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int i = index(seg, e);
      o[e] = i >= lo && i < hi ? order_of(v[e]) : i < n ? kCertain : 0;
    }
  };
  unsigned cut = kCertain - 1;             // orders above it are kept, and the first `left` of those equal to it
  int left = 0;
  if (segments == 1) load(0);
  if (!all && m > first + recent) {
    cut = 0;
    left = m;
#pragma unroll 1
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256 * 32; i += NT) s_hist[i] = 0;
      __syncthreads();
      for (int seg = 0; seg < segments; ++seg) {
        if (segments > 1) load(seg);
        const unsigned differ = shift == 24 ? 0xffffffffu : (1u << (shift + 8)) - 1;   // a digit counts below the cut's
#pragma unroll
        for (int e = 0; e < E; ++e)
          if ((o[e] ^ cut) <= differ) atomicAdd(&s_hist[(o[e] >> shift & 255) * 32 + (lane & 31)], 1);
      }
      __syncthreads();
      {                                    // four threads a digit, each from another bank
        const int bin = tid >> 2, at = bin * 32 + (tid & 3) * 8;
        int c = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) c += s_hist[at + ((i + (bin >> 1)) & 7)];
        c += __builtin_amdgcn_update_dpp(0, c, 0xb1, 0xf, 0xf, true);
        c += __builtin_amdgcn_update_dpp(0, c, 0x4e, 0xf, 0xf, true);
        if ((tid & 3) == 0) s_sum[bin] = c;
      }
      __syncthreads();
      if (wave == 0) {                     // digits from the greatest: lane l has 255 - 4 l and the three below
        int c[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += c[i] = s_sum[255 - 4 * lane - i];
        int before = sum;
#pragma unroll
        for (int x = 1; x < 64; x *= 2) {
          const int u = __shfl_up(before, x);
          if (lane >= x) before += u;
        }
        before -= sum;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (before < left && before + c[i] >= left) {
            s_digit = 255 - 4 * lane - i;
            s_left = left - before;
            s_whole = before + c[i] == left;
          }
          before += c[i];
        }
      }
      __syncthreads();
      cut |= (unsigned)s_digit << shift;
      left = s_left;
      if (s_whole) {                       // all of that digit are kept; rows it has, and not what is no row, since m < n
        --cut;
        left = 0;
        break;
      }
    }
  }

  int kept_before = 0, equal_before = 0;   // in the segments before
  for (int seg = 0; seg < segments; ++seg) {
    if (segments > 1) load(seg);
    int n_kept = 0, n_equal = 0;           // the wave's rows above the cut, and equal to it
#pragma unroll
    for (int e = 0; e < E; ++e) {
      n_kept += __popcll(__ballot(o[e] > cut));
      n_equal += __popcll(__ballot(o[e] == cut));
      asm volatile("" : "+s"(n_kept), "+s"(n_equal));    // one row's ballots after the other's: all at once they would not fit
    }
    if (lane == 0) {
      s_kept[wave] = n_kept;
      s_equal[wave] = n_equal;
    }
    __syncthreads();
    int k0 = kept_before, e0 = equal_before, ks = 0, es = 0;
    for (int x = 0; x < NW; ++x) {
      if (x == wave) k0 += ks, e0 += es;
      ks += s_kept[x];
      es += s_equal[x];
    }
    int at = k0 + min(e0, left);           // of the equal ones the first `left` are kept
#pragma unroll
    for (int e = 0; e < E; ++e) {
      asm volatile("" : "+v"(o[e]));       // ballots are made again: kept, they would not fit the scalar registers
      const unsigned long long eq = __ballot(o[e] == cut);
      unsigned long long got = __ballot(o[e] > cut);
      if (eq)                              // uniform
        got |= __ballot((eq >> lane & 1) && e0 + (int)__builtin_amdgcn_mbcnt_hi((unsigned)(eq >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)eq, 0)) < left);
      if (got >> lane & 1) {
        const int d = at + (int)__builtin_amdgcn_mbcnt_hi((unsigned)(got >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)got, 0));
        kept[d] = index(seg, e);
      }
      at += __popcll(got);
      e0 += __popcll(eq);
    }
    kept_before += ks;
    equal_before += es;
    __syncthreads();
  }
}

// The kept rows: a thread takes one block, of keys and of values, the first of a row its weight as well.  Bound: HBM at 64
// contiguous bytes a row (4 x 8192 rows of 8 heads of 128, 71 MB: 24 us, 3.0 TB/s).
__global__ __launch_bounds__(256) void k_packed_move(fe_packed_evict_args a, PackedCache from, PackedCache to, int blocks) {
  const int sh = blockIdx.x / blocks, blk = blockIdx.x % blocks, s = sh / a.n_kv_heads, h = sh - s * a.n_kv_heads;
  const int log_blocks = a.dh == 32 ? 0 : a.dh == 64 ? 1 : 2;
  const int m = min(a.keep, packed_len(from, s));
  const int e = blk * 256 + threadIdx.x, i = e >> log_blocks, x = e & ((1 << log_blocks) - 1);
  if (i >= m) return;
  const int j = a.kept[(long long)sh * a.keep + i];
  if (x == 0 && a.weight_out) a.weight_out[(long long)sh * to.cap + i] = a.weight[(long long)sh * from.cap + j];
  move_block(from, to, s, h, log_blocks, i, j, x);
}

}  // namespace

PackedCache packed_cache(const fe_packed_cache& c, int dh) {
  PackedCache k{};
  k.pages = static_cast<char*>(c.pages);
  k.page_ld = c.page_ld;
  k.table = c.table;
  k.len = c.len;
  k.cols = c.cols;
  k.page_rows = c.page_rows;
  k.n_pages = c.n_pages;
  k.cap = c.N > 0 ? c.cols * c.page_rows : 0;
  if (c.N > 0) {
    k.head_bytes = (c.page_rows * (dh + dh / 16) + 15) / 16 * 16;
    k.by_rows = divisor(c.page_rows);
  }
  return k;
}

hipError_t launch_packed_append(const fe_packed_append_args& a, hipStream_t s) {
  const PackedCache c = packed_cache(a.cache, a.dh);
  const int units = ((a.q ? a.n_heads : 0) + 2 * a.n_kv_heads) * (a.dh / 8);
  // about 2048 units a workgroup, 8 a thread (24 x 1999 rows of 24 heads of 128: 512 units 112 us with the reading back, 1024 91,
  // 2048 82, 4096 84; 16 x 2048 rows of 24 heads of 64: 90, 77, 74, 76), and no more sines than the LDS tables hold
  const int fit = std::min({a.S, kAppendRows, a.rot ? kTurns / (a.rot / 2) : kAppendRows, 2048 / std::max(1, units)});
  int log_rows = 0;
  while (2 << log_rows <= fit) ++log_rows;
  const int rows = 1 << log_rows, blocks = (a.S + rows - 1) / rows;
  const dim3 grid((unsigned)((long long)blocks * a.cache.N));
  if (a.dtype == FE_BF16)
    hipLaunchKernelGGL(k_packed_append<bf16>, grid, dim3(256), 0, s, a, c, log_rows, blocks);
  else
    hipLaunchKernelGGL(k_packed_append<float>, grid, dim3(256), 0, s, a, c, log_rows, blocks);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && a.len_out == a.cache.len && a.len_out && blocks > 1) e = launch_advance(a.len_out, a.new_len, a.cache.N, a.S, s);
  return e;
}

hipError_t launch_packed_read(const fe_packed_read_args& a, hipStream_t s) {
  const PackedCache c = packed_cache(a.cache, a.dh);
  const int blocks = (int)(((long long)a.S * a.n_kv_heads * (a.dh / 8) + 255) / 256);
  const dim3 grid((unsigned)((long long)blocks * a.cache.N));
  if (a.dtype == FE_BF16)
    hipLaunchKernelGGL(k_packed_read<bf16>, grid, dim3(256), 0, s, a, c, blocks);
  else
    hipLaunchKernelGGL(k_packed_read<float>, grid, dim3(256), 0, s, a, c, blocks);
  return hipGetLastError();
}

hipError_t launch_packed_evict(const fe_packed_evict_args& a, hipStream_t s) {
  const PackedCache from = packed_cache(a.from, a.dh), to = packed_cache(a.to, a.dh);
  const unsigned heads = (unsigned)a.from.N * a.n_kv_heads;
  // one launch up to 1024 rows: 1024 heads of 512 of 1024 rows 27 us (by histograms 43), 256 heads 16.2 (15.1); 320 rows 15.3 (33.9)
  if (from.cap <= 1024) {
    if (from.cap <= 64)
      hipLaunchKernelGGL(k_packed_evict_short<1>, dim3(heads), dim3(256), 0, s, a, from, to);
    else if (from.cap <= 256)
      hipLaunchKernelGGL(k_packed_evict_short<4>, dim3(heads), dim3(256), 0, s, a, from, to);
    else
      hipLaunchKernelGGL(k_packed_evict_short<16>, dim3(heads), dim3(256), 0, s, a, from, to);
    return hipGetLastError();
  }
  if (from.cap <= 8192)
    hipLaunchKernelGGL(k_packed_select<8>, dim3(heads), dim3(1024), 0, s, a, from, to);
  else
    hipLaunchKernelGGL(k_packed_select<32>, dim3(heads), dim3(1024), 0, s, a, from, to);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int blocks = (int)(((long long)std::min(a.keep, from.cap) * (a.dh / 32) + 255) / 256);
  hipLaunchKernelGGL(k_packed_move, dim3((unsigned)((long long)heads * blocks)), dim3(256), 0, s, a, from, to, blocks);
  return hipGetLastError();
}

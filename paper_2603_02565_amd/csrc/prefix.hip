// Shared-prefix attention (fe_prefix_attention) and its gradient.
//
// The rows of a (request, key head) -- every list's rows, with the query heads that share the key head
// innermost -- are one matrix of R = K S G rows, so that the shared keys are read once for all of them.
// A workgroup owns a tile of consecutive rows and walks the keys in chunks: first the shared rows,
// then the own rows of the lists that the tile touches, packed without gaps (lists are short, so a
// chunk holds the keys of several).  In those packed coordinates the keys that a row may see are one interval
// [lo, hi), whatever the lengths and the causal mask, so a mask is two comparisons per score.
#include <algorithm>

#include "prefix.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Eight consecutive elements along the summed axis: one operand of the 16 x 16 x 32 bf16 product, or
// of eight 16 x 16 x 4 fp32 ones.  Lane l holds row (or column) l % 16 and elements 8 (l / 16) + j; product j
// of the fp32 form sums over {8 g + j}, so both types use one layout.
typedef float f32x8 __attribute__((ext_vector_type(8)));
template <typename T> struct Vec8;
template <> struct Vec8<bf16> { typedef bf16x8 type; };
template <> struct Vec8<float> { typedef f32x8 type; };
template <typename T> using V8 = typename Vec8<T>::type;

FE_DEV f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
FE_DEV f32x4 mma(f32x8 a, f32x8 b, f32x4 c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
  return c;
}

template <typename T> FE_DEV V8<T> ld8(const T* p) { return *reinterpret_cast<const V8<T>*>(p); }
template <typename T> FE_DEV void st8(T* p, V8<T> v) { *reinterpret_cast<V8<T>*>(p) = v; }
// LDS row padding: 16 bytes
template <typename T> constexpr int kPad = 16 / sizeof(T);

FE_DEV bool finite8(bf16x8 v) {
  const u32x4 w = __builtin_bit_cast(u32x4, v);
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    bad |= (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
  return !bad;
}
FE_DEV bool finite8(f32x8 v) {
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) bad |= (__float_as_uint(v[i]) & 0x7f800000u) == 0x7f800000u;
  return !bad;
}

FE_DEV int clampi(int v, int lo, int hi) { return min(max(v, lo), hi); }
FE_DEV int wave_min(int v) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v = min(v, __shfl_xor(v, m));
  return __builtin_amdgcn_readfirstlane(v);
}
FE_DEV int wave_max(int v) { return -wave_min(-v); }

FE_DEV int q_rows(const PrefixArgs& a, int bk) { return a.q_len ? clampi(a.q_len[bk], 0, a.S) : a.S; }
FE_DEV int own_rows(const PrefixArgs& a, int bk) { return a.own_len ? clampi(a.own_len[bk], 0, a.L) : a.L; }
FE_DEV int ctx_rows(const PrefixArgs& a, int b) { return a.ctx_len ? clampi(a.ctx_len[b], 0, a.T) : a.T; }

// The packed own rows of lists k0 .. k0 + nb - 1 of request b: off[i] = first packed row of list k0 + i, off[nb] =
// their number; a list without query rows contributes none.  NT threads, nb <= NT; ends with a barrier.
template <int NT>
FE_DEV void pack_own(const PrefixArgs& a, int b, int k0, int nb, int* off) {
  __shared__ int s_tot[NT / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int v = 0;
  if (tid < nb) {
    const int bk = b * a.K + k0 + tid;
    v = q_rows(a, bk) > 0 ? own_rows(a, bk) : 0;
  }
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int u = __shfl_up(v, m);
    if (lane >= m) v += u;
  }
  if (lane == 63) s_tot[wave] = v;
  __syncthreads();
  for (int w = 0; w < wave; ++w) v += s_tot[w];
  if (tid < nb) off[tid + 1] = v;
  if (tid == 0) off[0] = 0;
  __syncthreads();
}

// List (relative to k0) that packed row c < off[nb] belongs to: the last i with off[i] <= c.
FE_DEV int packed_list(const int* off, int nb, int c) {
  int lo = 0, hi = nb;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (off[mid] <= c) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Row of own_k / own_v that holds logical own row j of list bk, or -1 (a page outside the pool).
FE_DEV long long own_row(const PrefixArgs& a, int bk, int j) {
  if (a.page_rows == 0) return (long long)bk * a.L + j;
  const int page = a.table[(long long)bk * (a.L / a.page_rows) + j / a.page_rows];
  return page >= 0 && page < a.n_pages ? (long long)page * a.page_rows + j % a.page_rows : -1;
}

// What a lane has to know about its query row r of (request b, key head g).
struct Row {
  int k, s, h;                          // list, row, query head
  bool live;                            // r < R and s < q_len
  long long at;                         // (b K + k) S + s
  int own;                              // own keys it sees: j < own
};
FE_DEV Row row_of(const PrefixArgs& a, int b, int g, int r) {
  Row w;
  const int rr = min(r, a.R - 1), sg = a.S * a.G;
  w.k = rr / sg;
  const int rem = rr - w.k * sg;
  w.s = rem / a.G;
  w.h = g * a.G + rem - w.s * a.G;
  const int bk = b * a.K + w.k, n = q_rows(a, bk), m = own_rows(a, bk);
  w.live = r < a.R && w.s < n;
  w.at = (long long)bk * a.S + w.s;
  w.own = !w.live ? 0 : a.causal ? clampi(m - n + w.s + 1, 0, m) : m;
  return w;
}

// ------------------------------------------------------------------------------------------
// Forward.  NW waves of QT 16-row tiles; chunks of KC keys staged through registers (the next chunk's loads in
// flight behind this one's products) into LDS, K by rows and V transposed.  Scores are formed transposed
// (keys x rows): a lane then holds keys 8 g + j of one row, which is the operand layout of the product with
// the values, so probabilities never leave the registers.
// ------------------------------------------------------------------------------------------
template <typename T, int DH, int QT, int NW, int KC>
__global__ __launch_bounds__(NW * 64) void k_prefix_fwd(PrefixArgs a) {
  constexpr int NT = NW * 64, ROWS = NW * QT * 16, NB = DH / 16, ND = DH / 32;
  constexpr int KLD = DH + kPad<T>, VLD = KC + kPad<T>;
  constexpr int PER_T = KC * DH / 8 / NT;
  static_assert(ROWS <= NT && KC * DH / 8 % NT == 0 && KC % 32 == 0, "tile shape");
  __shared__ __attribute__((aligned(16))) T Ks[KC * KLD];
  __shared__ __attribute__((aligned(16))) T Vt[DH * VLD];
  __shared__ int s_off[ROWS + 1];
  __shared__ int s_odd;                            // last chunk whose values are not all finite
  __shared__ int s_holes, s_hole[KC];              // last chunk with keys of pages outside the pool, and those keys

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g4 = lane >> 4, c16 = lane & 15;
  int id = xcd_tile(blockIdx.x, gridDim.x);        // a (request, key head)'s workgroups share an XCD's L2
  const int z = id % a.splits;
  id /= a.splits;
  const int t = id % a.tiles;
  id /= a.tiles;
  const int g = id % a.Hkv, b = id / a.Hkv;
  const int r0 = t * ROWS, r1 = min(r0 + ROWS, a.R), sg = a.S * a.G;
  const int k0 = r0 / sg, nb = (r1 - 1) / sg - k0 + 1;
  if (tid == 0) s_odd = s_holes = -1;
  if (tid < KC) s_hole[tid] = -1;
  pack_own<NT>(a, b, k0, nb, s_off);

  const int nctx = ctx_rows(a, b), nown = s_off[nb];
  const int cctx = (nctx + KC - 1) / KC, chunks = cctx + (nown + KC - 1) / KC;
  const int cb = (int)((long long)chunks * z / a.splits), ce = (int)((long long)chunks * (z + 1) / a.splits);

  Row row[QT];
  V8<T> qf[QT][ND];
  int lo[QT], hi[QT];                              // the packed own rows that the row sees
  int wlo[QT], whi[QT], alo[QT], ahi[QT];          // their union and intersection over the wave's tile
  float m_run[QT], l_run[QT];                      // l_run: this lane's keys only, until the end
  f32x4 o[QT][NB];
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    row[i] = row_of(a, b, g, r0 + (wave * QT + i) * 16 + c16);
    lo[i] = s_off[row[i].k - k0];
    hi[i] = lo[i] + row[i].own;
    wlo[i] = wave_min(row[i].own ? lo[i] : 0x7fffffff);
    whi[i] = wave_max(hi[i] * (row[i].own != 0));
    alo[i] = wave_max(lo[i]);
    ahi[i] = wave_min(hi[i]);
    const T* Q = static_cast<const T*>(a.q) + row[i].at * a.q_ld + row[i].h * DH;
#pragma unroll
    for (int c = 0; c < ND; ++c) qf[i][c] = row[i].live ? ld8(Q + c * 32 + g4 * 8) : V8<T>{};
    m_run[i] = -INFINITY;
    l_run[i] = 0.f;
#pragma unroll
    for (int n = 0; n < NB; ++n) o[i][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float sl2 = a.scale * kLog2e;

  V8<T> kreg[PER_T], vreg[PER_T];
  int hole = 0;                                    // bit p: kreg[p] belongs to a page outside the pool
  auto load_chunk = [&](int c) {
    hole = 0;
#pragma unroll
    for (int p = 0; p < PER_T; ++p) {
      const int e = p * NT + tid, key = e / (DH / 8), d0 = (e % (DH / 8)) * 8;
      const T *kp = nullptr, *vp = nullptr;
      if (c < cctx) {
        const int x = c * KC + key;
        if (x < nctx) {
          const long long at = ((long long)b * a.T + x) * a.ctx_ld + g * DH + d0;
          kp = static_cast<const T*>(a.ctx_k) + at;
          vp = static_cast<const T*>(a.ctx_v) + at;
        }
      } else {
        const int x = (c - cctx) * KC + key;
        if (x < nown) {
          const int i = packed_list(s_off, nb, x);
          const long long at = own_row(a, b * a.K + k0 + i, x - s_off[i]);
          if (at >= 0) {
            kp = static_cast<const T*>(a.own_k) + at * a.own_ld + g * DH + d0;
            vp = static_cast<const T*>(a.own_v) + at * a.own_ld + g * DH + d0;
          } else {
            hole |= 1 << p;
          }
        }
      }
      kreg[p] = kp ? ld8(kp) : V8<T>{};
      vreg[p] = vp ? ld8(vp) : V8<T>{};
    }
  };
  if (cb < ce) load_chunk(cb);

  for (int c = cb; c < ce; ++c) {
    __syncthreads();                               // the previous chunk is no longer read
#pragma unroll
    for (int p = 0; p < PER_T; ++p) {
      const int e = p * NT + tid, key = e / (DH / 8), d0 = (e % (DH / 8)) * 8;
      st8(&Ks[key * KLD + d0], kreg[p]);
#pragma unroll
      for (int i = 0; i < 8; ++i) Vt[(d0 + i) * VLD + key] = vreg[p][i];
      if (c >= cctx && !finite8(vreg[p])) s_odd = c;
      if (hole >> p & 1) s_hole[key] = s_holes = c;
    }
    __syncthreads();
    if (c + 1 < ce) load_chunk(c + 1);
    const bool shared = c < cctx;
    const int base = shared ? c * KC : (c - cctx) * KC, top = shared ? nctx : nown;
    const bool odd = !shared && s_odd == c;

#pragma unroll
    for (int kb = 0; kb < KC; kb += 32) {
      const int x0 = base + kb;
      if (x0 >= top) break;                        // uniform
      V8<T> kf[2][ND], vf[NB];
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int d = 0; d < ND; ++d)
          kf[x][d] = ld8(&Ks[(kb + (c16 >> 2) * 8 + (c16 & 3) + 4 * x) * KLD + d * 32 + g4 * 8]);
#pragma unroll
      for (int n = 0; n < NB; ++n) vf[n] = ld8(&Vt[(n * 16 + c16) * VLD + kb + g4 * 8]);
#pragma unroll
      for (int i = 0; i < QT; ++i) {
        if (!shared && (x0 >= whi[i] || x0 + 32 <= wlo[i])) continue;   // uniform: no row of the tile sees a key of the step
        float s[8];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int d = 0; d < ND; ++d) acc = mma(kf[x][d], qf[i][d], acc);
#pragma unroll
          for (int j = 0; j < 4; ++j) s[4 * x + j] = acc[j] * sl2;
        }
        if (shared ? x0 + 32 > nctx : (x0 < alo[i] || x0 + 32 > ahi[i])) {   // uniform
          const int l = shared ? 0 : lo[i], h = shared ? nctx : hi[i];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int x = x0 + g4 * 8 + j;
            if (x < l || x >= h) s[j] = -INFINITY;
          }
        }
        if (s_holes == c) {                        // uniform
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (s_hole[kb + g4 * 8 + j] == c) s[j] = -INFINITY;
        }
        float mx = s[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) mx = fmaxf(mx, s[j]);
        const float m_new = fmaxf(m_run[i], rows_max(mx));
        const float ref = m_new == -INFINITY ? 0.f : m_new;       // a row without keys so far: every factor below is 0
        const float alpha = __builtin_amdgcn_exp2f(m_run[i] - ref);
        m_run[i] = m_new;
        float psum = 0.f;
        V8<T> pb;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float e = __builtin_amdgcn_exp2f(s[j] - ref);
          psum += e;
          pb[j] = from_f32<T>(e);
        }
        l_run[i] = fmaf(l_run[i], alpha, psum);
#pragma unroll
        for (int n = 0; n < NB; ++n) o[i][n] *= alpha;
        if (!odd) {
#pragma unroll
          for (int n = 0; n < NB; ++n) o[i][n] = mma(vf[n], pb, o[i][n]);
        } else {
          // A value of the chunk is not finite: in a product it would reach the rows that do not see its key, as 0
          // times infinity.  The same sums key by key, over the keys that the row sees.
#pragma unroll 1
          for (int gg = 0; gg < 4; ++gg)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float e = __shfl(to_f32((T)pb[j]), gg * 16 + c16);
              const int x = x0 + gg * 8 + j;
              if (x < lo[i] || x >= hi[i]) continue;
#pragma unroll
              for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                  o[i][n][q] = fmaf(e, to_f32(Vt[(n * 16 + g4 * 4 + q) * VLD + kb + gg * 8 + j]), o[i][n][q]);
            }
        }
      }
    }
  }

#pragma unroll
  for (int i = 0; i < QT; ++i) {
    const float l = rows_sum(l_run[i]);
    if (r0 + (wave * QT + i) * 16 + c16 >= a.R) continue;
    const long long ro = row[i].at * a.Hq + row[i].h;
    if (a.splits > 1) {
      const long long rows = (long long)a.B * a.K * a.S * a.Hq;
      float* po = a.part_o + (z * rows + ro) * DH;
#pragma unroll
      for (int n = 0; n < NB; ++n) *reinterpret_cast<f32x4*>(po + n * 16 + g4 * 4) = o[i][n];
      if (g4 == 0) {
        a.part_ml[(z * rows + ro) * 2] = m_run[i];
        a.part_ml[(z * rows + ro) * 2 + 1] = l;
      }
      continue;
    }
    const bool none = !row[i].live || m_run[i] == -INFINITY;
    const float inv = none ? 0.f : 1.f / l;
    T* O = static_cast<T*>(a.out) + row[i].at * a.out_ld + row[i].h * DH;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int q = 0; q < 4; ++q) O[n * 16 + g4 * 4 + q] = from_f32<T>(none ? 0.f : o[i][n][q] * inv);
    if (a.lse && g4 == 0) a.lse[ro] = none ? -INFINITY : (m_run[i] + log2f(l)) * kLn2;
  }
}

// Joins the key ranges of a row: DH / 4 threads a row, ranges in ascending order.
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_prefix_join(PrefixArgs a) {
  const long long rows = (long long)a.B * a.K * a.S * a.Hq;
  const long long e = (long long)blockIdx.x * 256 + threadIdx.x, ro = e / (DH / 4);
  const int d0 = (int)(e % (DH / 4)) * 4;
  if (ro >= rows) return;
  float m = -INFINITY;
  for (int z = 0; z < a.splits; ++z) m = fmaxf(m, a.part_ml[(z * rows + ro) * 2]);
  const long long at = ro / a.Hq;
  const int h = (int)(ro % a.Hq), bk = (int)(at / a.S), s = (int)(at % a.S);
  const bool none = m == -INFINITY || s >= q_rows(a, bk);
  const float ref = m == -INFINITY ? 0.f : m;
  float l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int z = 0; z < a.splits; ++z) {
    const float w = __builtin_amdgcn_exp2f(a.part_ml[(z * rows + ro) * 2] - ref);
    l = fmaf(a.part_ml[(z * rows + ro) * 2 + 1], w, l);
    o += w * *reinterpret_cast<const f32x4*>(a.part_o + (z * rows + ro) * DH + d0);
  }
  const float inv = none ? 0.f : 1.f / l;
  T* O = static_cast<T*>(a.out) + at * a.out_ld + h * DH + d0;
#pragma unroll
  for (int q = 0; q < 4; ++q) O[q] = from_f32<T>(none ? 0.f : o[q] * inv);
  if (a.lse && d0 == 0) a.lse[ro] = none ? -INFINITY : (m + log2f(l)) * kLn2;
}

// ------------------------------------------------------------------------------------------
// Gradient.
// ------------------------------------------------------------------------------------------

// delta = dout . out per row and head: 16 lanes a row.
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_prefix_delta(PrefixGradArgs p) {
  const PrefixArgs& a = p.f;
  const long long rows = (long long)a.B * a.K * a.S * a.Hq;
  const long long ro = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
  const int x = threadIdx.x & 15;
  if (ro >= rows) return;
  const long long at = ro / a.Hq;
  const int h = (int)(ro % a.Hq), bk = (int)(at / a.S), s = (int)(at % a.S);
  float v = 0.f;
  if (s < q_rows(a, bk)) {
    const T* O = static_cast<const T*>(a.out) + at * a.out_ld + h * DH;
    const T* D = static_cast<const T*>(p.dout) + at * p.dout_ld + h * DH;
#pragma unroll
    for (int d = 0; d < DH; d += 16) v = fmaf(to_f32(D[d + x]), to_f32(O[d + x]), v);
  }
  v += dpp<0x128>(v);
  v += dpp<0x124>(v);
  v += dpp<0x4e>(v);
  v += dpp<0xb1>(v);
  if (x == 0) p.delta[ro] = v;
}

// dq: rows and chunks as in the forward, probabilities again from lse.
template <typename T, int DH, int NW, int KC>
__global__ __launch_bounds__(NW * 64) void k_prefix_dq(PrefixGradArgs p) {
  const PrefixArgs& a = p.f;
  constexpr int NT = NW * 64, ROWS = NW * 16, NB = DH / 16, ND = DH / 32;
  constexpr int KLD = DH + kPad<T>, VLD = KC + kPad<T>;
  constexpr int PER_T = KC * DH / 8 / NT;
  static_assert(KC * DH / 8 % NT == 0 && KC % 32 == 0, "tile shape");
  __shared__ __attribute__((aligned(16))) T Ks[KC * KLD];
  __shared__ __attribute__((aligned(16))) T Vs[KC * KLD];
  __shared__ __attribute__((aligned(16))) T Kt[DH * VLD];
  __shared__ int s_off[ROWS + 1];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g4 = lane >> 4, c16 = lane & 15;
  int id = xcd_tile(blockIdx.x, gridDim.x);
  const int t = id % a.tiles;
  id /= a.tiles;
  const int g = id % a.Hkv, b = id / a.Hkv;
  const int r0 = t * ROWS, r1 = min(r0 + ROWS, a.R), sg = a.S * a.G;
  const int k0 = r0 / sg, nb = (r1 - 1) / sg - k0 + 1;
  pack_own<NT>(a, b, k0, nb, s_off);
  const int nctx = ctx_rows(a, b), nown = s_off[nb];
  const int cctx = (nctx + KC - 1) / KC, chunks = cctx + (nown + KC - 1) / KC;

  const int r = r0 + wave * 16 + c16;
  const Row row = row_of(a, b, g, r);
  const int lo = s_off[row.k - k0], hi = lo + row.own;
  const int wlo = wave_min(row.own ? lo : 0x7fffffff), whi = wave_max(hi * (row.own != 0));
  const long long ro = row.at * a.Hq + row.h;
  const float lse = row.live ? a.lse[ro] : -INFINITY;
  const float lse2 = lse == -INFINITY ? INFINITY : lse * kLog2e;   // no keys: every probability 0
  const float delta = row.live ? p.delta[ro] : 0.f;
  V8<T> qf[ND], df[ND];
  {
    const T* Q = static_cast<const T*>(a.q) + row.at * a.q_ld + row.h * DH;
    const T* D = static_cast<const T*>(p.dout) + row.at * p.dout_ld + row.h * DH;
#pragma unroll
    for (int c = 0; c < ND; ++c) {
      qf[c] = row.live ? ld8(Q + c * 32 + g4 * 8) : V8<T>{};
      df[c] = row.live ? ld8(D + c * 32 + g4 * 8) : V8<T>{};
    }
  }
  f32x4 o[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) o[n] = f32x4{0.f, 0.f, 0.f, 0.f};
  const float sl2 = a.scale * kLog2e;

  V8<T> kreg[PER_T], vreg[PER_T];
  auto load_chunk = [&](int c) {
#pragma unroll
    for (int q = 0; q < PER_T; ++q) {
      const int e = q * NT + tid, key = e / (DH / 8), d0 = (e % (DH / 8)) * 8;
      const T *kp = nullptr, *vp = nullptr;
      if (c < cctx) {
        const int x = c * KC + key;
        if (x < nctx) {
          const long long at = ((long long)b * a.T + x) * a.ctx_ld + g * DH + d0;
          kp = static_cast<const T*>(a.ctx_k) + at;
          vp = static_cast<const T*>(a.ctx_v) + at;
        }
      } else {
        const int x = (c - cctx) * KC + key;
        if (x < nown) {
          const int i = packed_list(s_off, nb, x);
          const long long at = own_row(a, b * a.K + k0 + i, x - s_off[i]) * a.own_ld + g * DH + d0;
          kp = static_cast<const T*>(a.own_k) + at;
          vp = static_cast<const T*>(a.own_v) + at;
        }
      }
      kreg[q] = kp ? ld8(kp) : V8<T>{};
      vreg[q] = vp ? ld8(vp) : V8<T>{};
    }
  };
  if (chunks) load_chunk(0);
  for (int c = 0; c < chunks; ++c) {
    __syncthreads();
#pragma unroll
    for (int q = 0; q < PER_T; ++q) {
      const int e = q * NT + tid, key = e / (DH / 8), d0 = (e % (DH / 8)) * 8;
      st8(&Ks[key * KLD + d0], kreg[q]);
      st8(&Vs[key * KLD + d0], vreg[q]);
#pragma unroll
      for (int i = 0; i < 8; ++i) Kt[(d0 + i) * VLD + key] = kreg[q][i];
    }
    __syncthreads();
    if (c + 1 < chunks) load_chunk(c + 1);
    const bool shared = c < cctx;
    const int base = shared ? c * KC : (c - cctx) * KC, top = shared ? nctx : nown;
    const int l = shared ? 0 : lo, h = shared ? nctx : hi;
#pragma unroll
    for (int kb = 0; kb < KC; kb += 32) {
      const int x0 = base + kb;
      if (x0 >= top) break;                                            // uniform
      if (!shared && (x0 >= whi || x0 + 32 <= wlo)) continue;          // uniform
      V8<T> ds;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        f32x4 s = {0.f, 0.f, 0.f, 0.f}, dp = {0.f, 0.f, 0.f, 0.f};
        const int at = (kb + (c16 >> 2) * 8 + (c16 & 3) + 4 * x) * KLD + g4 * 8;
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          s = mma(ld8(&Ks[at + d * 32]), qf[d], s);
          dp = mma(ld8(&Vs[at + d * 32]), df[d], dp);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int y = x0 + g4 * 8 + 4 * x + j;
          const float e = __builtin_amdgcn_exp2f(fmaf(s[j], sl2, -lse2)) * (dp[j] - delta);
          ds[4 * x + j] = from_f32<T>(y >= l && y < h ? e : 0.f);
        }
      }
#pragma unroll
      for (int n = 0; n < NB; ++n) o[n] = mma(ld8(&Kt[(n * 16 + c16) * VLD + kb + g4 * 8]), ds, o[n]);
    }
  }
  if (r >= a.R) return;
  T* O = static_cast<T*>(p.dq) + row.at * p.dq_ld + row.h * DH;
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int q = 0; q < 4; ++q) O[n * 16 + g4 * 4 + q] = from_f32<T>(row.live ? o[n][q] * a.scale : 0.f);
}

// dk and dv of a tile of keys: the keys stay in registers, the rows stream through LDS in chunks of RC, by rows and
// transposed.  Tiles 0 .. ctx_tiles - 1 of a (request, key head) hold shared rows and meet every row; the others hold
// own rows (dense, list after list) and meet the rows of their lists.  In the tile's numbering -- shared row, or
// k L + j -- the keys that a row sees are again one interval.
template <typename T, int DH, int NW, int RC>
__global__ __launch_bounds__(NW * 64) void k_prefix_dkv(PrefixGradArgs p) {
  const PrefixArgs& a = p.f;
  constexpr int NT = NW * 64, COLS = NW * 16, NB = DH / 16, ND = DH / 32;
  constexpr int KLD = DH + kPad<T>, VLD = RC + kPad<T>;
  constexpr int PER_T = (RC * DH / 8 + NT - 1) / NT;
  static_assert(RC % 32 == 0 && RC <= NT, "tile shape");
  __shared__ __attribute__((aligned(16))) T Qs[RC * KLD], Ds[RC * KLD];
  __shared__ __attribute__((aligned(16))) T Qt[DH * VLD], Dt[DH * VLD];
  __shared__ float s_lse[RC], s_delta[RC];
  __shared__ int s_lo[RC], s_hi[RC];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g4 = lane >> 4, c16 = lane & 15;
  int id = xcd_tile(blockIdx.x, gridDim.x);
  const int t = id % (p.ctx_tiles + p.own_tiles);
  id /= p.ctx_tiles + p.own_tiles;
  const int g = id % a.Hkv, b = id / a.Hkv;
  const bool shared = t < p.ctx_tiles;
  const int x0 = (shared ? t : t - p.ctx_tiles) * COLS, cols = shared ? a.T : a.K * a.L, sg = a.S * a.G;
  const int nctx = ctx_rows(a, b);
  int rb = 0, re = a.R;
  if (shared) {
    if (x0 >= nctx) re = 0;
  } else {
    rb = x0 / a.L * sg;
    re = ((min(x0 + COLS, cols) - 1) / a.L + 1) * sg;
  }

  const int x = x0 + wave * 16 + c16;                                   // this lane's key
  bool live = false;
  long long at = 0;                                                     // its row of the tensors
  if (x < cols) {
    if (shared) {
      live = x < nctx;
      at = (long long)b * a.T + x;
    } else {
      const int bk = b * a.K + x / a.L;
      live = x % a.L < own_rows(a, bk) && q_rows(a, bk) > 0;
      at = (long long)b * cols + x;
    }
  }
  V8<T> kf[ND], vf[ND];
  {
    const long long off = at * (shared ? a.ctx_ld : a.own_ld) + g * DH + g4 * 8;
    const T *kp = static_cast<const T*>(shared ? a.ctx_k : a.own_k) + off, *vp = static_cast<const T*>(shared ? a.ctx_v : a.own_v) + off;
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      kf[d] = live ? ld8(kp + d * 32) : V8<T>{};
      vf[d] = live ? ld8(vp + d * 32) : V8<T>{};
    }
  }
  f32x4 dk[NB], dv[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) dk[n] = dv[n] = f32x4{0.f, 0.f, 0.f, 0.f};
  const float sl2 = a.scale * kLog2e;

  for (int rc = rb; rc < re; rc += RC) {
    __syncthreads();
#pragma unroll
    for (int q = 0; q < PER_T; ++q) {
      const int e = q * NT + tid, i = e / (DH / 8), d0 = (e % (DH / 8)) * 8;
      if (RC * DH / 8 % NT != 0 && i >= RC) continue;
      const Row w = row_of(a, b, g, rc + i);
      const bool in = w.live && rc + i < re;
      const V8<T> qv = in ? ld8(static_cast<const T*>(a.q) + w.at * a.q_ld + w.h * DH + d0) : V8<T>{};
      const V8<T> dv8 = in ? ld8(static_cast<const T*>(p.dout) + w.at * p.dout_ld + w.h * DH + d0) : V8<T>{};
      st8(&Qs[i * KLD + d0], qv);
      st8(&Ds[i * KLD + d0], dv8);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        Qt[(d0 + j) * VLD + i] = qv[j];
        Dt[(d0 + j) * VLD + i] = dv8[j];
      }
    }
    if (tid < RC) {
      const Row w = row_of(a, b, g, rc + tid);
      const bool in = w.live && rc + tid < re;
      const float l = in ? a.lse[w.at * a.Hq + w.h] : -INFINITY;
      s_lse[tid] = l == -INFINITY ? INFINITY : l * kLog2e;
      s_delta[tid] = in ? p.delta[w.at * a.Hq + w.h] : 0.f;
      s_lo[tid] = shared ? 0 : w.k * a.L;
      s_hi[tid] = !in ? 0 : shared ? nctx : w.k * a.L + w.own;
    }
    __syncthreads();
#pragma unroll
    for (int kb = 0; kb < RC; kb += 32) {
      V8<T> pb, ds;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f32x4 s = {0.f, 0.f, 0.f, 0.f}, dp = {0.f, 0.f, 0.f, 0.f};
        const int ar = (kb + (c16 >> 2) * 8 + (c16 & 3) + 4 * u) * KLD + g4 * 8;
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          s = mma(ld8(&Qs[ar + d * 32]), kf[d], s);
          dp = mma(ld8(&Ds[ar + d * 32]), vf[d], dp);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int i = kb + g4 * 8 + 4 * u + j;
          const bool sees = x >= s_lo[i] && x < s_hi[i];
          const float e = __builtin_amdgcn_exp2f(fmaf(s[j], sl2, -s_lse[i]));
          pb[4 * u + j] = from_f32<T>(sees ? e : 0.f);
          ds[4 * u + j] = from_f32<T>(sees ? e * (dp[j] - s_delta[i]) : 0.f);
        }
      }
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        dv[n] = mma(ld8(&Dt[(n * 16 + c16) * VLD + kb + g4 * 8]), pb, dv[n]);
        dk[n] = mma(ld8(&Qt[(n * 16 + c16) * VLD + kb + g4 * 8]), ds, dk[n]);
      }
    }
  }
  if (x >= cols) return;
  const long long off = at * (shared ? p.dctx_ld : p.down_ld) + g * DH;
  T *ko = static_cast<T*>(shared ? p.dctx_k : p.down_k) + off, *vo = static_cast<T*>(shared ? p.dctx_v : p.down_v) + off;
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      ko[n * 16 + g4 * 4 + q] = from_f32<T>(live ? dk[n][q] * a.scale : 0.f);
      vo[n * 16 + g4 * 4 + q] = from_f32<T>(live ? dv[n][q] : 0.f);
    }
}

template <typename T, int DH>
hipError_t fwd(const PrefixArgs& a, const PrefixPlan& p, hipStream_t s) {
  const dim3 grid((unsigned)((long long)a.B * a.Hkv * a.tiles * a.splits));
  hipLaunchKernelGGL((k_prefix_fwd<T, DH, 1, 4, 64>), grid, dim3(256), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  const long long rows = (long long)a.B * a.K * a.S * a.Hq;
  hipLaunchKernelGGL((k_prefix_join<T, DH>), dim3((unsigned)((rows * (DH / 4) + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T, int DH>
hipError_t grad(PrefixGradArgs p, hipStream_t s) {
  PrefixArgs& a = p.f;
  const long long rows = (long long)a.B * a.K * a.S * a.Hq, bg = (long long)a.B * a.Hkv;
  hipLaunchKernelGGL((k_prefix_delta<T, DH>), dim3((unsigned)((rows + 15) / 16)), dim3(256), 0, s, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  a.tiles = (a.R + 63) / 64;
  hipLaunchKernelGGL((k_prefix_dq<T, DH, 4, 64>), dim3((unsigned)(bg * a.tiles)), dim3(256), 0, s, p);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  p.ctx_tiles = (a.T + 63) / 64;
  p.own_tiles = (int)(((long long)a.K * a.L + 63) / 64);
  if (p.ctx_tiles + p.own_tiles == 0) return hipSuccess;
  hipLaunchKernelGGL((k_prefix_dkv<T, DH, 4, 32>), dim3((unsigned)(bg * (p.ctx_tiles + p.own_tiles))), dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace

PrefixPlan prefix_plan(const fe_prefix_args& a) {
  PrefixPlan p;
  p.rows = 64;
  const long long G = a.n_heads / a.n_kv_heads, R = (long long)a.K * a.S * G;
  p.tiles = (int)((R + p.rows - 1) / p.rows);
  // split the keys while the launch has fewer than four workgroups per compute unit and a range keeps two chunks
  const long long wgs = (long long)a.B * a.n_kv_heads * p.tiles;
  const long long lists = std::min<long long>(a.K, (p.rows - 1) / (a.S * G) + 2);
  const long long chunks = (a.T + 63) / 64 + (lists * a.L + 63) / 64;
  p.splits = (int)std::max(1LL, std::min({1024 / std::max(1LL, wgs), chunks / 2, 64LL}));
  const size_t rows = (size_t)a.B * a.K * a.S * a.n_heads;
  p.part_bytes = p.splits > 1 ? p.splits * rows * (a.dh + 2) * sizeof(float) : 0;
  return p;
}

hipError_t launch_prefix_fwd(PrefixArgs a, int dh, bool bf16_rows, const PrefixPlan& p, hipStream_t s) {
  a.tiles = p.tiles;
  a.splits = p.splits;
  if (bf16_rows) return dh == 32 ? fwd<bf16, 32>(a, p, s) : dh == 64 ? fwd<bf16, 64>(a, p, s) : fwd<bf16, 128>(a, p, s);
  return dh == 32 ? fwd<float, 32>(a, p, s) : dh == 64 ? fwd<float, 64>(a, p, s) : fwd<float, 128>(a, p, s);
}

hipError_t launch_prefix_grad(PrefixGradArgs a, int dh, bool bf16_rows, hipStream_t s) {
  if (bf16_rows) return dh == 32 ? grad<bf16, 32>(a, s) : dh == 64 ? grad<bf16, 64>(a, s) : grad<bf16, 128>(a, s);
  return dh == 32 ? grad<float, 32>(a, s) : dh == 64 ? grad<float, 64>(a, s) : grad<float, 128>(a, s);
}

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

// Eight elements along the summed axis: one operand of the 16 x 16 x 32 bf16 product.  Lane l holds row (or column) l % 16
// and the eight elements of its group l / 16; which element is which is free as long as both operands agree.
typedef float f32x8 __attribute__((ext_vector_type(8)));
template <typename T> struct Vec8;
template <> struct Vec8<bf16> { typedef bf16x8 type; };
template <> struct Vec8<float> { typedef f32x8 type; };
template <typename T> using V8 = typename Vec8<T>::type;

FE_DEV f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
// fp32 operands in three bf16 parts: truncation takes the first 8 bits of the significand, then the next 8, and leaves the
// last 8, so that x = p[0] + p[1] + p[2] exactly.  Of the nine products of parts the six largest are formed; the others are
// below 2^-21 of |x||y|, 2^-24.6 in the mean.  Six bf16 products take 3/8 of the time of the eight 16 x 16 x 4 fp32 ones (training
// step of 256 x 550 rows, heads of 32: 277 us with those, 222 in parts; 64 x 1024 rows, heads of 64: 698, 490).  An
// infinity is a first part alone; a NaN is one in its later parts, whatever the first 16 bits alone would be.
struct Parts { bf16x8 p[3]; };
FE_DEV f32x4 mma(Parts a, Parts b, f32x4 c) {
  c = mma(a.p[2], b.p[0], c);
  c = mma(a.p[0], b.p[2], c);
  c = mma(a.p[1], b.p[1], c);
  c = mma(a.p[1], b.p[0], c);
  c = mma(a.p[0], b.p[1], c);
  return mma(a.p[0], b.p[0], c);
}
template <bool FINITE> FE_DEV Parts parts8(const f32x8 v) {
  u32x4 w[3];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    unsigned h[2], m[2], l[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float x = v[2 * i + j];
      h[j] = __float_as_uint(x);
      float rest = x - __uint_as_float(h[j] & 0xffff0000u);
      if (!FINITE && __builtin_isinf(x)) rest = 0.f;
      m[j] = __float_as_uint(rest);
      l[j] = __float_as_uint(rest - __uint_as_float(m[j] & 0xffff0000u));
    }
    w[0][i] = __builtin_amdgcn_perm(h[1], h[0], 0x07060302);   // the upper halves of two
    w[1][i] = __builtin_amdgcn_perm(m[1], m[0], 0x07060302);
    w[2][i] = __builtin_amdgcn_perm(l[1], l[0], 0x07060302);
  }
  return Parts{{__builtin_bit_cast(bf16x8, w[0]), __builtin_bit_cast(bf16x8, w[1]), __builtin_bit_cast(bf16x8, w[2])}};
}

// The operand of a product, from eight elements or from eight floats (bf16: rounded to nearest even).
template <typename T> struct Form;
template <> struct Form<bf16> {
  typedef bf16x8 Op;
  static FE_DEV Op of(bf16x8 v) { return v; }
  static FE_DEV Op of(const float (&s)[8]) {
    return __builtin_convertvector((f32x8{s[0], s[1], s[2], s[3], s[4], s[5], s[6], s[7]}), bf16x8);
  }
  static FE_DEV float value(Op v, int j) { return to_f32((bf16)v[j]); }
};
template <> struct Form<float> {
  typedef Parts Op;
  static FE_DEV Op of(f32x8 v) { return parts8<false>(v); }
  static FE_DEV Op of(const float (&s)[8]) {
    return parts8<true>(f32x8{s[0], s[1], s[2], s[3], s[4], s[5], s[6], s[7]});
  }
  static FE_DEV float value(const Op& v, int j) { return (to_f32(v.p[2][j]) + to_f32(v.p[1][j])) + to_f32(v.p[0][j]); }
};

template <typename T> FE_DEV V8<T> ld8(const T* p) { return *reinterpret_cast<const V8<T>*>(p); }
// ... at a byte offset from a uniform base
template <typename T> FE_DEV V8<T> ld8_at(const T* base, unsigned at) {
  return *reinterpret_cast<const V8<T>*>(reinterpret_cast<const char*>(base) + at);
}
template <typename T> FE_DEV void st8(T* p, V8<T> v) { *reinterpret_cast<V8<T>*>(p) = v; }
FE_DEV void st4(float* p, f32x4 v) { *reinterpret_cast<f32x4*>(p) = v; }
FE_DEV void st4(bf16* p, f32x4 v) {
  bf16x4 w;
#pragma unroll
  for (int q = 0; q < 4; ++q) w[q] = (bf16)v[q];
  *reinterpret_cast<bf16x4*>(p) = w;
}

// The largest magnitudes among several vectors, as bit patterns (bf16: of the even and of the odd elements), and
// whether they are all finite.
FE_DEV unsigned peak(unsigned m, bf16x8 v) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  const u32x4 w = __builtin_bit_cast(u32x4, v);
  u16x2 top = __builtin_bit_cast(u16x2, m);
#pragma unroll
  for (int i = 0; i < 4; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu));
  return __builtin_bit_cast(unsigned, top);
}
FE_DEV unsigned peak(unsigned m, f32x8 v) {
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
  return m;
}
template <typename T> FE_DEV bool finite(unsigned m) {
  return sizeof(T) == 4 ? m < 0x7f800000u : max(m & 0xffffu, m >> 16) < 0x7f80u;
}

// v with zeros for its infinities and NaNs.
FE_DEV bf16x8 finite_of(bf16x8 v) {
  typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
  const u16x8 w = __builtin_bit_cast(u16x8, v);
  return __builtin_bit_cast(bf16x8, (u16x8)((w & 0x7f80) == 0x7f80 ? (u16x8)0 : w));
}
FE_DEV Parts finite_of(const Parts& v) { return Parts{{finite_of(v.p[0]), finite_of(v.p[1]), finite_of(v.p[2])}}; }

FE_DEV int clampi(int v, int lo, int hi) { return min(max(v, lo), hi); }

FE_DEV int q_rows(const PrefixArgs& a, int bk) { return a.q_len ? clampi(a.q_len[bk], 0, a.S) : a.S; }
FE_DEV int own_rows(const PrefixArgs& a, int bk) { return a.own_len ? clampi(a.own_len[bk], 0, a.L) : a.L; }
FE_DEV int ctx_rows(const PrefixArgs& a, int b) { return a.ctx_len ? clampi(a.ctx_len[b], 0, a.T) : a.T; }

// Key of a 32-key step that element j of a lane in group g4 stands for: 4 g4 and a part that is the same for all lanes
// (compared with a limit from which 4 g4 has been taken, it needs no register).
FE_DEV int key_of(int j) { return 16 * (j >> 2) + (j & 3); }
FE_DEV int key_of(int j, int g4) { return key_of(j) + 4 * g4; }

// log2(e) |scale|, the exponent's factor of a score; positive, so that masked scores stay -infinity when scale is 0.
FE_DEV float score_unit(float scale) { return fmaxf(fabsf(scale) * kLog2e, 1e-37f); }

// The key ranges of the forward are numbered request after request: request b has `n` of them, from `first` on.
struct Ranges { int first, n; };
// by_length (B <= 64): lane b finds those of request b.  Every request has one; the others are shared out in proportion
// to the chunks of keys, rounded down, so they may leave a few unused.
FE_DEV Ranges ranges_of_lane(const PrefixArgs& a) {
  const int lane = threadIdx.x & 63;
  const int mine = lane < a.B ? (ctx_rows(a, lane) + 63) / 64 + a.own_chunks + 1 : 0;
  int all = mine;                                  // at most 2^25
#pragma unroll
  for (int x = 1; x < 64; x *= 2) all += __shfl_xor(all, x);
  const int n = lane < a.B ? 1 + (int)((float)(a.B * (a.splits - 1)) * (float)mine / (float)all) : 0;
  int end = n;
#pragma unroll
  for (int x = 1; x < 64; x *= 2) {
    const int before = __shfl_up(end, x);
    if (lane >= x) end += before;
  }
  return {end - n, n};
}

// Four consecutive elements of an output row, and what their rounding left (bf16, when asked for).
template <typename T>
FE_DEV void store_out(const PrefixArgs& a, long long at, int col, f32x4 v);
template <>
FE_DEV void store_out<bf16>(const PrefixArgs& a, long long at, int col, f32x4 v) {
  bf16x4 w;
#pragma unroll
  for (int q = 0; q < 4; ++q) w[q] = (bf16)v[q];
  *reinterpret_cast<bf16x4*>(static_cast<bf16*>(a.out) + at * a.out_ld + col) = w;
  if (!a.out_rest) return;                         // uniform
  // the eight bits below the rounded value's, as a signed step of its bit pattern: the second byte of the difference
  int d[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) d[q] = min((int)__float_as_uint(v[q]) - (int)__float_as_uint((float)w[q]), 0x7fff);
  *reinterpret_cast<unsigned*>(a.out_rest + at * a.Hq * a.dh + col) =
      __builtin_amdgcn_perm(d[1], d[0], 0x0c0c0501) | __builtin_amdgcn_perm(d[3], d[2], 0x05010c0c);
}
// ... and back: out with its rest, 16 bits of the significand, the others cut.
FE_DEV float with_rest(bf16 v, int step) { return __uint_as_float(__float_as_uint((float)v) + step * 256); }
FE_DEV float with_rest(float v, int) { return v; }
template <>
FE_DEV void store_out<float>(const PrefixArgs& a, long long at, int col, f32x4 v) {
  *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at * a.out_ld + col) = v;
}

// The packed own rows of lists k0 .. k0 + nb - 1 of request b: off[i] = first packed row of list k0 + i, off[nb] =
// their number; a list without query rows contributes none.  NT threads, nb <= NT; ends with a barrier.
template <int NT>
FE_DEV void pack_own(const PrefixArgs& a, int b, int k0, int nb, int* off) {
  __shared__ int s_tot[NT / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (!a.q_len && !a.own_len) {                    // uniform: lists of one length
    if (tid <= nb) off[tid] = tid * a.L;
    if (tid == 0) off[nb] = nb * a.L;
    __syncthreads();
    return;
  }
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

// Where row c of the lists packed in off lies in own_k / own_v: find() says it, row() turns it into the row's number,
// -2 past the last row, -1 for a page outside the pool.  A page is requested by find() and looked at by row(), a chunk
// later, so that nothing waits for the table.
template <bool PAGED> struct OwnAt;
template <> struct OwnAt<false> {
  long long at = -2;
  FE_DEV void find(const PrefixArgs& a, int b, int k0, int nb, const int* off, int c) {
    at = -2;
    if (c >= off[nb]) return;
    const int i = packed_list(off, nb, c);
    at = ((long long)b * a.K + k0 + i) * a.L + c - off[i];
  }
  FE_DEV long long row(const PrefixArgs&) const { return at; }
};
template <> struct OwnAt<true> {
  int page = 0, rest = -1;
  FE_DEV void find(const PrefixArgs& a, int b, int k0, int nb, const int* off, int c) {
    rest = -1;
    if (c >= off[nb]) return;
    const int i = packed_list(off, nb, c), j = c - off[i], p = j / a.page_rows;
    page = a.table[((long long)b * a.K + k0 + i) * (a.L / a.page_rows) + p];
    rest = j - p * a.page_rows;
  }
  FE_DEV long long row(const PrefixArgs& a) const {
    return rest < 0 ? -2 : page >= 0 && page < a.n_pages ? (long long)page * a.page_rows + rest : -1;
  }
};

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

// A tile of rows of DH elements in LDS, read as an operand along its rows (summed over columns) and along its columns
// (summed over rows).  bf16: rows of DH without padding, their 16-byte units exchanged inside a row, so that 16 rows at
// one unit and 8 rows at one pair of units both fall on all 64 banks (measured: a row read 8.4 cycles, 7.9 at best; a
// transposed one 10.1, the same at every stride); fp32: three such tiles, one for each part.
//
// Both reads start from a number that depends on the lane alone (row_lane, col_lane); what differs from read to read is a
// constant xor and a row offset.
template <typename T, int DH, int ROWS> struct Tile;
template <int DH, int ROWS> struct Tile<bf16, DH, ROWS> {
  typedef bf16 Elem;
  static constexpr int SIZE = ROWS * DH, UNITS = DH / 8, PER = 128 / DH;   // PER rows span the banks
  static FE_DEV int swap(int row) {                // repeats every 16 rows
    const int h = row / PER % UNITS;
    return (h % (UNITS / 2)) << 1 | h / (UNITS / 2);
  }
  static FE_DEV int at(int row, int unit) { return row * DH + ((unit ^ swap(row)) << 3); }
  template <bool FINITE> static FE_DEV void put(bf16* X, int row, int unit, bf16x8 v) { st8(X + at(row, unit), v); }
  static FE_DEV float value(const bf16* X, int row, int col) { return to_f32(X[at(row, col >> 3) + (col & 7)]); }
  // Operand along rows: lane l is row base + l % 16, its elements are columns 32 d + 8 (l / 16) + j (base a multiple
  // of 16).
  static FE_DEV int row_lane(int lane) { return at(lane & 15, lane >> 4); }
  static FE_DEV bf16x8 rows(const bf16* X, int base, int d, int row_lane) {
    return ld8(X + base * DH + (row_lane ^ (d << 5)));
  }
  // Operand along columns: lane l is column 16 n + l % 16; its elements 4 x + j are rows base + 16 x + 4 (l / 16) + j, the
  // order in which a lane holds the results of two 16-row products.  Each group of 16 lanes reads a 4 x 16 block
  // transposed (ds_read_b64_tr_b16).
  static FE_DEV int col_lane(int lane) {
    return at(4 * (lane >> 4) + ((lane & 15) >> 2), (lane & 3) >> 1) + (lane & 1) * 4;
  }
  static FE_DEV bf16x8 cols(const bf16* X, int base, int n, int col_lane) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4* lds_ptr;
    bf16* p = const_cast<bf16*>(X) + base * DH + (col_lane ^ (n << 4));
    const s16x4 u = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p);
    const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + 16 * DH));
    return __builtin_shufflevector(__builtin_bit_cast(bf16x4, u), __builtin_bit_cast(bf16x4, v), 0, 1, 2, 3, 4, 5, 6, 7);
  }
};
template <int DH, int ROWS> struct Tile<float, DH, ROWS> {
  typedef Tile<bf16, DH, ROWS> Part;
  typedef bf16 Elem;
  static constexpr int SIZE = 3 * Part::SIZE;
  template <bool FINITE> static FE_DEV void put(bf16* X, int row, int unit, f32x8 v) {
    const Parts w = parts8<FINITE>(v);
#pragma unroll
    for (int i = 0; i < 3; ++i) Part::template put<true>(X + i * Part::SIZE, row, unit, w.p[i]);
  }
  static FE_DEV float value(const bf16* X, int row, int col) {
    return (Part::value(X + 2 * Part::SIZE, row, col) + Part::value(X + Part::SIZE, row, col)) + Part::value(X, row, col);
  }
  static FE_DEV int row_lane(int lane) { return Part::row_lane(lane); }
  static FE_DEV int col_lane(int lane) { return Part::col_lane(lane); }
  static FE_DEV Parts rows(const bf16* X, int base, int d, int row_lane) {
    return Parts{{Part::rows(X, base, d, row_lane), Part::rows(X + Part::SIZE, base, d, row_lane),
                  Part::rows(X + 2 * Part::SIZE, base, d, row_lane)}};
  }
  static FE_DEV Parts cols(const bf16* X, int base, int n, int col_lane) {
    return Parts{{Part::cols(X, base, n, col_lane), Part::cols(X + Part::SIZE, base, n, col_lane),
                  Part::cols(X + 2 * Part::SIZE, base, n, col_lane)}};
  }
};
// Keeps a lane's number in one register, instead of a register for every xor of it that a loop uses.
FE_DEV int fresh(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Waves per SIMD that the register file is shared between (more hide more latency; fewer would spill).
constexpr int waves_of(int bytes, int dh, int qt) {
  return dh == 128 ? 2 : dh * qt <= (bytes == 2 ? 64 : 32) ? 4 : dh * qt <= 64 || bytes == 2 ? 3 : 2;
}
constexpr int dkv_waves(int dh) { return dh == 32 ? 3 : 2; }

// ------------------------------------------------------------------------------------------
// Forward.  NW waves of QT 16-row tiles; chunks of KC keys staged through registers (the next chunk's loads in
// flight behind this one's products) into LDS.  Scores are formed transposed (keys x rows): a lane then holds
// eight keys of one row, which is the operand layout of the product with the values, so probabilities never leave the
// registers.
// Bound: with many rows a key the vector unit: a product-sum, an exponential, a sum, half a maximum and half a rounding a
// score beside its 4 dh matrix operations, and the staging, the masks and the prologue (64 x 1024 rows of 1088 keys, heads
// of 64: 33.5 us, 529 TFLOP/s, 8.8 vector instructions a score; vector unit 57% of the time, LDS 49%, matrix cores 24%, one
// after another within a step; 256 x 550 rows of 267 keys, heads of 32: 24.2 us, 199 TFLOP/s, 13.8 a score, vector unit 66%);
// with few rows HBM (4 x 32 lists of 4 rows a key head, heads of 128, 539 MB: 129 us, 4.2 TB/s); fp32 the vector unit, which
// also splits the operands (72% of the time; 256 x 550 rows, heads of 32: 62 us, 77 TFLOP/s); a short context its few
// dependent trips to memory (20 rows of 181 + 12 keys: 7.1 us).
// ------------------------------------------------------------------------------------------
template <typename T, int DH, int QT, int NW, int KC, bool PAGED, bool FINE>
__global__ __launch_bounds__(NW * 64, waves_of(sizeof(T), DH, QT)) void k_prefix_fwd(PrefixArgs a) {
  constexpr int NT = NW * 64, ROWS = NW * QT * 16, NB = DH / 16, ND = DH / 32;
  typedef Tile<T, DH, KC> L;
  typedef Form<T> F;
  typedef typename F::Op Op;
  typedef typename L::Elem E;
  constexpr int PER_T = KC * DH / 8 / NT, STEP = NT / (DH / 8);
  constexpr int NBUF = sizeof(T) == 4 ? 1 : 2;
  constexpr int NS = sizeof(T) * DH * QT > 256 ? 1 : 2;
  static_assert(ROWS <= NT && KC * DH / 8 % NT == 0 && KC % (32 * NS) == 0 && KC <= NT, "tile shape");
  __shared__ __attribute__((aligned(16))) E Ks_[NBUF][L::SIZE], Vs_[NBUF][L::SIZE];
  __shared__ int s_off[ROWS + 1];
  // by chunk parity: the last chunk whose values are not all finite, the last chunk with keys of pages outside the
  // pool, and those keys; rows of the next own chunks
  __shared__ int s_odd[2], s_holes[2], s_hole[2][KC];
  // FINE: the infinities (1, 2: -infinity) and NaNs (4) of every column of the shared values; whether there are any
  __shared__ int s_wild[FINE ? DH : 1], s_any_wild;
  __shared__ long long s_at[2][KC];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g4 = lane >> 4, c16 = lane & 15;
  // Workgroups that read the same keys, or the same lines of them, share an XCD's L2; where there are none, the ranges
  // of a request are spread over the XCDs.
  int id = a.tiles == 1 && sizeof(T) * DH >= 128 ? (int)blockIdx.x : xcd_tile(blockIdx.x, gridDim.x);
  const int t = id % a.tiles;
  id /= a.tiles;
  const int g = id % a.Hkv, range = id / a.Hkv;
  int b = range / a.splits, z = range % a.splits, splits = a.splits;
  if (a.by_length) {                               // uniform
    const Ranges mine = ranges_of_lane(a);
    b = __popcll(__ballot(lane < a.B && mine.first + mine.n <= range));
    if (b >= a.B) return;                          // left over
    z = range - __builtin_amdgcn_readlane(mine.first, b);
    splits = __builtin_amdgcn_readlane(mine.n, b);
  }
  const int r0 = t * ROWS, r1 = min(r0 + ROWS, a.R), sg = a.S * a.G;
  const int k0 = r0 / sg, nb = (r1 - 1) / sg - k0 + 1;
  if (tid < 2) s_odd[tid] = s_holes[tid] = -1;
  if (tid < KC) s_hole[0][tid] = s_hole[1][tid] = -1;
  if (FINE && tid < DH) s_wild[tid] = s_any_wild = 0;
  // This workgroup's share of the shared chunks and, below, of the own chunks.  The shared ones need no more than ctx_len,
  // so they are under way while the lists' lengths, packing and pages are found.
  const int nctx = ctx_rows(a, b), cctx = (nctx + KC - 1) / KC;
  const int cb = (int)((long long)cctx * z / splits), cm = (int)((long long)cctx * (z + 1) / splits);

  // The loads are unconditional: rows that do not count read one that exists and are cleared when they are staged.
  V8<T> kreg[PER_T], vreg[PER_T];
  const int key0 = tid / (DH / 8), d0 = tid % (DH / 8) * 8;            // this thread's part of a chunk: keys key0 + p STEP
  const unsigned ctx_at = (key0 * a.ctx_ld + d0) * sizeof(T), ctx_step = STEP * a.ctx_ld * sizeof(T);   // bytes
  auto load_ctx = [&](int c) __attribute__((always_inline)) {
    const long long base = ((long long)b * a.T + c * KC) * a.ctx_ld + g * DH;
    const T *kp = static_cast<const T*>(a.ctx_k) + base, *vp = static_cast<const T*>(a.ctx_v) + base;
    if ((c + 1) * KC <= nctx) {                    // uniform
#pragma unroll
      for (int p = 0; p < PER_T; ++p) {
        kreg[p] = ld8_at(kp, ctx_at + p * ctx_step);
        vreg[p] = ld8_at(vp, ctx_at + p * ctx_step);
      }
      return;
    }
    const int last = nctx - c * KC - 1;
#pragma unroll
    for (int p = 0; p < PER_T; ++p) {
      const unsigned at = (min(key0 + p * STEP, last) * a.ctx_ld + d0) * sizeof(T);
      kreg[p] = ld8_at(kp, at);
      vreg[p] = ld8_at(vp, at);
    }
  };
  if (cb < cm) load_ctx(cb);
  Row row[QT];
  V8<T> qreg[QT][ND];
  Op qf[QT][ND];
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    row[i] = row_of(a, b, g, r0 + (wave * QT + i) * 16 + c16);
    const T* Q = static_cast<const T*>(a.q) + row[i].at * a.q_ld + row[i].h * DH;
#pragma unroll
    for (int c = 0; c < ND; ++c) qreg[i][c] = ld8(Q + c * 32 + g4 * 8);
  }

  pack_own<NT>(a, b, k0, nb, s_off);
  const int nown = __builtin_amdgcn_readfirstlane(s_off[nb]), cown = (nown + KC - 1) / KC;
  const int ob = (int)((long long)cown * z / splits), oe = (int)((long long)cown * (z + 1) / splits);
  int gone = 0, hole = 0;                          // bit p: the key does not count; because its page is outside the pool
  auto load_own = [&](int c) __attribute__((always_inline)) {
    const T *kp = static_cast<const T*>(a.own_k) + g * DH + d0, *vp = static_cast<const T*>(a.own_v) + g * DH + d0;
    gone = hole = 0;
#pragma unroll
    for (int p = 0; p < PER_T; ++p) {
      const long long x = s_at[c & 1][key0 + p * STEP], at = max(x, 0LL) * a.own_ld;
      gone |= (x < 0) << p;
      if (PAGED) hole |= (x == -1) << p;
      kreg[p] = ld8(kp + at);
      vreg[p] = ld8(vp + at);
    }
  };
  // own rows are found one chunk before they are loaded, so that a page table's latency is hidden as well
  OwnAt<PAGED> found;
  auto find = [&](int c) __attribute__((always_inline)) {
    if (c < oe && tid < KC) found.find(a, b, k0, nb, s_off, c * KC + tid);
  };
  auto first_own = [&]() __attribute__((always_inline)) {
    find(ob);
    if (tid < KC) s_at[ob & 1][tid] = found.row(a);
  };
  if (cb >= cm && ob < oe) {                       // uniform
    first_own();
    lds_barrier();
    load_own(ob);
    find(ob + 1);
  }

  int lo[QT], hi[QT];                              // the packed own rows that the row sees
  // of the wave's tile, uniform: bounds of what its rows see, and (empty where they belong to several lists) what every
  // row sees.  lo does not fall from row to row, nor hi within a list; rows past q_len may see anything.
  int wlo[QT], whi[QT], alo[QT], ahi[QT];
  float m_run[QT], l_run[QT];                      // maximum of q.k; l_run: this lane's keys only, until the end
  f32x4 o[QT][NB];
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    lo[i] = s_off[row[i].k - k0];
    hi[i] = lo[i] + row[i].own;
    wlo[i] = __builtin_amdgcn_readlane(lo[i], 0);
    alo[i] = __builtin_amdgcn_readlane(lo[i], 15);
    whi[i] = __builtin_amdgcn_readlane(s_off[row[i].k - k0 + 1], 15);
    ahi[i] = wlo[i] == alo[i] ? __builtin_amdgcn_readlane(hi[i], 0) : -1;
    if (__any(!row[i].live)) {
#pragma unroll
      for (int c = 0; c < ND; ++c)
        if (!row[i].live) qreg[i][c] = V8<T>{};
    }
#pragma unroll
    for (int c = 0; c < ND; ++c) {
      if (a.scale < 0) qreg[i][c] = -qreg[i][c];   // exact; the largest score is then the largest product
      qf[i][c] = F::of(qreg[i][c]);
    }
    m_run[i] = -INFINITY;
    l_run[i] = 0.f;
#pragma unroll
    for (int n = 0; n < NB; ++n) o[i][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float sl2 = score_unit(a.scale), lag = fminf(8.f / sl2, 1e30f);

  // Products q.k of tiles [i0, i1) with 32 keys.
  auto scores = [&](const E* Ks, int kb, int rl, int i0, int i1, float (&s)[QT][8]) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      f32x4 acc[QT];
#pragma unroll
      for (int i = 0; i < QT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        const Op kf = L::rows(Ks, kb + 16 * x, d, rl);
#pragma unroll
        for (int i = i0; i < i1; ++i) acc[i] = mma(kf, qf[i][d], acc[i]);
      }
#pragma unroll
      for (int i = i0; i < i1; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i][4 * x + j] = acc[i][j];
    }
  };
  // one chain: two values an instruction
  auto max8 = [&](float m, const float (&s)[8]) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 8; j += 2) m = fmaxf(fmaxf(m, s[j]), s[j + 1]);
    return m;
  };
  // Moves the reference of tile i's rows to the largest product (mx: this lane's) where that is more than `lag` above
  // it.  The reference is the running maximum, but it follows only once a score is 8 / log2(e) above it: a probability
  // is then at most 2^8, of no consequence to fp32 sums or to bf16's relative rounding, while with the exact maximum
  // some row of a tile moves in most steps (32 x 64 x 1024 rows: 40.6 us, 39.2 so).  Whether a row's reference moves
  // depends on that row alone.
  auto follow = [&](int i, float mx) __attribute__((always_inline)) {
    const float top = rows_max(mx);
    if (top > m_run[i] + lag) {
      const float alpha = __builtin_amdgcn_exp2f((m_run[i] - top) * sl2);
      m_run[i] = top;
      l_run[i] *= alpha;
#pragma unroll
      for (int n = 0; n < NB; ++n) o[i][n] *= alpha;
    }
  };
  // Probabilities against the reference, added to the sum, as the operand of the product with the values.  bf16 rounds them,
  // for one product in place of two (out off by 2.0e-3 to 2.2e-3 of its norm, its own rounding 1.66e-3).  FINE: what that
  // rounding cut is a second one.  A training step over few keys needs it, as its gradient takes D = dout . out from out and
  // ds = p (dp - D) may be small beside D: keys 1 + 2, dq off by 3.1e-3 of its norm without, 2.3e-3 with; 4 + 11 2.6e-3,
  // 2.3e-3; 130 + 44 2.40e-3, 2.36e-3; 1024 + 64 the same, at 142 us a step for 155.
  auto probs = [&](int i, float (&s)[8], Op& fine) __attribute__((always_inline)) {
    const float ref = m_run[i] == -INFINITY ? 0.f : m_run[i] * sl2;   // a row without keys so far: exp2(-inf) = 0
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = __builtin_amdgcn_exp2f(fmaf(s[j], sl2, -ref));
    l_run[i] += ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
    const Op p = F::of(s);
    if constexpr (FINE) {
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] -= F::value(p, j);
      fine = F::of(s);
    }
    return p;
  };
  auto all_finite = [&]() __attribute__((always_inline)) {             // this thread's values
    unsigned top = 0;
#pragma unroll
    for (int p = 0; p < PER_T; ++p) top = peak(top, vreg[p]);
    return finite<T>(top);
  };
  auto stage = [&](E* Ks, E* Vs) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < PER_T; ++p) {
      L::template put<false>(Ks, key0 + p * STEP, d0 / 8, kreg[p]);
      L::template put<false>(Vs, key0 + p * STEP, d0 / 8, vreg[p]);
    }
  };

  // A value of the chunk that is not finite would reach, in a product, the rows that do not see its key, as 0 times infinity.
  // The products take a zero in its place, so that the other rows' results have the bits that they have beside finite
  // values, and this adds it to tile i's rows that see it: those with from <= key < to, of the 32 keys from kb on.
  auto add_odd = [&](const E* Vs, int kb, int i, int from, int to, const Op& pb, const Op& pf) __attribute__((always_inline)) {
#pragma unroll 1
    for (int key = 0; key < 32; ++key) {
      float e = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float p = F::value(pb, j);
        if (FINE) p += F::value(pf, j);
        e = key_of(j, key >> 2 & 3) == key ? p : e;
      }
      e = __shfl(e, (key >> 2 & 3) * 16 + c16);
      if (key < from || key >= to) continue;
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        __builtin_amdgcn_sched_barrier(0);         // few values in registers at a time
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float v = L::value(Vs, kb + key, n * 16 + g4 * 4 + q);
          o[i][n][q] = fmaf(e, __builtin_isfinite(v) ? 0.f : v, o[i][n][q]);
        }
      }
    }
  };

  const bool idle = r0 + wave * QT * 16 >= a.R;    // no row in the wave's tiles
  int rl = L::row_lane(lane), cl = L::col_lane(lane);
  int cur = 0;
  for (int c = cb; c < cm; ++c, cur ^= NBUF - 1) {
    E *Ks = Ks_[cur], *Vs = Vs_[cur];
    if constexpr (NBUF == 1) lds_barrier();        // the previous chunk is no longer read
    if ((c + 1) * KC > nctx) {                     // uniform
#pragma unroll
      for (int p = 0; p < PER_T; ++p)
        if (c * KC + key0 + p * STEP >= nctx) kreg[p] = vreg[p] = V8<T>{};
    }
    if constexpr (FINE) {
      // Infinity times a probability's second part, which may be zero or negative, is not the infinity that it has to be.
      // Every row sees every shared key: such a value makes its column infinite, or NaN, in all of them, at the end.
      if (!all_finite()) {
#pragma unroll
        for (int p = 0; p < PER_T; ++p) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float v = to_f32((T)vreg[p][j]);
            if (!__builtin_isfinite(v)) atomicOr(&s_wild[d0 + j], v != v ? 4 : v > 0 ? 1 : 2);
          }
          vreg[p] = finite_of(vreg[p]);
        }
        s_any_wild = 1;
      }
    }
    stage(Ks, Vs);
    if (c + 1 == cm && ob < oe) first_own();       // uniform; the first own chunk follows
    lds_barrier();   // two buffers: also the end of every wave's reads of the one written next
    if (c + 1 < cm) {
      load_ctx(c + 1);
    } else if (ob < oe) {
      load_own(ob);
      find(ob + 1);
    }
    if (idle) continue;
    rl = fresh(rl);
    cl = fresh(cl);
    // Steps of NS 32-key blocks: the products of every tile and block first, one branch for the references, then the
    // probabilities and the products with the values, so that the tiles' and blocks' chains overlap.
#pragma unroll
    for (int kb = 0; kb < KC; kb += 32 * NS) {
      const int left = nctx - c * KC - kb;         // keys of the step
      if (left <= 0) break;                        // uniform
      float s[NS][QT][8];
#pragma unroll
      for (int u = 0; u < NS; ++u) scores(Ks, kb + 32 * u, rl, 0, QT, s[u]);
      if (left < 32 * NS) {                        // uniform
        const int end = left - 4 * g4;
#pragma unroll
        for (int u = 0; u < NS; ++u)
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (32 * u + key_of(j) >= end) {
#pragma unroll
              for (int i = 0; i < QT; ++i) s[u][i][j] = -INFINITY;
            }
      }
      float mx[QT];
      bool move = false;
#pragma unroll
      for (int i = 0; i < QT; ++i) {
        mx[i] = m_run[i];
#pragma unroll
        for (int u = 0; u < NS; ++u) mx[i] = max8(mx[i], s[u][i]);
        move |= mx[i] > m_run[i] + lag;
      }
      if (__any(move)) {
#pragma unroll
        for (int i = 0; i < QT; ++i) follow(i, mx[i]);
      }
      Op pb[NS][QT], pf[NS][QT];
#pragma unroll
      for (int u = 0; u < NS; ++u)
#pragma unroll
        for (int i = 0; i < QT; ++i) pb[u][i] = probs(i, s[u][i], pf[u][i]);
#pragma unroll
      for (int u = 0; u < NS; ++u)
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          const Op vf = L::cols(Vs, kb + 32 * u, n, cl);
#pragma unroll
          for (int i = 0; i < QT; ++i) {
            if (FINE) o[i][n] = mma(vf, pf[u][i], o[i][n]);
            o[i][n] = mma(vf, pb[u][i], o[i][n]);
          }
        }
    }
  }

  for (int c = ob; c < oe; ++c, cur ^= NBUF - 1) {
    E *Ks = Ks_[cur], *Vs = Vs_[cur];
    if constexpr (NBUF == 1) lds_barrier();
    if (__any(gone)) {
#pragma unroll
      for (int p = 0; p < PER_T; ++p) {
        if (gone >> p & 1) kreg[p] = vreg[p] = V8<T>{};
        if (PAGED && hole >> p & 1) s_hole[c & 1][key0 + p * STEP] = s_holes[c & 1] = c;
      }
    }
    if (!all_finite()) s_odd[c & 1] = c;
    stage(Ks, Vs);
    if (tid < KC) s_at[(c + 1) & 1][tid] = found.row(a);
    lds_barrier();
    if (c + 1 < oe) load_own(c + 1);
    find(c + 2);
    if (idle) continue;
    rl = fresh(rl);
    cl = fresh(cl);
    const bool odd = __builtin_amdgcn_readfirstlane(s_odd[c & 1]) == c;
    const bool holes = PAGED && __builtin_amdgcn_readfirstlane(s_holes[c & 1]) == c;
#pragma unroll 1
    for (int kb = 0; kb < KC; kb += 32) {
      const int x0 = c * KC + kb;
      if (x0 >= nown) break;                       // uniform
#pragma unroll
      for (int i = 0; i < QT; ++i) {
        if (x0 >= whi[i] || x0 + 32 <= wlo[i]) continue;   // uniform: no row of the tile sees a key of the step
        float all[QT][8];
        scores(Ks, kb, rl, i, i + 1, all);
        float (&s)[8] = all[i];
        if (x0 < alo[i] || x0 + 32 > ahi[i]) {     // uniform
          const int from = lo[i] - x0 - 4 * g4, to = hi[i] - x0 - 4 * g4;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (key_of(j) < from || key_of(j) >= to) s[j] = -INFINITY;
        }
        if (holes) {                               // uniform
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (s_hole[c & 1][kb + key_of(j, g4)] == c) s[j] = -INFINITY;
        }
        const float mx = max8(m_run[i], s);
        if (__any(mx > m_run[i] + lag)) follow(i, mx);
        Op pf;
        const Op pb = probs(i, s, pf);
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          Op vf = L::cols(Vs, kb, n, cl);
          if (odd) vf = finite_of(vf);             // uniform
          if (FINE) o[i][n] = mma(vf, pf, o[i][n]);
          o[i][n] = mma(vf, pb, o[i][n]);
        }
        if (odd) add_odd(Vs, kb, i, lo[i] - x0, hi[i] - x0, pb, pf);
      }
    }
  }

  if (FINE && __builtin_amdgcn_readfirstlane(s_any_wild)) {   // uniform
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int w = s_wild[n * 16 + g4 * 4 + q];
        const float v = w == 0 ? 0.f : w == 1 ? INFINITY : w == 2 ? -INFINITY : NAN;
#pragma unroll
        for (int i = 0; i < QT; ++i) o[i][n][q] += v;
      }
  }

#pragma unroll
  for (int i = 0; i < QT; ++i) {
    const float l = rows_sum(l_run[i]);
    if (r0 + (wave * QT + i) * 16 + c16 >= a.R) continue;
    const float m2 = m_run[i] * sl2;
    const long long ro = row[i].at * a.Hq + row[i].h;
    if (a.splits > 1) {
      const long long at = ro + (long long)(range - b) * a.K * a.S * a.Hq;   // [range][row of the request]
      float* po = a.part_o + at * DH;
#pragma unroll
      for (int n = 0; n < NB; ++n) *reinterpret_cast<f32x4*>(po + n * 16 + g4 * 4) = o[i][n];
      if (g4 == 0) {
        a.part_ml[at * 2] = m2;
        a.part_ml[at * 2 + 1] = l;
      }
      continue;
    }
    const bool none = !row[i].live || l == 0.f;    // no key; a NaN score leaves a NaN sum
    const float inv = none ? 0.f : 1.f / l;
    if (__any(none)) {
#pragma unroll
      for (int n = 0; n < NB; ++n)
        if (none) o[i][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int n = 0; n < NB; ++n) store_out<T>(a, row[i].at, row[i].h * DH + n * 16 + g4 * 4, o[i][n] * inv);
    if (a.lse && g4 == 0) a.lse[ro] = none ? -INFINITY : (m2 + log2f(l)) * kLn2;
  }
}

// Joins the key ranges of a row: DH / 4 threads a row, ranges in ascending order.
// Bound: the partial sums, from HBM or L2 (4096 rows of 128 in 16 ranges, 34 MB: 9.9 us); one trip for a few (3.9 us).
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_prefix_join(PrefixArgs a) {
  const long long rows = (long long)a.B * a.K * a.S * a.Hq;
  const long long e = (long long)blockIdx.x * 256 + threadIdx.x, ro = e / (DH / 4);
  const int d0 = (int)(e % (DH / 4)) * 4;
  int b = (int)(min(ro, rows - 1) / (rows / a.B)), first = b * a.splits, splits = a.splits;
  if (a.by_length) {                               // uniform
    const Ranges mine = ranges_of_lane(a);
    first = __shfl(mine.first, b);
    splits = __shfl(mine.n, b);
  }
  if (ro >= rows) return;
  const long long at = ro / a.Hq, step = rows / a.B, from = (first - b) * step + ro;
  const int h = (int)(ro % a.Hq), bk = (int)(at / a.S), s = (int)(at % a.S);
  const bool dead = s >= q_rows(a, bk);
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int z0 = 0; z0 < splits; z0 += 8) {         // eight ranges requested at once
    float2 ml[8];
    f32x4 v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const long long e = min(z0 + u, splits - 1) * step + from;
      ml[u] = reinterpret_cast<const float2*>(a.part_ml)[e];
      v[u] = *reinterpret_cast<const f32x4*>(a.part_o + e * DH + d0);
      if (z0 + u >= splits) ml[u].x = -INFINITY;
    }
    float top = m;
#pragma unroll
    for (int u = 0; u < 8; ++u) top = fmaxf(top, ml[u].x);
    const float ref = top == -INFINITY ? 0.f : top, old = __builtin_amdgcn_exp2f(m - ref);
    m = top;
    l *= old;
    o *= old;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float w = __builtin_amdgcn_exp2f(ml[u].x - ref);
      l = fmaf(ml[u].y, w, l);
      if (ml[u].x != -INFINITY) o += w * v[u];     // a range without keys for the row says nothing
    }
  }
  const bool none = dead || l == 0.f;
  const float inv = none ? 0.f : 1.f / l;
#pragma unroll
  for (int q = 0; q < 4; ++q) o[q] = none ? 0.f : o[q] * inv;
  store_out<T>(a, at, h * DH + d0, o);
  if (a.lse && d0 == 0) a.lse[ro] = none ? -INFINITY : (m + log2f(l)) * kLn2;
}

// ------------------------------------------------------------------------------------------
// Gradient.
// ------------------------------------------------------------------------------------------

// dq: rows and chunks as in the forward, probabilities again from lse.  Before that it forms what the gradient's
// products need of every row and leaves it for dk and dv, in the order of the rows of a (request, key head):
//   x = log2(e) lse (+infinity for a row without keys or past q_len: its probabilities are then 0),
//   y = dout . out,   z, w = the own rows that it sees, numbered k L + j  [z, w).
// ds goes into the product with the keys as it lies in the registers, as the probabilities do in the forward: bf16 rounds it
// there, for one product in place of two (dq off by 2.4e-3 of its norm, of which its own rounding makes 1.66e-3).
// Bound: LDS (58% of the time: every wave reads keys twice and values once for its 16 rows) and the vector unit (50%)
// beside 29% of matrix cores (64 x 1024 rows of 1088 keys, heads of 64: 47 us, 564 TFLOP/s); fp32 the vector unit (63%;
// 256 x 550 rows, heads of 32: 72 us, 100 TFLOP/s; at heads of 64 8 registers, 36 bytes a lane, are spilled).
template <typename T, int DH, int QT, int NW, int KC>
__global__ __launch_bounds__(NW * 64, waves_of(sizeof(T), DH, QT)) void k_prefix_dq(PrefixGradArgs p) {
  const PrefixArgs& a = p.f;
  constexpr int NT = NW * 64, ROWS = NW * QT * 16, NB = DH / 16, ND = DH / 32;
  typedef Tile<T, DH, KC> L;
  typedef Form<T> F;
  typedef typename F::Op Op;
  typedef typename L::Elem E;
  constexpr int PER_T = KC * DH / 8 / NT, STEP = NT / (DH / 8);
  constexpr int NBUF = sizeof(T) == 4 ? 1 : 2;
  static_assert(ROWS <= NT && KC * DH / 8 % NT == 0 && KC % 32 == 0, "tile shape");
  __shared__ __attribute__((aligned(16))) E Ks_[NBUF][L::SIZE], Vs_[NBUF][L::SIZE];
  __shared__ int s_off[ROWS + 1];
  __shared__ long long s_at[2][KC];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g4 = lane >> 4, c16 = lane & 15;
  int id = xcd_tile(blockIdx.x, gridDim.x);
  const int z = id % a.splits;
  id /= a.splits;
  const int t = id % a.tiles;
  id /= a.tiles;
  const int g = id % a.Hkv, b = id / a.Hkv;
  const int r0 = t * ROWS, r1 = min(r0 + ROWS, a.R), sg = a.S * a.G;
  const int k0 = r0 / sg, nb = (r1 - 1) / sg - k0 + 1;
  pack_own<NT>(a, b, k0, nb, s_off);
  const int nctx = ctx_rows(a, b), nown = __builtin_amdgcn_readfirstlane(s_off[nb]);
  const int cctx = (nctx + KC - 1) / KC, chunks = cctx + (nown + KC - 1) / KC;
  const int cb = (int)((long long)chunks * z / a.splits), ce = (int)((long long)chunks * (z + 1) / a.splits);
  const int cm = min(max(cctx, cb), ce);

  V8<T> kreg[PER_T], vreg[PER_T];
  const int key0 = tid / (DH / 8), d0 = tid % (DH / 8) * 8;
  const unsigned ctx_at = (key0 * a.ctx_ld + d0) * sizeof(T), ctx_step = STEP * a.ctx_ld * sizeof(T);   // bytes
  auto load_ctx = [&](int c) __attribute__((always_inline)) {
    const long long base = ((long long)b * a.T + c * KC) * a.ctx_ld + g * DH;
    const T *kp = static_cast<const T*>(a.ctx_k) + base, *vp = static_cast<const T*>(a.ctx_v) + base;
    if ((c + 1) * KC <= nctx) {                    // uniform
#pragma unroll
      for (int q = 0; q < PER_T; ++q) {
        kreg[q] = ld8_at(kp, ctx_at + q * ctx_step);
        vreg[q] = ld8_at(vp, ctx_at + q * ctx_step);
      }
      return;
    }
    const int last = nctx - c * KC - 1;
#pragma unroll
    for (int q = 0; q < PER_T; ++q) {
      const unsigned at = (min(key0 + q * STEP, last) * a.ctx_ld + d0) * sizeof(T);
      kreg[q] = ld8_at(kp, at);
      vreg[q] = ld8_at(vp, at);
    }
  };
  int gone = 0;
  auto load_own = [&](int c) __attribute__((always_inline)) {
    const T *kp = static_cast<const T*>(a.own_k) + g * DH + d0, *vp = static_cast<const T*>(a.own_v) + g * DH + d0;
    gone = 0;
#pragma unroll
    for (int q = 0; q < PER_T; ++q) {
      const long long x = s_at[c & 1][key0 + q * STEP], at = max(x, 0LL) * a.own_ld;
      gone |= (x < 0) << q;
      kreg[q] = ld8(kp + at);
      vreg[q] = ld8(vp + at);
    }
  };
  OwnAt<false> found;
  auto find = [&](int c) __attribute__((always_inline)) {
    if (c < ce && tid < KC) found.find(a, b, k0, nb, s_off, (c - cctx) * KC + tid);
  };
  if (cb < cm) {
    load_ctx(cb);
  } else if (cm < ce) {
    find(cm);
    if (tid < KC) s_at[cm & 1][tid] = found.row(a);
    lds_barrier();
    load_own(cm);
    find(cm + 1);
  }

  Op qf[QT][ND], df[QT][ND];
  int lo[QT], hi[QT], wlo[QT], whi[QT], alo[QT], ahi[QT];              // as in the forward
  float lse2[QT], delta[QT];
  f32x4 o[QT][NB];
#pragma unroll
  for (int i = 0; i < QT; ++i) {
    const int r = r0 + (wave * QT + i) * 16 + c16;
    const Row row = row_of(a, b, g, r);
    const T* Q = static_cast<const T*>(a.q) + row.at * a.q_ld + row.h * DH;
    const T* D = static_cast<const T*>(p.dout) + row.at * p.dout_ld + row.h * DH;
    const T* O = static_cast<const T*>(a.out) + row.at * a.out_ld + row.h * DH;
    const signed char* rest = a.out_rest ? a.out_rest + (row.at * a.Hq + row.h) * DH : nullptr;
    float v = 0.f;
#pragma unroll
    for (int c = 0; c < ND; ++c) {
      qf[i][c] = F::of(row.live ? ld8(Q + c * 32 + g4 * 8) : V8<T>{});
      const V8<T> dout = row.live ? ld8(D + c * 32 + g4 * 8) : V8<T>{};
      df[i][c] = F::of(dout);
      const V8<T> out = row.live ? ld8(O + c * 32 + g4 * 8) : V8<T>{};
      uint2 step = make_uint2(0, 0);
      if (sizeof(T) == 2 && rest) step = *reinterpret_cast<const uint2*>(rest + c * 32 + g4 * 8);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int w = (int)((j < 4 ? step.x : step.y) << (24 - 8 * (j & 3))) >> 24;
        v = fmaf(to_f32((T)dout[j]), with_rest((T)out[j], row.live ? w : 0), v);
      }
    }
    delta[i] = rows_sum(v);
    const float lse = row.live ? a.lse[row.at * a.Hq + row.h] : -INFINITY;
    lse2[i] = lse == -INFINITY ? INFINITY : lse * kLog2e;
    if (z == 0 && g4 == 0 && r < a.R)
      p.rows[((long long)b * a.Hkv + g) * a.R + r] =
          make_float4(lse2[i], delta[i], __int_as_float(row.k * a.L), __int_as_float(row.k * a.L + row.own));
    lo[i] = s_off[row.k - k0];
    hi[i] = lo[i] + row.own;
    wlo[i] = __builtin_amdgcn_readlane(lo[i], 0);
    alo[i] = __builtin_amdgcn_readlane(lo[i], 15);
    whi[i] = __builtin_amdgcn_readlane(s_off[row.k - k0 + 1], 15);
    ahi[i] = wlo[i] == alo[i] ? __builtin_amdgcn_readlane(hi[i], 0) : -1;
#pragma unroll
    for (int n = 0; n < NB; ++n) o[i][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float sl2 = a.scale * kLog2e;

  auto stage = [&](E* Ks, E* Vs) __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < PER_T; ++q) {
      L::template put<true>(Ks, key0 + q * STEP, d0 / 8, kreg[q]);
      L::template put<true>(Vs, key0 + q * STEP, d0 / 8, vreg[q]);
    }
  };
  // p (dp - delta) of tile i for the 32 keys from kb on
  auto dscores = [&](const E* Ks, const E* Vs, int kb, int rl, int i, float (&e)[8]) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      f32x4 s = {0.f, 0.f, 0.f, 0.f}, dp = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        s = mma(L::rows(Ks, kb + 16 * x, d, rl), qf[i][d], s);
        dp = mma(L::rows(Vs, kb + 16 * x, d, rl), df[i][d], dp);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) e[4 * x + j] = __builtin_amdgcn_exp2f(fmaf(s[j], sl2, -lse2[i])) * (dp[j] - delta[i]);
    }
  };

  const bool idle = r0 + wave * QT * 16 >= a.R;
  int rl = L::row_lane(lane), cl = L::col_lane(lane);
  int cur = 0;
  for (int c = cb; c < cm; ++c, cur ^= NBUF - 1) {
    E *Ks = Ks_[cur], *Vs = Vs_[cur];
    if constexpr (NBUF == 1) lds_barrier();
    if ((c + 1) * KC > nctx) {                     // uniform
#pragma unroll
      for (int q = 0; q < PER_T; ++q)
        if (c * KC + key0 + q * STEP >= nctx) kreg[q] = vreg[q] = V8<T>{};
    }
    stage(Ks, Vs);
    if (c + 1 == cm && cm < ce) {                  // uniform; the first own chunk follows
      find(cm);
      if (tid < KC) s_at[cm & 1][tid] = found.row(a);
    }
    lds_barrier();
    if (c + 1 < cm) {
      load_ctx(c + 1);
    } else if (cm < ce) {
      load_own(cm);
      find(cm + 1);
    }
    if (idle) continue;
    rl = fresh(rl);
    cl = fresh(cl);
    const int left = nctx - c * KC;                // keys of the chunk
    Op ds[KC / 32][QT];
#pragma unroll
    for (int u = 0; u < KC / 32; ++u)
#pragma unroll
      for (int i = 0; i < QT; ++i) {
        float e[8];
        dscores(Ks, Vs, 32 * u, rl, i, e);
        if (left < KC) {                           // uniform; a key past the length is zero, its probability may be anything
          const int end = left - 4 * g4;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (32 * u + key_of(j) >= end) e[j] = 0.f;
        }
        ds[u][i] = F::of(e);
      }
#pragma unroll
    for (int u = 0; u < KC / 32; ++u)
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const Op kt = L::cols(Ks, 32 * u, n, cl);
#pragma unroll
        for (int i = 0; i < QT; ++i) o[i][n] = mma(kt, ds[u][i], o[i][n]);
      }
  }

  for (int c = cm; c < ce; ++c, cur ^= NBUF - 1) {
    E *Ks = Ks_[cur], *Vs = Vs_[cur];
    if constexpr (NBUF == 1) lds_barrier();
    if (__any(gone)) {
#pragma unroll
      for (int q = 0; q < PER_T; ++q)
        if (gone >> q & 1) kreg[q] = vreg[q] = V8<T>{};
    }
    stage(Ks, Vs);
    if (tid < KC) s_at[(c + 1) & 1][tid] = found.row(a);
    lds_barrier();
    if (c + 1 < ce) load_own(c + 1);
    find(c + 2);
    if (idle) continue;
    rl = fresh(rl);
    cl = fresh(cl);
#pragma unroll 1
    for (int kb = 0; kb < KC; kb += 32) {
      const int x0 = (c - cctx) * KC + kb;
      if (x0 >= nown) break;                                           // uniform
#pragma unroll
      for (int i = 0; i < QT; ++i) {
        if (x0 >= whi[i] || x0 + 32 <= wlo[i]) continue;               // uniform
        float e[8];
        dscores(Ks, Vs, kb, rl, i, e);
        if (x0 < alo[i] || x0 + 32 > ahi[i]) {                         // uniform
          const int from = lo[i] - x0 - 4 * g4, to = hi[i] - x0 - 4 * g4;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (key_of(j) < from || key_of(j) >= to) e[j] = 0.f;
        }
        const Op ds = F::of(e);
#pragma unroll
        for (int n = 0; n < NB; ++n) o[i][n] = mma(L::cols(Ks, kb, n, cl), ds, o[i][n]);
      }
    }
  }

#pragma unroll
  for (int i = 0; i < QT; ++i) {
    const int r = r0 + (wave * QT + i) * 16 + c16;
    if (r >= a.R) continue;
    const Row row = row_of(a, b, g, r);
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const f32x4 v = row.live ? o[i][n] * a.scale : f32x4{0.f, 0.f, 0.f, 0.f};
      if (a.splits > 1) {
        const long long rows = (long long)a.B * a.K * a.S * a.Hq;
        *reinterpret_cast<f32x4*>(a.part_o + (z * rows + row.at * a.Hq + row.h) * DH + n * 16 + g4 * 4) = v;
      } else {
        st4(static_cast<T*>(p.dq) + row.at * p.dq_ld + row.h * DH + n * 16 + g4 * 4, v);
      }
    }
  }
}

// dk and dv of a tile of keys: NW waves of KT 16-key tiles whose keys and values stay in registers, the rows stream through
// LDS in chunks of RC.  Tiles 0 .. ctx_tiles - 1 of a (request, key head) hold shared rows and meet every row; the others
// hold own rows (dense, list after list) and meet the rows of their lists.  In the tile's numbering -- shared row, or
// k L + j -- the keys that a row sees are again one interval.  Few tiles: several workgroups share a tile's rows.
// Scores are formed a second time: sums of dq by key tiles would be B K S n_heads dh floats for every tile of 128 keys,
// more traffic than the two products cost.
// Bound: vector unit (44% of the time), LDS and matrix cores (30% each) with two waves a SIMD (64 x 1024 rows of 1088
// keys, heads of 64: 59 us, 602 TFLOP/s); fp32 the vector unit (66%; 256 x 550 rows, heads of 32: 94 us, 102
// TFLOP/s).  fp32 heads of 128 take a whole compute unit's LDS and one wave a SIMD, whose registers hold everything.
// The own tiles' second products spill in bf16, 14 registers at heads of 32 (60 bytes a lane) and 8 at heads of 128 (36 bytes;
// 4 x 1332 rows, 333 + 37 keys: 17.5 us without these products, 20.5 with them).
template <typename T, int DH, int KT, int NW, int RC>
__global__ __launch_bounds__(NW * 64, dkv_waves(DH)) void k_prefix_dkv(PrefixGradArgs p) {
  const PrefixArgs& a = p.f;
  constexpr int NT = NW * 64, COLS = NW * KT * 16, NB = DH / 16, ND = DH / 32;
  typedef Tile<T, DH, RC> L;
  typedef Form<T> F;
  typedef typename F::Op Op;
  typedef typename L::Elem E;
  constexpr int PER_T = RC * DH / 8 / NT, STEP = NT / (DH / 8);
  constexpr bool FINE = sizeof(T) == 2;
  static_assert(RC % 32 == 0 && RC <= NT && RC * DH / 8 % NT == 0, "tile shape");
  __shared__ __attribute__((aligned(16))) E Qs_[2][L::SIZE], Ds_[2][L::SIZE];
  __shared__ __attribute__((aligned(16))) float s_lse[2][RC], s_delta[2][RC];
  __shared__ __attribute__((aligned(16))) int s_lo[2][RC], s_hi[2][RC];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g4 = lane >> 4, c16 = lane & 15;
  // Shared tiles meet every row and come first; the own tiles, a few rows each, fill in behind them.
  const int n_ctx = a.B * a.Hkv * p.ctx_tiles * p.ctx_splits;
  const bool shared = (int)blockIdx.x < n_ctx;
  int id = shared ? xcd_tile(blockIdx.x, n_ctx) : xcd_tile(blockIdx.x - n_ctx, gridDim.x - n_ctx);
  const int splits = shared ? p.ctx_splits : p.own_splits, z = id % splits;
  id /= splits;
  const int tiles = shared ? p.ctx_tiles : p.own_tiles, t = id % tiles;
  id /= tiles;
  const int g = id % a.Hkv, b = id / a.Hkv;
  const int x0 = t * COLS, cols = shared ? a.T : a.K * a.L, sg = a.S * a.G;
  const int nctx = ctx_rows(a, b);
  int rb = 0, re = a.R;
  if (shared) {
    if (x0 >= nctx) re = 0;
  } else {
    rb = x0 / a.L * sg;
    re = ((min(x0 + COLS, cols) - 1) / a.L + 1) * sg;
  }
  const int steps = (re - rb + RC - 1) / RC;
  const int cb = (int)((long long)steps * z / splits), ce = (int)((long long)steps * (z + 1) / splits);

  V8<T> qreg[PER_T], dreg[PER_T];
  float lreg[PER_T];
  float4 rreg;
  const int i0 = tid / (DH / 8), d0 = tid % (DH / 8) * 8;              // this thread's part of a chunk: rows i0 + q STEP
  const float4* rows = p.rows + ((long long)b * a.Hkv + g) * a.R;
  // Rows past the end repeat the last one, with lse = infinity.
  const T *q_base = static_cast<const T*>(a.q), *d_base = static_cast<const T*>(p.dout);
  // uniform: every chunk's rows lie as the first one's do, and q_at, d_at are their byte offsets
  const bool even = RC % a.G == 0 && a.q_ld <= (1 << 23) && p.dout_ld <= (1 << 23);
  unsigned q_at[PER_T], d_at[PER_T];
#pragma unroll
  for (int q = 0; q < PER_T; ++q) {
    const int i = i0 + q * STEP;
    q_at[q] = (i / a.G * a.q_ld + (i % a.G) * DH + d0) * sizeof(T);
    d_at[q] = (i / a.G * p.dout_ld + (i % a.G) * DH + d0) * sizeof(T);
  }
  auto load_chunk = [&](int c) __attribute__((always_inline)) {
    const int r0 = rb + c * RC;                    // a multiple of G
    if (even && r0 + RC <= re) {                   // uniform
      const long long at = (long long)b * a.K * a.S + r0 / a.G;
      const T *qp = q_base + at * a.q_ld + g * a.G * DH, *dp = d_base + at * p.dout_ld + g * a.G * DH;
#pragma unroll
      for (int q = 0; q < PER_T; ++q) {
        qreg[q] = ld8_at(qp, q_at[q]);
        dreg[q] = ld8_at(dp, d_at[q]);
      }
    } else {
#pragma unroll
      for (int q = 0; q < PER_T; ++q) {
        const int r = min(r0 + i0 + q * STEP, re - 1);
        const long long at = (long long)b * a.K * a.S + r / a.G;
        const int h = g * a.G + r % a.G;
        qreg[q] = ld8(q_base + at * a.q_ld + h * DH + d0);
        dreg[q] = ld8(d_base + at * p.dout_ld + h * DH + d0);
      }
    }
    if (a.q_len) {                                 // uniform
#pragma unroll
      for (int q = 0; q < PER_T; ++q) lreg[q] = rows[min(r0 + i0 + q * STEP, re - 1)].x;
    }
    if (tid < RC) rreg = rows[min(r0 + tid, re - 1)];
  };
  if (cb < ce) load_chunk(cb);

  Op kf[KT][ND], vf[KT][ND];
  bool live[KT];
  long long at[KT];                                                     // the key's row of the tensors
  f32x4 dk[KT][NB], dv[KT][NB];
#pragma unroll
  for (int i = 0; i < KT; ++i) {
    const int x = x0 + (wave * KT + i) * 16 + c16;                      // this lane's key
    live[i] = false;
    at[i] = 0;
    if (x < cols) {
      if (shared) {
        live[i] = x < nctx;
        at[i] = (long long)b * a.T + x;
      } else {
        const int bk = b * a.K + x / a.L;
        live[i] = x % a.L < own_rows(a, bk) && q_rows(a, bk) > 0;
        at[i] = (long long)b * cols + x;
      }
    }
    const long long off = at[i] * (shared ? a.ctx_ld : a.own_ld) + g * DH + g4 * 8;
    const T* kp = static_cast<const T*>(shared ? a.ctx_k : a.own_k) + off;
    const T* vp = static_cast<const T*>(shared ? a.ctx_v : a.own_v) + off;
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      kf[i][d] = F::of(live[i] ? ld8(kp + d * 32) : V8<T>{});
      vf[i][d] = F::of(live[i] ? ld8(vp + d * 32) : V8<T>{});
    }
#pragma unroll
    for (int n = 0; n < NB; ++n) dk[i][n] = dv[i][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float sl2 = a.scale * kLog2e;

  int rl = L::row_lane(lane), cl = L::col_lane(lane);

  // q.k and dout.v of 32 rows from kb on with the wave's keys
  auto products = [&](const E* Qs, const E* Ds, int kb, f32x4 (&s)[2][KT],
                      f32x4 (&dp)[2][KT]) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int i = 0; i < KT; ++i) s[u][i] = dp[u][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        const Op qv = L::rows(Qs, kb + 16 * u, d, rl), dv8 = L::rows(Ds, kb + 16 * u, d, rl);
#pragma unroll
        for (int i = 0; i < KT; ++i) {
          s[u][i] = mma(qv, kf[i][d], s[u][i]);
          dp[u][i] = mma(dv8, vf[i][d], dp[u][i]);
        }
      }
    }
  };
  // ... and with them the rows' part of dk and dv; own: rows see the keys [lo, hi)
  auto add = [&](const E* Qs, const E* Ds, int cur, int kb, bool own, const f32x4 (&s)[2][KT],
                 const f32x4 (&dp)[2][KT]) __attribute__((always_inline)) {
    float pe[KT][8], de[KT][8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const f32x4 lse = *reinterpret_cast<const f32x4*>(&s_lse[cur][kb + 16 * u + 4 * g4]);
      const f32x4 delta = *reinterpret_cast<const f32x4*>(&s_delta[cur][kb + 16 * u + 4 * g4]);
#pragma unroll
      for (int i = 0; i < KT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float e = __builtin_amdgcn_exp2f(fmaf(s[u][i][j], sl2, -lse[j]));
          pe[i][4 * u + j] = e;
          de[i][4 * u + j] = e * (dp[u][i][j] - delta[j]);
        }
      if (own) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int l = s_lo[cur][kb + 16 * u + 4 * g4 + j], h = s_hi[cur][kb + 16 * u + 4 * g4 + j];
#pragma unroll
          for (int i = 0; i < KT; ++i) {
            const int x = x0 + (wave * KT + i) * 16 + c16;
            if (x < l || x >= h) pe[i][4 * u + j] = de[i][4 * u + j] = 0.f;
          }
        }
      }
    }
    Op pb[KT], ds[KT];
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      pb[i] = F::of(pe[i]);
      ds[i] = F::of(de[i]);
    }
    // bf16 rounds p and ds of shared keys for the products, whose sums have many rows' terms (dk off by 2.35e-3 of its norm).
    // An own key meets few rows, and one may make most of its sums: bf16 adds what the roundings cut (dk off by 2.4e-3
    // to 3.3e-3 of its norm without, 1.7e-3 with, which is its own rounding; training step of 256 x 550 rows, heads of 32,
    // 87 us without, 93 with, of 64 x 1024 rows, heads of 64, the same).
    Op pf[KT], df[KT];
    if (FINE && own) {
#pragma unroll
      for (int i = 0; i < KT; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          pe[i][j] -= F::value(pb[i], j);
          de[i][j] -= F::value(ds[i], j);
        }
        pf[i] = F::of(pe[i]);
        df[i] = F::of(de[i]);
      }
    }
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const Op dt = L::cols(Ds, kb, n, cl), qt = L::cols(Qs, kb, n, cl);
#pragma unroll
      for (int i = 0; i < KT; ++i) {
        if (FINE && own) {
          dv[i][n] = mma(dt, pf[i], dv[i][n]);
          dk[i][n] = mma(qt, df[i], dk[i][n]);
        }
        dv[i][n] = mma(dt, pb[i], dv[i][n]);
        dk[i][n] = mma(qt, ds[i], dk[i][n]);
      }
    }
  };

  // Two loops, so that each keeps the sums in place.
  int cur = 0;
  auto stage = [&](int c) __attribute__((always_inline)) {
    E *Qs = Qs_[cur], *Ds = Ds_[cur];
#pragma unroll
    for (int q = 0; q < PER_T; ++q) {
      if (a.q_len && lreg[q] == INFINITY) qreg[q] = dreg[q] = V8<T>{};  // a row that sees nothing may hold anything
      L::template put<true>(Qs, i0 + q * STEP, d0 / 8, qreg[q]);
      L::template put<true>(Ds, i0 + q * STEP, d0 / 8, dreg[q]);
    }
    if (tid < RC) {
      const bool past = rb + c * RC + tid >= re;
      s_lse[cur][tid] = past ? INFINITY : rreg.x;
      s_delta[cur][tid] = rreg.y;
      s_lo[cur][tid] = __float_as_int(rreg.z);
      s_hi[cur][tid] = __float_as_int(past ? rreg.z : rreg.w);
    }
    lds_barrier();
    if (c + 1 < ce) load_chunk(c + 1);
    rl = fresh(rl);
    cl = fresh(cl);
  };
  if (shared) {
    for (int c = cb; c < ce; ++c, cur ^= 1) {
      stage(c);
      if (x0 + wave * KT * 16 >= nctx) continue;                        // uniform: the wave's keys are past the length
#pragma unroll
      for (int kb = 0; kb < RC; kb += 32) {                             // rows past the end have probability 0
        f32x4 s[2][KT], dp[2][KT];
        products(Qs_[cur], Ds_[cur], kb, s, dp);
        add(Qs_[cur], Ds_[cur], cur, kb, false, s, dp);
      }
    }
  } else {
    for (int c = cb; c < ce; ++c, cur ^= 1) {
      stage(c);
#pragma unroll 1
      for (int kb = 0; kb < RC; kb += 32) {
        if (rb + c * RC + kb >= re) break;                              // uniform
        // uniform: lists of the block's rows, keys of the wave
        const int first = __builtin_amdgcn_readfirstlane(s_lo[cur][kb]);
        const int last = __builtin_amdgcn_readfirstlane(s_lo[cur][kb + 31]);
        const int xa = x0 + wave * KT * 16;
        if (first >= xa + KT * 16 || last + a.L <= xa) continue;
        f32x4 s[2][KT], dp[2][KT];
        products(Qs_[cur], Ds_[cur], kb, s, dp);
        add(Qs_[cur], Ds_[cur], cur, kb, true, s, dp);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < KT; ++i) {
    const int x = x0 + (wave * KT + i) * 16 + c16;
    if (x >= cols) continue;
    const long long off = at[i] * (shared ? p.dctx_ld : p.down_ld) + g * DH + g4 * 4;
    T* ko = static_cast<T*>(shared ? p.dctx_k : p.down_k) + off;
    T* vo = static_cast<T*>(shared ? p.dctx_v : p.down_v) + off;
    const long long n_keys = (long long)a.B * cols * a.Hkv;
    float* po = nullptr;
    if (splits > 1) po = (shared ? p.part_ctx : p.part_own) + (z * n_keys + at[i] * a.Hkv + g) * 2 * DH + g4 * 4;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const f32x4 zero = {0.f, 0.f, 0.f, 0.f};                          // a key past its length: its sums mean nothing
      const f32x4 k4 = live[i] ? dk[i][n] * a.scale : zero, v4 = live[i] ? dv[i][n] : zero;
      if (po) {
        *reinterpret_cast<f32x4*>(po + n * 16) = k4;
        *reinterpret_cast<f32x4*>(po + DH + n * 16) = v4;
      } else {
        st4(ko + n * 16, k4);
        st4(vo + n * 16, v4);
      }
    }
  }
}

// Adds the partial sums of dq (key ranges) and of dk and dv (row ranges) in ascending order, in one launch: the first
// blocks[0] workgroups dq, the next blocks[1] the shared keys, the rest the own keys.
// Bound: one trip to memory (5328 rows of 128 in 2 parts, 1332 keys in 7 and 1332 in 2, 18 MB: 5.0 us).
struct SumBlocks { unsigned dq, ctx; };
// workgroups that add `bytes` of partial sums in `splits` parts, four sums a thread
long long sum_blocks(size_t bytes, int splits) { return (long long)((bytes / splits + 4095) / 4096); }
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_prefix_sum(PrefixGradArgs p, SumBlocks blocks) {
  const PrefixArgs& a = p.f;
  unsigned blk = blockIdx.x;
  const float* part;
  long long n;                          // rows, or keys with dk and dv side by side
  int splits, heads, ld, width = 2 * DH;
  T *dst, *dst_v = nullptr;
  if (blk < blocks.dq) {                // uniform
    part = a.part_o; n = (long long)a.B * a.K * a.S * a.Hq; splits = a.splits; heads = a.Hq; ld = p.dq_ld; width = DH;
    dst = static_cast<T*>(p.dq);
  } else if ((blk -= blocks.dq) < blocks.ctx) {
    part = p.part_ctx; n = (long long)a.B * a.T * a.Hkv; splits = p.ctx_splits; heads = a.Hkv; ld = p.dctx_ld;
    dst = static_cast<T*>(p.dctx_k); dst_v = static_cast<T*>(p.dctx_v);
  } else {
    blk -= blocks.ctx;
    part = p.part_own; n = (long long)a.B * a.K * a.L * a.Hkv; splits = p.own_splits; heads = a.Hkv; ld = p.down_ld;
    dst = static_cast<T*>(p.down_k); dst_v = static_cast<T*>(p.down_v);
  }
  const long long e = (long long)blk * 256 + threadIdx.x, row = e / (width / 4);
  const int d0 = (int)(e % (width / 4)) * 4;
  if (row >= n) return;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int z = 0; z < splits; ++z) v += *reinterpret_cast<const f32x4*>(part + (z * n + row) * width + d0);
  st4((d0 >= DH ? dst_v : dst) + row / heads * ld + row % heads * DH + d0 % DH, v);
}

// Tile shapes.  Forward and dq: QT 16-row tiles a wave; dkv: KT 16-key tiles a wave and RC rows a chunk.
template <typename T, int DH> constexpr int kKT = sizeof(T) == 2 && DH <= 64 ? 2 : 1;
template <typename T, int DH> constexpr int kRC = sizeof(T) * DH > 128 && sizeof(T) == 4 ? 32 : 64;
template <typename T, int DH> constexpr int kKC = sizeof(T) * DH > 256 ? 32 : 64;

template <typename T, int DH, int QT>
hipError_t launch_fwd_qt(const PrefixArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((long long)a.B * a.Hkv * a.tiles * a.splits));
  // FINE, for a training step over few keys: out is off by its own rounding alone, 1.66e-3 of its norm, at 2 to 20% of the step.
  // Without it, over 16, 64 and 256 keys, out is off by 2.0e-3, 2.1e-3, 2.2e-3, and dq by 2.47e-3, 2.40e-3, 2.43e-3 for 2.36e-3,
  // 2.37e-3, 2.42e-3 (heads of 32): the gradients' gain ends there.  A step of 256 x 550 rows takes 73, 73, 96 us without
  // and 79, 81, 109 with it (heads of 32), 106, 107, 137 and 111, 117, 154 (of 64).  The lengths are on the device, so
  // the capacities decide.
  if (a.page_rows > 0)
    hipLaunchKernelGGL((k_prefix_fwd<T, DH, QT, 4, kKC<T, DH>, true, false>), grid, dim3(256), 0, s, a);
  else if (sizeof(T) == 2 && a.out_rest && a.T + a.L <= 256)
    hipLaunchKernelGGL((k_prefix_fwd<T, DH, QT, 4, kKC<T, DH>, false, sizeof(T) == 2>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((k_prefix_fwd<T, DH, QT, 4, kKC<T, DH>, false, false>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T, int DH>
hipError_t fwd(const PrefixArgs& a, const PrefixPlan& p, hipStream_t s) {
  hipError_t e;
  if constexpr (sizeof(T) * DH <= 256)
    e = p.rows == 128 ? launch_fwd_qt<T, DH, 2>(a, s) : launch_fwd_qt<T, DH, 1>(a, s);
  else
    e = launch_fwd_qt<T, DH, 1>(a, s);
  if (e != hipSuccess || a.splits == 1) return e;
  const long long rows = (long long)a.B * a.K * a.S * a.Hq;
  hipLaunchKernelGGL((k_prefix_join<T, DH>), dim3((unsigned)((rows * (DH / 4) + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T, int DH>
hipError_t grad(PrefixGradArgs p, const PrefixGradPlan& pl, hipStream_t s) {
  PrefixArgs& a = p.f;
  const long long bg = (long long)a.B * a.Hkv;
  a.tiles = pl.tiles;
  a.splits = pl.splits;
  const dim3 gq((unsigned)(bg * a.tiles * a.splits));
  hipLaunchKernelGGL((k_prefix_dq<T, DH, 1, 4, kKC<T, DH>>), gq, dim3(256), 0, s, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  p.ctx_tiles = pl.ctx_tiles;
  p.own_tiles = pl.own_tiles;
  p.ctx_splits = pl.ctx_splits;
  p.own_splits = pl.own_splits;
  if (pl.dkv_blocks > 0) {
    const dim3 gk((unsigned)pl.dkv_blocks);
    hipLaunchKernelGGL((k_prefix_dkv<T, DH, kKT<T, DH>, 4, kRC<T, DH>>), gk, dim3(256), 0, s, p);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (pl.sum_blocks == 0) return hipSuccess;
  const SumBlocks blocks{(unsigned)sum_blocks(pl.dq_bytes, pl.splits), (unsigned)sum_blocks(pl.ctx_bytes, pl.ctx_splits)};
  hipLaunchKernelGGL((k_prefix_sum<T, DH>), dim3((unsigned)pl.sum_blocks), dim3(256), 0, s, p, blocks);
  return hipGetLastError();
}

// Ranges that `items` chunks of 64 are split into, for each of `wgs` tiles: up to two workgroups per compute unit, at
// least three chunks a range (a range costs its partial sums, and all of them a launch).  64 tiles of 24 chunks: one range
// 28.6 us, four 23.0, eight 19.5, sixteen 20.5; 8 tiles of 4 chunks: 7.4 us whole, 8.9 in two.  In fp32 also as many as
// keep a range at 2048 keys or rows, up to 256 of them: one chain of fp32 sums over n of them is off by about 2^-25 sqrt(n / 8)
// of its result, 1.1e-6 at 6400 and, by this, 1.3e-6 at 4194304 keys in 256 ranges.
// narrow (forward, bf16 heads of at most 64, three of whose workgroups a compute unit holds): up to three as long as a
// range keeps eight chunks (heads of 64, 128 tiles of 512 + 16 chunks: 237 us -> 181, of 32 + 16: 33 -> 30; heads of 32,
// 32 tiles of 32 + 32 chunks: two 16.1, three 18.0).
int ranges(long long wgs, long long items, int most, bool f32, bool narrow = false) {
  const long long two = std::min(512 / std::max(1LL, wgs), items / 3);
  const long long three = narrow ? std::min(768 / std::max(1LL, wgs), items / 8) : 0;
  const long long by_size = std::min(std::max(two, three), (long long)most);
  const long long grid = ((1 << 24) - 1) / std::max(1LL, wgs);           // a launch holds 2^24 - 1 workgroups of 256
  return (int)std::max(1LL, std::min({std::max({1LL, by_size, f32 ? (items + 31) / 32 : 1LL}), 256LL, grid}));
}
// 64-key chunks that a tile of `rows` rows meets: the shared ones and those of the lists it touches.
long long chunks_of(const fe_prefix_args& a, long long rows) {
  const long long sg = (long long)a.S * (a.n_heads / a.n_kv_heads);
  return (a.T + 63) / 64 + (std::min<long long>(a.K, (rows - 1) / sg + 2) * a.L + 63) / 64;
}
}  // namespace

PrefixPlan prefix_plan(const fe_prefix_args& a) {
  PrefixPlan p;
  const long long G = a.n_heads / a.n_kv_heads, R = (long long)a.K * a.S * G, bg = (long long)a.B * a.n_kv_heads;
  // 128 rows a workgroup read a chunk's keys from memory and from LDS half as often, for half the waves and, in fp32 at head
  // width 128, more registers than there are.  They pay
  //  - where 64 rows would read every key twice and 128 read it once (4 x 128 rows of 32768 keys: 236 us -> 175);
  //  - with workgroups to spare, unless they leave more rows of the last tile empty (72 x 3168 rows, heads of 128: of 81 keys
  //    65 -> 56 us, of 1500 339 -> 249; 64 x 2048 rows, heads of 64, of 364 keys 35 -> 31; 256 x 550 rows, whose 640 are 11%
  //    more than 576, of 267 keys 28.5 -> 33.4; 32 x 576 rows of 1064 keys 25 -> 29);
  //  - over long contexts with fewer to spare (64 x 1024 rows: of 4096 keys 126 -> 112, of 1088 38.2 -> 39.0).
  const bool fits = a.dtype == FE_BF16 || a.dh <= 64;
  const long long t128 = (R + 127) / 128, t64 = (R + 63) / 64;
  const bool spare = bg * t128 >= (a.T >= 2048 ? 512 : 1024) && 100 * 2 * t128 <= 108 * t64;
  p.rows = fits && ((R > 64 && R <= 128) || spare) ? 128 : 64;
  p.tiles = (int)((R + p.rows - 1) / p.rows);
  p.splits = ranges(bg * p.tiles, chunks_of(a, p.rows), 64, a.dtype == FE_F32, a.dtype == FE_BF16 && a.dh <= 64);
  // Ranges by the requests' lengths: with enough of them for the rounding and long enough for the arithmetic that shares
  // them out (4 requests, lengths from half of T to T, 32 lists, heads of 128: T = 32768 in 16 ranges 133 us -> 115, 8192
  // 51.4 -> 50.0; heads of 64, 16 lists: 56 -> 52, 27.0 -> 29.4; 16 requests of 8192 in 4 ranges 68 -> 72; 8 of 1024 in 8
  // 15.4 -> 18.0).  fp32 keeps equal numbers, for the length of its chains of sums.
  p.by_length = p.splits > 1 && a.dtype == FE_BF16 && a.ctx_len && a.B > 1 && a.B <= 64 &&
                p.splits >= 8 && a.T >= 1024 * p.splits;
  p.own_chunks = (int)((chunks_of(a, p.rows) - (a.T + 63) / 64) / 2);    // lists half full
  const size_t rows = (size_t)a.B * a.K * a.S * a.n_heads;
  p.part_bytes = p.splits > 1 ? p.splits * rows * (a.dh + 2) * sizeof(float) : 0;
  return p;
}

PrefixGradPlan prefix_grad_plan(const fe_prefix_args& a) {
  PrefixGradPlan p;
  const long long G = a.n_heads / a.n_kv_heads, R = (long long)a.K * a.S * G, bg = (long long)a.B * a.n_kv_heads;
  const bool f32 = a.dtype == FE_F32;
  // dq: 64 rows a workgroup (128: 64 x 1024 rows of 1088 keys at head width 64 the same; fp32 training step of 256 x 550
  // rows, heads of 32, 196 us -> 219)
  p.tiles = (int)((R + 63) / 64);
  p.splits = ranges(bg * p.tiles, chunks_of(a, 64), 16, f32);
  // dk, dv: a shared tile meets every row, an own tile those of its lists
  const long long cols = a.dtype == FE_BF16 && a.dh <= 64 ? 128 : 64;
  p.ctx_tiles = (int)((a.T + cols - 1) / cols);
  p.own_tiles = (int)(((long long)a.K * a.L + cols - 1) / cols);
  const long long lists = a.L ? std::min<long long>(a.K, (cols - 1) / a.L + 2) : 0;
  p.ctx_splits = a.T ? ranges(bg * p.ctx_tiles, (R + 63) / 64, 16, f32) : 1;
  p.own_splits = a.L ? ranges(bg * p.own_tiles, (lists * a.S * G + 63) / 64, 16, f32) : 1;
  const size_t rows = (size_t)a.B * a.K * a.S * a.n_heads, row_bytes = 2 * a.dh * sizeof(float);
  p.rows_bytes = rows * sizeof(float4);
  p.dq_bytes = p.splits > 1 ? p.splits * rows * a.dh * sizeof(float) : 0;
  p.ctx_bytes = p.ctx_splits > 1 ? p.ctx_splits * (size_t)a.B * a.T * a.n_kv_heads * row_bytes : 0;
  p.own_bytes = p.own_splits > 1 ? p.own_splits * (size_t)a.B * a.K * a.L * a.n_kv_heads * row_bytes : 0;
  p.dkv_blocks = bg * ((long long)p.ctx_tiles * p.ctx_splits + (long long)p.own_tiles * p.own_splits);
  p.sum_blocks = sum_blocks(p.dq_bytes, p.splits) + sum_blocks(p.ctx_bytes, p.ctx_splits) +
                 sum_blocks(p.own_bytes, p.own_splits);
  return p;
}

hipError_t launch_prefix_fwd(PrefixArgs a, int dh, bool bf16_rows, const PrefixPlan& p, hipStream_t s) {
  a.tiles = p.tiles;
  a.splits = p.splits;
  a.by_length = p.by_length;
  a.own_chunks = p.own_chunks;
  if (bf16_rows) return dh == 32 ? fwd<bf16, 32>(a, p, s) : dh == 64 ? fwd<bf16, 64>(a, p, s) : fwd<bf16, 128>(a, p, s);
  return dh == 32 ? fwd<float, 32>(a, p, s) : dh == 64 ? fwd<float, 64>(a, p, s) : fwd<float, 128>(a, p, s);
}

hipError_t launch_prefix_grad(const PrefixGradArgs& a, int dh, bool bf16_rows, const PrefixGradPlan& p, hipStream_t s) {
  if (bf16_rows) return dh == 32 ? grad<bf16, 32>(a, p, s) : dh == 64 ? grad<bf16, 64>(a, p, s) : grad<bf16, 128>(a, p, s);
  return dh == 32 ? grad<float, 32>(a, p, s) : dh == 64 ? grad<float, 64>(a, p, s) : grad<float, 128>(a, p, s);
}

// Attention of a request's lists over rows held in 4 bits (fe_packed_attention), and the weight that every cached row
// received (fe_packed_weights).
#include <algorithm>
#include <type_traits>

#include "packed.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

FE_DEV f32x16 mma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

// The side of a product that is not held in 4 bits: eight bf16 values, or eight floats in three bf16 parts whose sum they are
// (each truncation takes the next 8 bits of the significand; an infinity is a first part alone).
struct Parts { bf16x8 p[3]; };
FE_DEV Parts parts8(f32x8 v) {
  u32x4 w[3];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    unsigned h[2], m[2], l[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float x = v[2 * i + j];
      h[j] = __float_as_uint(x);
      float rest = x - __uint_as_float(h[j] & 0xffff0000u);
      if (__builtin_isinf(x)) rest = 0.f;
      m[j] = __float_as_uint(rest);
      l[j] = __float_as_uint(rest - __uint_as_float(m[j] & 0xffff0000u));
    }
    w[0][i] = __builtin_amdgcn_perm(h[1], h[0], 0x07060302);
    w[1][i] = __builtin_amdgcn_perm(m[1], m[0], 0x07060302);
    w[2][i] = __builtin_amdgcn_perm(l[1], l[0], 0x07060302);
  }
  return Parts{{__builtin_bit_cast(bf16x8, w[0]), __builtin_bit_cast(bf16x8, w[1]), __builtin_bit_cast(bf16x8, w[2])}};
}
template <typename T> struct Form;
template <> struct Form<bf16> {
  typedef bf16x8 Op;
  typedef bf16x8 V;
  static FE_DEV Op of(V v) { return v; }
  static FE_DEV Op rounded(f32x8 v) { return __builtin_convertvector(v, bf16x8); }
};
template <> struct Form<float> {
  typedef Parts Op;
  typedef f32x8 V;
  static FE_DEV Op of(V v) { return parts8(v); }
  static FE_DEV Op rounded(f32x8 v) { return parts8(v); }
};
// held x other, the held values exact in bf16: one product, or one a part, the smallest first.
FE_DEV f32x16 mma_held(bf16x8 held, bf16x8 x, f32x16 c) { return mma(held, x, c); }
FE_DEV f32x16 mma_held(bf16x8 held, const Parts& x, f32x16 c) {
  return mma(held, x.p[0], mma(held, x.p[1], mma(held, x.p[2], c)));
}
FE_DEV f32x16 mma_held_right(bf16x8 x, bf16x8 held, f32x16 c) { return mma(x, held, c); }
FE_DEV f32x16 mma_held_right(const Parts& x, bf16x8 held, f32x16 c) {
  return mma(x.p[0], held, mma(x.p[1], held, mma(x.p[2], held, c)));
}

template <typename V, typename T> FE_DEV V ldv(const T* p) { return *reinterpret_cast<const V*>(p); }


FE_DEV int q_rows(const PackedArgs& a, int bk) { return a.q_len ? min(max(a.q_len[bk], 0), a.S) : a.S; }
FE_DEV int own_rows(const PackedArgs& a, int bk) { return a.own.cap ? packed_len(a.own, bk) : 0; }
FE_DEV int ctx_rows(const PackedArgs& a, int b) { return a.ctx.cap ? packed_len(a.ctx, b) : 0; }

// Whether one of the first `n` rows of sequence s has a page in the pool.
FE_DEV bool any_key(const PackedCache& x, long long s, int n) {
  for (int j = 0, p = 0; j < n; j += x.page_rows, ++p)
    if ((unsigned)x.table[s * x.cols + p] < (unsigned)x.n_pages) return true;
  return false;
}
// Whether row `at` = (b K + k) S + s, one in use, sees a key at all.  Asked where a sum is 0 alone: of rows without keys, and of
// rows whose scores are all -infinity, which are NaN.
FE_DEV bool any_key(const PackedArgs& a, long long at) {
  const int bk = (int)(at / a.S), s = (int)(at % a.S), b = bk / a.K, n = q_rows(a, bk), m = own_rows(a, bk);
  return any_key(a.ctx, b, ctx_rows(a, b)) || any_key(a.own, bk, a.causal ? min(max(m - n + s + 1, 0), m) : m);
}

// log2(e) |scale|; positive, so that masked scores stay -infinity: with a scale of 0 the queries are 0 in its place.
FE_DEV float score_unit(float scale) { return scale == 0.f ? 1.f : fabsf(scale) * kLog2e; }

// The two halves of a wave hold the same rows.
FE_DEV float halves_max(float v) {
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
FE_DEV float halves_sum(float v) {
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Query row r of (request b, key head g).
struct Row {
  int k, s, h;                           // list, row, query head
  bool live;                             // r < R and s < q_len
  long long at;                          // (b K + k) S + s
  int own;                               // own keys it sees: j < own
};
FE_DEV Row row_of(const PackedArgs& a, int b, int g, int r) {
  Row w;
  const int rr = min(r, a.R - 1), sg = a.S * a.G;
  w.k = quotient(a.by_sg, rr);
  const int rem = rr - w.k * sg;
  w.s = quotient(a.by_g, rem);
  w.h = g * a.G + rem - w.s * a.G;
  const int bk = b * a.K + w.k, n = q_rows(a, bk), m = own_rows(a, bk);
  w.live = r < a.R && w.s < n;
  w.at = (long long)bk * a.S + w.s;
  w.own = !w.live ? 0 : a.causal ? min(max(m - n + w.s + 1, 0), m) : m;
  return w;
}

// Key ranges by length are numbered request after request: request b has `n` of them, from `first` on; B <= 64, lane b finds
// those of request b.  Every request has one; the others of B * splits are shared out in proportion to the chunks of 64 keys,
// `more` beside the shared ones, rounded down, so they may leave a few unused.
struct Ranges { int first, n; };
FE_DEV Ranges ranges_of_lane(const PackedArgs& a, int splits, int more) {
  const int lane = threadIdx.x & 63;
  const int mine = lane < a.B ? (ctx_rows(a, lane) + 63) / 64 + more + 1 : 0;
  int all = mine;
#pragma unroll
  for (int x = 1; x < 64; x *= 2) all += __shfl_xor(all, x);
  const int n = lane < a.B ? 1 + (int)((float)(a.B * (splits - 1)) * (float)mine / (float)all) : 0;
  int end = n;
#pragma unroll
  for (int x = 1; x < 64; x *= 2) {
    const int before = __shfl_up(end, x);
    if (lane >= x) end += before;
  }
  return {end - n, n};
}
// Turns number `range` into request b's range z of `splits`; false: left over.
FE_DEV bool range_of(const PackedArgs& a, int range, int more, int& b, int& z, int& splits) {
  const int lane = threadIdx.x & 63;
  const Ranges mine = ranges_of_lane(a, splits, more);
  b = __popcll(__ballot(lane < a.B && mine.first + mine.n <= range));
  if (b >= a.B) return false;
  z = range - __builtin_amdgcn_readlane(mine.first, b);
  splits = __builtin_amdgcn_readlane(mine.n, b);
  return true;
}

// The packed own rows of lists k0 .. k0 + nb - 1 of request b: off[i] = first packed row of list k0 + i, off[nb] =
// their number; a list without query rows contributes none.  nb <= 128.  Every wave writes the same; a barrier follows.
struct Packing {
  int n[2], end[2];                        // own rows of lists 2 lane and 2 lane + 1; their ends, past the last list out of reach
  FE_DEV void load(const PackedArgs& a, int b, int k0, int nb) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int bk = b * a.K + k0 + min(2 * lane + x, nb - 1);
      const int q = q_rows(a, bk), m = own_rows(a, bk);
      n[x] = 2 * lane + x < nb && q > 0 ? m : 0;
    }
  }
  FE_DEV void store(int nb, int* off) {
    const int lane = threadIdx.x & 63;
    int v = n[0] + n[1];
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      if (m >= nb) break;                  // uniform
      const int x = __shfl_up(v, m);
      if (lane >= m) v += x;
    }
    if (lane == 0) off[0] = 0;
    if (2 * lane < nb) off[2 * lane + 1] = v - n[1];
    if (2 * lane + 1 < nb) off[2 * lane + 2] = v;
    end[0] = 2 * lane < nb ? v - n[1] : 0x7fffffff;
    end[1] = 2 * lane + 1 < nb ? v : 0x7fffffff;
  }
  FE_DEV int list(int x) const {           // that packed row x, the same in all lanes, lies in
    return __popcll(__ballot(end[0] <= x)) + __popcll(__ballot(end[1] <= x));
  }
};

// Share z of `splits` of n things: the first n % splits shares have one more.
FE_DEV int share(int n, int z, int splits) {
  if (splits == 1) return z ? n : 0;
  const int each = n / splits;
  return z * each + min(z, n - each * splits);
}

// A tile of keys or values in LDS as bf16, rows of DH without padding, their units of 8 columns exchanged inside a row so that
// 16 rows at one unit, 4 rows at 4 neighbouring units, and what 16 neighbouring threads write at a time (a unit of each of
// their blocks of 32 columns) all fall on all 64 banks.
template <int DH> struct Tile {
  static FE_DEV int swap(int row) {        // a bijection of the rows that share a unit's banks
    const int r0 = row & 3, r1 = row >> 2 & 3;
    if (DH == 128) return r0 << 2 | (r1 ^ r0);
    if (DH == 64) return ((r0 & 2) << 1) | ((r1 & 2) ^ (r0 & 2)) | (r1 & 1);
    return r1;
  }
  static FE_DEV int at(int row, int unit) { return row * DH + ((unit ^ swap(row)) << 3); }
  // Operand along rows: lane l is row base + l % 32, its elements columns 16 c + 8 (l / 32) + j (base a multiple of 32).
  static FE_DEV int row_lane(int lane) { return at(lane & 31, lane >> 5); }
  static FE_DEV bf16x8 rows(const bf16* X, int base, int c, int row_lane) {
    return ldv<bf16x8>(X + base * DH + (row_lane ^ (c << 4)));
  }
  // Operand along columns: lane l is column 32 n + l % 32, its elements 4 x + j are rows base + 8 x + 4 (l / 32) + j: the
  // order in which a lane holds the scores of a 32-row product.  Every 16 lanes read a 4 x 16 block transposed.
  static FE_DEV int col_lane(int lane) {
    const int row = 4 * (lane >> 5) + (lane >> 2 & 3);
    return at(row, 2 * (lane >> 4 & 1) + (lane >> 1 & 1)) + (lane & 1) * 4;
  }
  static FE_DEV bf16x8 cols(const bf16* X, int base, int n, int col_lane) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4* lds_ptr;
    bf16* p = const_cast<bf16*>(X) + base * DH + (col_lane ^ (n << 5) ^ step(base));
    bf16* q = const_cast<bf16*>(X) + (base + 8) * DH + (col_lane ^ (n << 5) ^ step(base + 8));
    const s16x4 u = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p);
    const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)q);
    return __builtin_shufflevector(__builtin_bit_cast(bf16x4, u), __builtin_bit_cast(bf16x4, v), 0, 1, 2, 3, 4, 5, 6, 7);
  }
  // What a base that is a multiple of 8 changes in the exchange.
  static FE_DEV constexpr int step(int base) { return (base >> 2 & 3) << 3; }
};

FE_DEV int fresh(int x) {                // keeps a lane's number in one register, not one for every xor of it
  asm volatile("" : "+v"(x));
  return x;
}
// The kernel's arguments, to be read again where they are used: what only the own rows need does not take registers from the
// loop over the shared ones.
typedef const __attribute__((address_space(4))) PackedArgs* ArgsAgain;
FE_DEV ArgsAgain args_again() {
  ArgsAgain p = (ArgsAgain)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return p;
}
FE_DEV void order() { asm volatile("" ::: "memory"); }   // LDS operations of one wave stay in order

// ------------------------------------------------------------------------------------------
// Forward.  The rows of a (request, key head) are one matrix of R rows; W waves are WK groups of WR waves with 32
// rows each.  A group takes every WK-th chunk of KC keys (first the shared rows, then the own rows of the lists that the
// tile touches, packed without gaps); a thread loads PER units of UE codes of the keys and of the values, the next
// chunk's in flight behind this one's products, turns them into bf16, which holds them exactly, and puts them into LDS.
// Scores are formed transposed (keys x rows, 32 x 32 x 16 products, at twice the rate of 16 x 16 x 32 ones), so that a lane
// holds 16 keys of one row in the operand layout of the product with the values.  With WK > 1 the groups' sums are joined in LDS
// at the end.
//
// 128 rows a workgroup above 64, so that a key is turned into bf16 once for 128; 64 above 32; up to 32 the groups have a wave
// each, which meet no barrier.  Own rows of short lists are seen by few of a tile's rows: staged by every wave for itself (4
// x 32 lists over 32768 rows, heads of 128: 105 us -> 97; 64 x 50 slates of 11: 34 -> 27).  Two blocks of keys at a time, at one
// or two waves fewer a SIMD (115 -> 108, prompts 281 -> 261).
// Bound: no unit alone.  2 x 2048 rows of 16 heads of 128 over 5120 keys: 225 us, 763 TFLOP/s, with the vector unit busy 42% of
// the time, matrix cores 32%, LDS 33%, waits 30% of the waves' time; leaving out any one of staging, exponentials, either product or
// the loads takes 8 to 15% away.  4 x 32 x 4 rows a key head over 16384 .. 32768: 97 us and the join's 10 (145 MB,
// 52 GFLOP).  64 x 550 rows of 4 heads of 32 over 267 keys: 24.4 us, vector unit 60%, a third of it outside the score loop.
// 5 rows of 181 keys: 7.6 us, a chain of dependent trips to memory.
// ------------------------------------------------------------------------------------------
template <typename T, int DH, int WR, int UE, int W> struct Shape {
  static constexpr int WK = W / WR, GT = 64 * WR, ROWS = 32 * WR, UPR = DH / UE;
  static constexpr int PER = 32 * UPR > GT ? 32 * UPR / GT : 1, KC = GT * PER / UPR;
  static constexpr int NBUF = WR > 1 ? 2 : 1, ND = DH / 16, NB = DH / 32;
  static constexpr int NS = KC >= 64 && sizeof(T) == 2 ? 2 : 1;   // 32-key blocks at a time
};
constexpr int fwd_waves(int bytes, int dh, int wr) {
  return dh == 128 ? (bytes == 4 ? 1 : 2) : dh == 64 ? (bytes == 4 ? 2 : 3) : bytes == 4 ? 3 : 4;
}

template <typename T, int DH, int WR, int UE, int W>
__global__ __launch_bounds__(64 * W, W > 4 ? W / 4 : fwd_waves(sizeof(T), DH, WR)) void k_packed_fwd(PackedArgs a) {
  typedef Shape<T, DH, WR, UE, W> C;
  typedef Form<T> F;
  typedef typename F::Op Op;
  typedef Tile<DH> L;
  constexpr int WK = C::WK, GT = C::GT, ROWS = C::ROWS, UPR = C::UPR, PER = C::PER, KC = C::KC, NBUF = C::NBUF;
  constexpr int ND = C::ND, NB = C::NB, TILE = KC * DH, NS = C::NS;
  constexpr bool FINE = WR == 1 && sizeof(T) == 2;
  static_assert(WR == 1 || (WK * 2 * KC >= 128 && WK * NBUF * 2 * TILE >= 4 * 64 * DH), "own rows by wave fit the tiles");
  static_assert(KC % (32 * NS) == 0 && (WK == 1 || W * 32 * DH * 4 <= WK * NBUF * 2 * TILE * 2), "the join fits the tiles");
  __shared__ __attribute__((aligned(16))) bf16 s_kv[WK][NBUF][2][TILE];
  __shared__ int s_off[ROWS + 1];
  // of a chunk (by its parity in the group): the last one with rows of no page, those rows; the last one with own values
  // of NaN, those units
  __shared__ int s_holes[WK][2], s_hole[WK][2][KC], s_odds[WK][2], s_odd[WK][2][KC * UPR];
  __shared__ int s_wave_hole[4], s_wave_odd[4];         // ... of a wave's own rows
  __shared__ float s_ml[W][32][2];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = wave / WR, wr = wave % WR, gt = tid % GT, half = lane >> 5, c32 = lane & 31;
  int id = xcd_tile(blockIdx.x, gridDim.x);
  const int t = id % a.tiles;
  id /= a.tiles;
  const int g = id % a.Hkv, range = id / a.Hkv;
  int b = range / a.splits, z = range % a.splits, splits = a.splits;
  if (a.by_length && !range_of(a, range, a.own_chunks, b, z, splits)) return;   // uniform
  const int r0 = t * ROWS, r1 = min(r0 + ROWS, a.R);
  const int k0 = quotient(a.by_sg, r0), nb = quotient(a.by_sg, r1 - 1) - k0 + 1;
  // what needs only the sizes to be found is under way first: the lists' lengths, this wave's rows
  Packing packing;
  packing.load(a, b, k0, nb);
  const Row row = row_of(a, b, g, r0 + wr * 32 + c32);
  typename F::V qreg[ND];
  {
    const T* Q = static_cast<const T*>(a.q) + row.at * a.q_ld + row.h * DH + 8 * half;
#pragma unroll
    for (int c = 0; c < ND; ++c) qreg[c] = ldv<typename F::V>(Q + 16 * c);
  }
  const int last_q = q_rows(a, b * a.K + k0 + nb - 1), last_own = own_rows(a, b * a.K + k0 + nb - 1);
  for (int i = tid; i < WK * 2 * KC; i += 64 * W) (&s_hole[0][0][0])[i] = -1;
  for (int i = tid; i < WK * 2 * KC * UPR; i += 64 * W) (&s_odd[0][0][0])[i] = -1;
  if (tid < WK * 2) (&s_holes[0][0])[tid] = (&s_odds[0][0])[tid] = -1;
  if (tid < 4) s_wave_hole[tid] = s_wave_odd[tid] = -1;

  // This group's chunks: numbers q = grp + WK i of the range's share of the shared ones (from cb on) and, after these nc, of
  // the own ones (from ob on).  A thread's units of a chunk: their pages are looked up a chunk before they are loaded.
  const int nctx = ctx_rows(a, b), cctx = (nctx + KC - 1) / KC;
  const int cb = share(cctx, z, splits), nc = share(cctx, z + 1, splits) - cb;
  constexpr int MOST = DH == 128 && PER < 2 ? 2 : PER;   // units of a thread, here or in own rows by wave
  u32x4 kc[MOST], vc[MOST];
  unsigned ks[MOST], vs[MOST];
  int entry[MOST], rest[MOST];             // rest: row inside the page, -1 past the rows
  int page[PER], row_in[PER];              // of the next shared chunk
  int gone = 0, hole = 0;                  // bit p: does not count; as its page is none
  const int jump = a.ctx.cap ? packed_page(a.ctx, WK * KC) : 0, jump_rows = WK * KC - jump * a.ctx.page_rows;
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    const int j = (cb + grp) * KC + (gt + p * GT) / UPR;
    page[p] = a.ctx.cap ? packed_page(a.ctx, j) : 0;
    row_in[p] = j - page[p] * a.ctx.page_rows;
  }
  const int32_t* ctx_table = a.ctx.cap ? a.ctx.table + (long long)b * a.ctx.cols : nullptr;
  auto find_ctx = [&](int q) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      rest[p] = -1;
      if ((cb + q) * KC + (gt + p * GT) / UPR < nctx) {
        rest[p] = row_in[p];
        entry[p] = ctx_table[(unsigned)page[p]];
      }
      page[p] += jump;
      row_in[p] += jump_rows;
      if (row_in[p] >= a.ctx.page_rows) {
        row_in[p] -= a.ctx.page_rows;
        ++page[p];
      }
    }
  };
  // Units of U codes, `threads` apart: a group's share of a chunk, or (own rows by wave) a lane's of a wave's 32 keys.
  auto load_units = [&](const auto& x, auto width, auto count, int first, int threads) __attribute__((always_inline)) {
    constexpr int U = decltype(width)::value, N = decltype(count)::value, ROW = DH / U;
    gone = hole = 0;
    const unsigned all = (unsigned)x.page_rows * ROW;
#pragma unroll
    for (int p = 0; p < N; ++p) {
      const bool none = rest[p] >= 0 && (unsigned)entry[p] >= (unsigned)x.n_pages, skip = rest[p] < 0 || none;
      gone |= skip << p;
      hole |= none << p;
      const unsigned u = (first + p * threads) % ROW, at = (skip ? 0 : rest[p]) * ROW + u;   // what does not count reads row 0 of page 0
      const char* head = x.pages + (unsigned long long)(skip ? 0u : (unsigned)entry[p]) * (unsigned)x.page_ld;
      const unsigned k = (unsigned)g * x.head_bytes + at * (U / 2), s = (unsigned)g * x.head_bytes + all * U + (U == 32 ? at : at >> 1);
      if constexpr (U == 32) {
        kc[p] = ldv<u32x4>(head + k);
        vc[p] = ldv<u32x4>(head + (k + all * (U / 2)));
      } else {
        const uint2 kk = ldv<uint2>(head + k), vv = ldv<uint2>(head + (k + all * (U / 2)));
        kc[p] = u32x4{kk.x, kk.y, 0, 0};
        vc[p] = u32x4{vv.x, vv.y, 0, 0};
      }
      ks[p] = *reinterpret_cast<const unsigned char*>(head + s);
      vs[p] = *reinterpret_cast<const unsigned char*>(head + (s + (U == 32 ? all : all >> 1)));
    }
  };
  constexpr std::integral_constant<int, UE> kUnit{};
  constexpr std::integral_constant<int, PER> kPer{};
  if (grp < nc) {                          // under way while the lists' lengths and packing are found
    find_ctx(grp);
    load_units(a.ctx, kUnit, kPer, gt, GT);
  }

  packing.store(nb, s_off);
  __syncthreads();
  const int lo = s_off[row.k - k0], hi = lo + row.own;   // the packed own rows that the row sees
  // Of the wave, uniform: bounds of what its rows see, and (empty where they belong to several lists) what all of them see.
  // Neither lo nor the live rows' hi falls from row to row.
  const unsigned live = (unsigned)__ballot(row.live);
  const int wlo = __builtin_amdgcn_readlane(lo, 0), alo = __builtin_amdgcn_readlane(lo, 31);
  const int whi = live ? __builtin_amdgcn_readlane(hi, 31 - __builtin_clz(live)) : 0;
  const int ahi = !live ? 0x7fffffff : wlo == alo ? __builtin_amdgcn_readlane(hi, __builtin_ctz(live)) : -1;
  // the tile's packed rows end with what the last list's last live row in it sees
  int nown = s_off[nb - 1];
  {
    const int s = min(quotient(a.by_g, r1 - 1 - (k0 + nb - 1) * a.S * a.G), last_q - 1);
    if (s >= 0) nown += a.causal ? min(max(last_own - last_q + s + 1, 0), last_own) : last_own;
    nown = __builtin_amdgcn_readfirstlane(nown);
  }
  // Own rows of long lists are taken as the shared ones are; of short ones, which few of the tile's rows see, every wave takes
  // those of its rows' lists by itself, after the shared ones.
  const bool by_wave = WR > 1 && 2 * a.S * a.G <= ROWS;
  const int cown = by_wave ? 0 : (nown + KC - 1) / KC, ob = share(cown, z, splits), nq = nc + share(cown, z + 1, splits) - ob;

  if (a.scale <= 0) {                      // uniform
#pragma unroll
    for (int c = 0; c < ND; ++c)           // negative: exact, and the largest score is then the largest product; 0: 0, of infinities NaN
      qreg[c] = a.scale < 0 ? -qreg[c] : qreg[c] - qreg[c];
  }
  Op qf[ND];
#pragma unroll
  for (int c = 0; c < ND; ++c) {
    if (!row.live) qreg[c] = typename F::V{};
    qf[c] = F::of(qreg[c]);
  }
  const float sl2 = score_unit(a.scale), lag = fminf(8.f / sl2, 1e30f);
  float m_run = -INFINITY, l_run = 0.f;    // maximum of q.k; l_run: this lane's keys only, until the end
  f32x16 o[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) o[n] = f32x16{};

  // packed rows x0 + key of the units, below `to`
  auto find_own = [&](int x0, int to, auto width, auto count, int first, int threads) __attribute__((always_inline)) {
    constexpr int U = decltype(width)::value, N = decltype(count)::value, ROW = DH / U;
    const ArgsAgain A = args_again();
    const unsigned rows = A->own.page_rows;
    const int32_t* table = A->own.table + ((long long)b * A->K + k0) * A->own.cols;
    const int list = packing.list(x0);
#pragma unroll
    for (int p = 0; p < N; ++p) {
      const int x = x0 + (first + p * threads) / ROW;
      rest[p] = -1;
      if (x < to) {
        int i = list;
        while (s_off[i + 1] <= x) ++i;
        const int j = x - s_off[i], pg = (int)((unsigned long long)(unsigned)j * A->own.by_rows.magic >> A->own.by_rows.shift);
        rest[p] = j - pg * rows;
        entry[p] = table[(long long)i * A->own.cols + pg];
      }
    }
  };
  auto find = [&](int q) __attribute__((always_inline)) {
    if (q < nc) find_ctx(q);               // uniform
    else if (q < nq) find_own((ob + q - nc) * KC, nown, kUnit, kPer, gt, GT);
  };
  auto load = [&](int q) __attribute__((always_inline)) {
    if (q < nc) load_units(a.ctx, kUnit, kPer, gt, GT);          // uniform
    else if (q < nq) load_units(args_again()->own, kUnit, kPer, gt, GT);
  };
  // Puts the units into tiles K and V; marks rows of no page with `tag` in holes[key] and any_hole, and (own rows) values of
  // NaN in odds[unit] and any_odd: NaN would reach the rows of other lists, as 0 times NaN, so they get zeros and the rows that
  // see it get it at the end.
  auto stage = [&](bf16* K, bf16* V, auto width, auto count, int first, int threads, bool own, int tag, int* holes, int* any_hole,
                   int* odds, int* any_odd) __attribute__((always_inline)) {
    constexpr int U = decltype(width)::value, N = decltype(count)::value, ROW = DH / U;
#pragma unroll
    for (int p = 0; p < N; ++p) {
      const int key = (first + p * threads) / ROW, u = (first + p * threads) % ROW;
      float ku = unit_of(ks[p]), vu = unit_of(vs[p]);
      if (gone >> p & 1) {
        kc[p] = vc[p] = u32x4{0, 0, 0, 0};
        ku = vu = 1.f;
        if (hole >> p & 1) holes[key] = *any_hole = tag;
      } else if (own && vs[p] == 255) {
        vc[p] = u32x4{0, 0, 0, 0};
        vu = 1.f;
        odds[key * ROW + u] = *any_odd = tag;
      }
      const int base = L::at(key, u * (U / 8));
#pragma unroll
      for (int i = 0; i < U / 8; ++i) {
        *reinterpret_cast<bf16x8*>(K + (base ^ i << 3)) = values8(kc[p][i], ku);
        *reinterpret_cast<bf16x8*>(V + (base ^ i << 3)) = values8(vc[p][i], vu);
      }
    }
  };

  int rl = L::row_lane(lane), cl = L::col_lane(lane);
  // N blocks of 32 keys from row kb of the tiles on, key x0 the first of them, whose chains of products overlap; element i of a lane
  // is key 8 (i / 4) + 4 half + i % 4 of a block.  The lane's row sees keys [from0, to0), all rows [all_from, all_to).
  auto blocks = [&](auto number, auto width, const bf16* K, const bf16* V, int kb, int x0, bool own, int from0, int to0, int all_from,
                    int all_to, int tag, const int* holes, int any_hole, const int* odds, int any_odd) __attribute__((always_inline)) {
    constexpr int N = decltype(number)::value, U = decltype(width)::value, ROW = DH / U;
    f32x16 s[N];
#pragma unroll
    for (int u = 0; u < N; ++u) s[u] = f32x16{};
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int u = 0; u < N; ++u) s[u] = mma_held(L::rows(K, kb + 32 * u, d, rl), qf[d], s[u]);
    __builtin_amdgcn_s_setprio(0);
    if (x0 < all_from || x0 + 32 * N > all_to) {      // uniform
      const int from = from0 - x0 - 4 * half, to = to0 - x0 - 4 * half;
#pragma unroll
      for (int u = 0; u < N; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (32 * u + 8 * (i >> 2) + (i & 3) < from || 32 * u + 8 * (i >> 2) + (i & 3) >= to) s[u][i] = -INFINITY;
    }
    if (__builtin_amdgcn_readfirstlane(any_hole) == tag) {  // uniform
#pragma unroll
      for (int u = 0; u < N; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (holes[kb + 32 * u + 8 * (i >> 2) + 4 * half + (i & 3)] == tag) s[u][i] = -INFINITY;
    }
    float mx = m_run;
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int i = 0; i < 16; i += 2) mx = fmaxf(fmaxf(mx, s[u][i]), s[u][i + 1]);
    // The reference follows the running maximum once a score is 8 / log2(e) above it: a probability is at most 2^8 then.
    // Whether a row's moves depends on that row alone; the others are multiplied by 1.
    if (__any(mx > m_run + lag)) {
      const float top = halves_max(mx), next = top > m_run + lag ? top : m_run;
      const float alpha = next == m_run ? 1.f : __builtin_amdgcn_exp2f((m_run - next) * sl2);
      m_run = next;
      l_run *= alpha;
#pragma unroll
      for (int n = 0; n < NB; ++n) o[n] *= alpha;
    }
    const float ref = m_run == -INFINITY ? 0.f : m_run * sl2;   // a row without keys so far: exp2(-inf) = 0
#pragma unroll
    for (int u = 0; u < N; ++u) {
      float sum[4];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[u][i] = __builtin_amdgcn_exp2f(fmaf(s[u][i], sl2, -ref));
        sum[i & 3] = i < 4 ? s[u][i] : sum[i & 3] + s[u][i];
      }
      l_run += (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        f32x8 w;
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = s[u][8 * m + j];
        const Op p = F::rounded(w);
        // bf16: one rounding of p, of about the size of out's own (out off by 2.3e-3 of its norm, 1.7e-3 without it).  Up to 32 rows
        // what it cut is a second product, since these calls wait for memory (4 x 16 rows a key head: 15.7 us either way).  For more
        // rows it would take 32 lists over 32768 rows from 106 to 119 us, slates from 24.8 to 29.5 and prompts from 224 to 283.
        Op rest;
        if constexpr (FINE) {
#pragma unroll
          for (int j = 0; j < 8; ++j) w[j] -= (float)p[j];
          rest = F::rounded(w);
        }
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          const bf16x8 v = L::cols(V, kb + 32 * u + 16 * m, n, cl);
          if constexpr (FINE) o[n] = mma_held(v, rest, o[n]);
          o[n] = mma_held(v, p, o[n]);
        }
      }
    }
    if (own && __builtin_amdgcn_readfirstlane(any_odd) == tag) {
      // uniform: the columns of a NaN block, in the rows that see its key
#pragma unroll 1
      for (int e = 0; e < 32 * N * ROW; ++e) {
        const int x = x0 + e / ROW, n = e % ROW * U / 32;
        if (__builtin_amdgcn_readfirstlane(odds[kb * ROW + e]) != tag) continue;
        const float nan = x < lo || x >= hi ? 0.f : NAN;
#pragma unroll
        for (int y = 0; y < NB; ++y) o[y] += y == n ? nan : 0.f;
      }
    }
  };
  const bool idle = r0 + wr * 32 >= a.R;
  if (grp >= nc) {                         // uniform: no shared chunk was under way
    find(grp);
    load(grp);
  }
  find(grp + WK);
  const int trips = (nq + WK - 1) / WK;
  for (int it = 0; it < trips; ++it) {
    const int q = grp + it * WK, par = it & 1;
    bf16 *K = s_kv[grp][it % NBUF][0], *V = s_kv[grp][it % NBUF][1];
    const bool own = q >= nc;
    if (q < nq) stage(K, V, kUnit, kPer, gt, GT, own, q, s_hole[grp][par], &s_holes[grp][par], s_odd[grp][par], &s_odds[grp][par]);
    load(q + WK);
    find(q + 2 * WK);
    if constexpr (WR > 1) lds_barrier();   // also the end of every wave's reads of the buffer written next
    else order();
    if (q >= nq || idle) continue;         // uniform
    rl = fresh(rl);
    cl = fresh(cl);
    const int x1 = own ? (ob + q - nc) * KC : (cb + q) * KC;   // first key: packed own rows, or shared ones
    const int first = own ? wlo : 0, end = own ? whi : nctx;
    const int any_hole = s_holes[grp][par], any_odd = s_odds[grp][par];
#pragma unroll 1
    for (int kb = 0; kb < KC; kb += 32 * NS) {
      const int x0 = x1 + kb;
      if (x0 >= end) break;                // uniform
      if (x0 + 32 * NS <= first) continue;
      blocks(std::integral_constant<int, NS>{}, kUnit, K, V, kb, x0, own, own ? lo : 0, own ? hi : nctx, own ? alo : 0,
             own ? ahi : nctx, q, s_hole[grp][par], any_hole, s_odd[grp][par], any_odd);
    }
    if constexpr (WR == 1) order();        // this chunk's reads before the next one's writes
  }
  if (WR > 1 && by_wave) {                 // uniform
    // the wave's packed rows [wlo, whi) in chunks of 32, in tiles of its own; rows of the tile's other waves do not matter here
    constexpr std::integral_constant<int, DH == 32 ? 16 : 32> width{};
    constexpr std::integral_constant<int, DH == 128 ? 2 : 1> count{};
    const int chunks = max(whi - wlo + 31, 0) / 32, c1 = share(chunks, z + 1, splits);
    int c = share(chunks, z, splits) + grp;
    bf16 *K = &s_kv[0][0][0][0] + wave * 64 * DH, *V = K + 32 * DH;
    int *holes = &s_hole[0][0][0] + wave * 32, *odds = &s_odd[0][0][0] + wave * (32 * (DH / width.value));
    int *any_hole = &s_wave_hole[wave], *any_odd = &s_wave_odd[wave];
    if (c < c1) find_own(wlo + 32 * c, whi, width, count, lane, 64);
    if (c < c1) load_units(args_again()->own, width, count, lane, 64);
    if (c + WK < c1) find_own(wlo + 32 * (c + WK), whi, width, count, lane, 64);
    __syncthreads();                       // the shared chunks are no longer read, nor their marks
    for (int i = lane; i < 32 * (1 + DH / width.value); i += 64) (i < 32 ? holes[i] : odds[i - 32]) = -1;
    order();
    for (; c < c1; c += WK) {
      stage(K, V, width, count, lane, 64, true, c, holes, any_hole, odds, any_odd);
      if (c + WK < c1) load_units(args_again()->own, width, count, lane, 64);
      if (c + 2 * WK < c1) find_own(wlo + 32 * (c + 2 * WK), whi, width, count, lane, 64);
      order();
      rl = fresh(rl);
      cl = fresh(cl);
      blocks(std::integral_constant<int, 1>{}, width, K, V, 0, wlo + 32 * c, true, lo, hi, alo, ahi, c, holes, *any_hole, odds, *any_odd);
      order();
    }
  }

  const float l_all = halves_sum(l_run);
  const bool in = r0 + wr * 32 + c32 < a.R;
  const long long ro = row.at * a.Hq + row.h;
  // No key; a NaN score leaves a NaN sum, and 0 for all keys, where each is -infinity, NaN as 0 times 1 / 0.
  auto none_of = [&](float l) __attribute__((always_inline)) {
    if (!row.live || l != 0.f) return !row.live;
    const PackedArgs& again = *(const PackedArgs*)args_again();
    return again.splits == 1 && !any_key(again, row.at);
  };
  // Slice i of a lane: columns 8 i + 4 half .. + 3, v its sums against reference m (in units of 1 / sl2).
  auto store = [&](int i, f32x4 v, float m, float l, bool none) __attribute__((always_inline)) {
    const float m2 = m * sl2;
    if (a.splits > 1) {
      const long long at = ro + (long long)(range - b) * a.K * a.S * a.Hq;   // [range][row of the request]
      *reinterpret_cast<f32x4*>(a.part_o + at * DH + 8 * i + 4 * half) = v;
      if (i == 0 && half == 0) *reinterpret_cast<float2*>(a.part_ml + at * 2) = float2{m2, l};
      return;
    }
    const float inv = none ? 0.f : 1.f / l;
    typedef T T4 __attribute__((ext_vector_type(4)));
    T4 w;
#pragma unroll
    for (int x = 0; x < 4; ++x) w[x] = from_f32<T>(none ? 0.f : v[x] * inv);
    *reinterpret_cast<T4*>(static_cast<T*>(a.out) + row.at * a.out_ld + row.h * DH + 8 * i + 4 * half) = w;
    if (a.lse && i == 0 && half == 0) a.lse[ro] = none ? -INFINITY : l == 0.f ? NAN : (m2 + log2f(l)) * kLn2;
  };
  auto slice = [&](int i) __attribute__((always_inline)) {
    const f32x16 v = o[i >> 2];
    return f32x4{v[4 * (i & 3)], v[4 * (i & 3) + 1], v[4 * (i & 3) + 2], v[4 * (i & 3) + 3]};
  };
  if constexpr (WK == 1) {
    if (!in) return;
    const bool none = none_of(l_all);
#pragma unroll
    for (int i = 0; i < 4 * NB; ++i) store(i, slice(i), m_run, l_all, none);
  } else {                                 // joins the groups in their order, every group some of the slices
    __syncthreads();
    float* X = reinterpret_cast<float*>(s_kv);
#pragma unroll
    for (int i = 0; i < 4 * NB; ++i) *reinterpret_cast<f32x4*>(X + ((wave * 4 * NB + i) * 64 + lane) * 4) = slice(i);
    if (half == 0) {
      s_ml[wave][c32][0] = m_run;
      s_ml[wave][c32][1] = l_all;
    }
    __syncthreads();
    if (!in) return;
    float top = -INFINITY, l = 0.f, f[WK];
#pragma unroll
    for (int w = 0; w < WK; ++w) top = fmaxf(top, s_ml[w * WR + wr][c32][0]);
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int w = 0; w < WK; ++w) {
      f[w] = __builtin_amdgcn_exp2f((s_ml[w * WR + wr][c32][0] - ref) * sl2);
      l = fmaf(s_ml[w * WR + wr][c32][1], f[w], l);
    }
    const bool none = none_of(l);
#pragma unroll 1
    for (int i = grp; i < 4 * NB; i += WK) {
      f32x4 v{};
#pragma unroll
      for (int w = 0; w < WK; ++w) {
        const f32x4 x = ldv<f32x4>(X + (((w * WR + wr) * 4 * NB + i) * 64 + lane) * 4);
#pragma unroll
        for (int y = 0; y < 4; ++y) v[y] = fmaf(x[y], f[w], v[y]);
      }
      store(i, v, top, l, none);
    }
  }
}

// Joins the key ranges of a row in ascending order: DH / 4 threads a row.
// Bound: the partial sums (4096 rows of 128 in about 16 ranges, 34 MB: 10 us); one trip for a few (4 us).
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_packed_join(PackedArgs a) {
  const long long per = (long long)a.K * a.S * a.Hq, rows = a.B * per;
  const long long e = (long long)blockIdx.x * 256 + threadIdx.x, ro = e / (DH / 4);
  const int d0 = (int)(e % (DH / 4)) * 4;
  const int b = (int)(min(ro, rows - 1) / per);
  int first = b * a.splits, splits = a.splits;
  if (a.by_length) {                       // uniform
    const Ranges mine = ranges_of_lane(a, a.splits, a.own_chunks);
    first = __shfl(mine.first, b);
    splits = __shfl(mine.n, b);
  }
  if (ro >= rows) return;
  const long long at0 = (first - b) * per + ro;
  // ranges in batches, their loads together
  constexpr int N = 8;
  float top = -INFINITY, l = 0.f;
  f32x4 o{};
  for (int z0 = 0; z0 < splits; z0 += N) {
    float2 ml[N];
    f32x4 v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const long long at = min(z0 + i, splits - 1) * per + at0;
      ml[i] = ldv<float2>(a.part_ml + at * 2);
      v[i] = ldv<f32x4>(a.part_o + at * DH + d0);
    }
    float next = top;
#pragma unroll
    for (int i = 0; i < N; ++i) next = fmaxf(next, ml[i].x);
    const float ref = next == -INFINITY ? 0.f : next;
    float f = __builtin_amdgcn_exp2f(top - ref);
    l *= f;
    o *= f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (z0 + i >= splits) break;         // uniform in a request
      f = __builtin_amdgcn_exp2f(ml[i].x - ref);
      l = fmaf(ml[i].y, f, l);
#pragma unroll
      for (int x = 0; x < 4; ++x) o[x] = fmaf(v[i][x], f, o[x]);
    }
    top = next;
  }
  const long long at = ro / a.Hq;
  const int h = (int)(ro % a.Hq), bk = (int)(at / a.S), s = (int)(at % a.S);
  const bool none = s >= q_rows(a, bk) || (l == 0.f && !any_key(a, at));
  const float inv = none ? 0.f : 1.f / l;
  typedef T T4 __attribute__((ext_vector_type(4)));
  T4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = from_f32<T>(none ? 0.f : o[i] * inv);
  *reinterpret_cast<T4*>(static_cast<T*>(a.out) + at * a.out_ld + h * DH + d0) = v;
  if (a.lse && d0 == 0) a.lse[ro] = none ? -INFINITY : l == 0.f ? NAN : (top + log2f(l)) * kLn2;
}

// ------------------------------------------------------------------------------------------
// Weights.  A workgroup takes a range of a sequence's keys of one head, and a range of the query rows that see them: every
// list's for shared keys, the list's for own keys.  The rows lie in LDS, as many as fit; each wave walks tiles of 32 keys
// without meeting the others, its operands made in registers from the codes, whose loads run a tile ahead and their pages two.
// Which column a summed element is does not matter: lane l has the half l / 32 of its key's columns.  A lane then holds 16
// rows' scores of its key, and their exponentials are added up in it.
//
// Operands of 32 keys a wave and four waves a SIMD: two operands, half the reads of LDS, leave room for two waves (32 lists
// over 32768 rows, heads of 128: 73 us and 54).  Key ranges by the requests' lengths: 54 -> 48; 1024 workgroups: 512
// 59 us, 768 50, 1024 51, 2048 57.
// Bound: the vector unit, 63% (a product-sum, an exponential and a sum a score; the codes' conversion): 45 us, 575 TFLOP/s,
// with three registers spilled while the rows are put into LDS.  8 x 16 lists over 1024: 7.7 us, three dependent trips to memory.
// ------------------------------------------------------------------------------------------
template <typename T, int DH> struct Weigh {
  typedef Form<T> F;
  typedef Tile<DH> L;
  static constexpr int ND = DH / 16, PARTS = sizeof(T) == 4 ? 3 : 1;
  static constexpr int ROWS = (sizeof(T) == 4 ? 8192 : 16384) / DH;    // rows in LDS at a time
  struct Lds {
    __attribute__((aligned(16))) bf16 q[PARTS][ROWS * DH];
    __attribute__((aligned(16))) float lse[ROWS];
    __attribute__((aligned(16))) int seen[ROWS];                       // own keys that the row sees
    int any;
  };

  template <bool OWN> static FE_DEV void run(const PackedArgs& a, int id, Lds& S) {
    constexpr int WORDS = DH / 16, SCALES = DH == 128 ? 2 : 1;         // of a lane: half a key's codes, and their blocks' scales
    const PackedCache& x = OWN ? a.own : a.ctx;
    const int key_splits = OWN ? a.own_keys : a.ctx_keys, row_splits = OWN ? a.own_splits : a.ctx_splits;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
    const int z = id % row_splits;
    id /= row_splits;
    const int g = id % a.Hkv;
    id /= a.Hkv;
    int sq = id / key_splits, zk = id % key_splits, ranges = key_splits;
    if (!OWN && a.keys_by_length && !range_of(a, id, 0, sq, zk, ranges)) return;   // uniform over the workgroup
    const int b = OWN ? sq / a.K : sq;
    const int n = packed_len(x, sq), tiles = (n + 31) / 32;
    const int tb = share(tiles, zk, ranges), te = share(tiles, zk + 1, ranges);
    if (tb == te) return;                  // uniform over the workgroup
    const int nq = OWN ? q_rows(a, sq) : 0, rows = OWN ? nq * a.G : a.R, first = OWN ? (sq - b * a.K) * a.S * a.G : 0;
    const int rb = share(rows, z, row_splits), re = share(rows, z + 1, row_splits);

    int page, row;                         // of the tile after the next: row -1 past the length
    unsigned code[WORDS], scale[SCALES];
    bool counts;                           // of the tile whose codes are under way
    const int32_t* table = x.table + (long long)sq * x.cols;
    auto find = [&](int t) __attribute__((always_inline)) {
      const int j = t * 32 + (lane & 31);
      row = -1;
      if (t < te && j < n) {
        const int p = packed_page(x, j);
        row = j - p * x.page_rows;
        page = table[(unsigned)p];
      }
    };
    auto load = [&]() __attribute__((always_inline)) {
      counts = row >= 0 && (unsigned)page < (unsigned)x.n_pages;
      const unsigned r = counts ? row : 0;                             // what does not count reads row 0 of page 0
      const char* head = x.pages + (unsigned long long)(counts ? (unsigned)page : 0u) * (unsigned)x.page_ld;
      const unsigned at = (unsigned)g * x.head_bytes;
      const unsigned* w = reinterpret_cast<const unsigned*>(head + (at + r * (DH / 2) + half * (DH / 4)));
      const unsigned char* s = reinterpret_cast<const unsigned char*>(head + (at + (unsigned)x.page_rows * DH + r * (DH / 32)));
#pragma unroll
      for (int i = 0; i < WORDS; ++i) code[i] = w[i];
#pragma unroll
      for (int i = 0; i < SCALES; ++i) scale[i] = s[DH == 32 ? 0 : half * SCALES + i];
    };
    const int t0 = tb + wave;
    find(t0);

    const float sl2 = a.scale * kLog2e;
    const int from = L::at(lane & 31, half * (DH / 16));
    const float* w_in = OWN ? a.own_w : a.ctx_w;
    float* out = OWN ? a.own_w_out : a.ctx_w_out;
    if (row_splits > 1) out = (OWN ? a.part_own : a.part_ctx) + z * ((long long)(OWN ? a.B * a.K : a.B) * a.Hkv) * x.cap;
    const long long base = ((long long)sq * a.Hkv + g) * x.cap;
    // at least one trip, so that every key gets its entry
    for (int rc = rb; rc == rb || rc < re; rc += ROWS) {
      const int here = min(ROWS, re - rc);               // rows of this trip, 0 where there are none
      if (rc > rb) {
        find(t0);
        __syncthreads();                   // the rows before are no longer read
      }
      // the rows' loads two units of a thread at a time, the first ones' and the keys' together
      constexpr int BATCH = 2;
      const int units = (here + 31) / 32 * 32 * (DH / 8);
      typename F::V v[BATCH];
      float lse[BATCH];
      int sees[BATCH];
      auto rows_load = [&](int u0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
          const int u = u0 + 256 * i, r = u / (DH / 8);
          if (u >= units) break;
          const Row q = row_of(a, b, g, first + rc + min(r, here - 1));
          v[i] = ldv<typename F::V>(static_cast<const T*>(a.q) + q.at * a.q_ld + q.h * DH + u % (DH / 8) * 8);
          lse[i] = a.lse[b * a.lse_b + (q.k * a.lse_k + q.s * a.lse_s + q.h * a.lse_h)];
          sees[i] = r < here && q.live ? (a.causal ? n - nq + q.s + 1 : n) : -0x7fffffff;
        }
      };
      auto rows_store = [&](int u0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
          const int u = u0 + 256 * i, r = u / (DH / 8), at = L::at(r, u % (DH / 8));
          if (u >= units) break;
          const bool live = sees[i] != -0x7fffffff && lse[i] != -INFINITY;
          if (!live) v[i] = typename F::V{};
          if constexpr (PARTS == 1) {
            *reinterpret_cast<bf16x8*>(S.q[0] + at) = v[i];
          } else {
            const Parts w = parts8(v[i]);
#pragma unroll
            for (int x = 0; x < 3; ++x) *reinterpret_cast<bf16x8*>(S.q[x] + at) = w.p[x];
          }
          if (u % (DH / 8) == 0) {
            S.lse[r] = live ? lse[i] * kLog2e : INFINITY;
            if (OWN) S.seen[r] = live ? sees[i] : 0;
            if (live) S.any = 1;
          }
        }
      };
      rows_load(tid);
      load();
      find(t0 + 4);
      if (tid == 0) S.any = 0;
      __syncthreads();
      for (int u = tid; u < units; u += 256 * BATCH) {
        if (u != tid) rows_load(u);
        rows_store(u);
      }
      __syncthreads();
      const bool any = S.any;              // a row that counts: those that do not may have met NaN
      for (int t = t0; t < te; t += 4) {
        bf16x8 k[ND];
        const bool got = counts;
#pragma unroll
        for (int c = 0; c < ND; ++c) k[c] = values8(code[c], unit_of(scale[c * SCALES / ND]));
        if (t + 4 < te) {                  // uniform
          load();
          find(t + 8);
        }
        float sum = 0.f;
        const int j = t * 32 + (lane & 31);
#pragma unroll 1
        for (int r = 0; r < here; r += 32) {
          f32x16 s{};
#pragma unroll
          for (int c = 0; c < ND; ++c) {
            const int at = r * DH + (from ^ c << 3);
            typename F::Op q;
            if constexpr (PARTS == 1) q = ldv<bf16x8>(S.q[0] + at);
            else q = Parts{{ldv<bf16x8>(S.q[0] + at), ldv<bf16x8>(S.q[1] + at), ldv<bf16x8>(S.q[2] + at)}};
            s = mma_held_right(q, k[c], s);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {    // rows 8 e + 4 half + 0 .. 3
            if (r + 8 * e >= here) break;  // uniform
            const f32x4 ls = ldv<f32x4>(S.lse + r + 8 * e + 4 * half);
            int4 seen;
            if (OWN) seen = ldv<int4>(S.seen + r + 8 * e + 4 * half);
            float p[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(s[4 * e + i], sl2, -ls[i]));
            if (OWN) {
              p[0] = j < seen.x ? p[0] : 0.f;
              p[1] = j < seen.y ? p[1] : 0.f;
              p[2] = j < seen.z ? p[2] : 0.f;
              p[3] = j < seen.w ? p[3] : 0.f;
            }
            sum += (p[0] + p[1]) + (p[2] + p[3]);
          }
        }
        const float total = halves_sum(sum), add = got && any ? total : 0.f;
        if (j >= n || half) continue;
        const float had = rc > rb ? out[base + j] : row_splits > 1 ? 0.f : w_in[base + j];
        out[base + j] = had + add;
      }
    }
  }
};

template <typename T, int DH>
__global__ __launch_bounds__(256, sizeof(T) * DH > 256 ? 2 : 4) void k_packed_weigh(PackedArgs a) {
  typedef Weigh<T, DH> W;
  __shared__ typename W::Lds S;
  const int id = blockIdx.x, n_ctx = a.ctx_w ? a.B * a.Hkv * a.ctx_splits * a.ctx_keys : 0;
  if (id < n_ctx) W::template run<false>(a, xcd_tile(id, n_ctx), S);   // uniform
  else W::template run<true>(a, id - n_ctx, S);
}

// Adds the row ranges of every key in ascending order.  Bound: the partial sums; launch latency where they are few.
__global__ __launch_bounds__(256) void k_packed_weigh_sum(PackedCache x, int Hkv, int splits, long long keys, const float* part,
                                                          const float* w, float* out) {
  const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
  if (at >= keys) return;
  const int s = (int)(at / x.cap / Hkv);
  if (at % x.cap >= packed_len(x, s)) return;
  float v = 0.f;
  for (int z = 0; z < splits; ++z) v += part[z * keys + at];
  out[at] = w[at] + v;
}

template <typename T, int DH>
hipError_t fwd(const PackedArgs& a, const PackedPlan& p, hipStream_t s) {
  // waves of the wide form, which heads of 128 in fp32 do not have
  constexpr int UE = DH == 128 ? 32 : 16, U1 = DH == 32 ? 16 : 32, W1 = sizeof(T) == 4 ? (DH == 128 ? 4 : 8) : DH == 128 ? 8 : 16;
  const dim3 grid((unsigned)((long long)a.B * a.Hkv * a.splits * a.tiles));
  if (p.waves == 1 && p.wide) hipLaunchKernelGGL((k_packed_fwd<T, DH, 1, U1, W1>), grid, dim3(64 * W1), 0, s, a);
  else if (p.waves == 1) hipLaunchKernelGGL((k_packed_fwd<T, DH, 1, U1, 4>), grid, dim3(256), 0, s, a);
  else if (p.waves == 2) hipLaunchKernelGGL((k_packed_fwd<T, DH, 2, UE, 4>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_packed_fwd<T, DH, 4, UE, 4>), grid, dim3(256), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  const long long n = (long long)a.B * a.K * a.S * a.Hq * (DH / 4);
  hipLaunchKernelGGL((k_packed_join<T, DH>), dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T, int DH>
hipError_t weigh(const PackedArgs& a, hipStream_t s) {
  const long long bg = (long long)a.B * a.Hkv;
  const long long blocks = (a.ctx_w ? bg * a.ctx_splits * a.ctx_keys : 0) + (a.own_w ? bg * a.K * a.own_splits * a.own_keys : 0);
  if (blocks > 0) hipLaunchKernelGGL((k_packed_weigh<T, DH>), dim3((unsigned)blocks), dim3(256), 0, s, a);
  hipError_t e = hipGetLastError();
  auto sum = [&](const PackedCache& x, long long n, int splits, const float* part, const float* w, float* out) {
    if (e != hipSuccess || splits <= 1) return;
    const long long keys = n * a.Hkv * x.cap;
    hipLaunchKernelGGL(k_packed_weigh_sum, dim3((unsigned)((keys + 255) / 256)), dim3(256), 0, s, x, a.Hkv, splits, keys, part, w, out);
    e = hipGetLastError();
  };
  if (a.ctx_w) sum(a.ctx, a.B, a.ctx_splits, a.part_ctx, a.ctx_w, a.ctx_w_out);
  if (a.own_w) sum(a.own, (long long)a.B * a.K, a.own_splits, a.part_own, a.own_w, a.own_w_out);
  return e;
}

}  // namespace

PackedPlan packed_plan(const fe_packed_args& a) {
  PackedPlan p;
  const long long G = a.n_heads / a.n_kv_heads, R = (long long)a.K * a.S * G, bg = (long long)a.B * a.n_kv_heads;
  p.waves = R <= 32 ? 1 : R <= 64 ? 2 : 4;
  const long long rows = 32 * p.waves, sg = (long long)a.S * G;
  p.tiles = (int)((R + rows - 1) / rows);
  const long long T = a.ctx.N > 0 ? (long long)a.ctx.cols * a.ctx.page_rows : 0;
  const long long L = a.own.N > 0 ? (long long)a.own.cols * a.own.page_rows : 0;
  const long long own = std::min<long long>(a.K, (rows - 1) / sg + 2) * L, wgs = bg * p.tiles;
  const long long items = (T + 63) / 64 + (own + 63) / 64;
  // Few rows and few workgroups: more waves share a workgroup's keys and join in LDS (fp32 at head width 128 has no registers
  // for it).  One wave of rows, heads of 64: 8 x 5 of 8192 keys 22.3 us -> 17.5; 256 x 4 of 2048 24.1 -> 18.3; heads of 128, 8 x 32
  // of 32768 43.6 -> 32.7.
  p.wide = p.waves == 1 && wgs < 512 && (a.dtype == FE_BF16 || a.dh < 128);
  // Ranges of keys until there are two workgroups a compute unit (wide: one), each of 4 chunks of 64 keys at least (wide: 16;
  // fp32: 2).  32 x 128 rows of 32768 keys, 256 / 512 / 768 / 1024 workgroups: 162, 107, 137, 123 us; 64 x 16 rows of 1024 in 8
  // and 16 chunks 16.1, 15.7; fp32, 6 x 399 rows of 777 in 2 and 4 chunks 18.1, 20.9.
  long long want = ((p.wide ? 256 : 512) + wgs - 1) / wgs;
  want = std::min(want, std::max(1LL, items / (p.wide ? 16 : a.dtype == FE_F32 ? 2 : 4)));
  // fp32 sums over at most 2048 keys, up to 524288 of them; above, over a 256th (more on grids past their limit)
  if (a.dtype == FE_F32) want = std::max(want, (items + 31) / 32);
  const long long grid = ((1 << 24) - 1) / std::max(1LL, wgs);
  p.splits = (int)std::max(1LL, std::min({want, 256LL, grid}));
  p.by_length = a.dtype == FE_BF16 && p.splits >= 8 && a.B > 1 && a.B <= 64 && T >= 1024 * p.splits;
  p.own_chunks = (int)((own + 63) / 64 / 2);                    // lists half full
  const size_t out_rows = (size_t)a.B * a.K * a.S * a.n_heads;
  p.part_bytes = p.splits > 1 ? p.splits * out_rows * (a.dh + 2) * sizeof(float) : 0;
  return p;
}

PackedWeighPlan packed_weigh_plan(const fe_packed_args& a) {
  PackedWeighPlan p{};
  const long long G = a.n_heads / a.n_kv_heads, R = (long long)a.K * a.S * G, sg = (long long)a.S * G;
  const long long T = a.ctx.N > 0 && a.ctx_w ? (long long)a.ctx.cols * a.ctx.page_rows : 0;
  const long long L = a.own.N > 0 && a.own_w ? (long long)a.own.cols * a.own.page_rows : 0;
  const long long bg = (long long)a.B * a.n_kv_heads, most = (1 << 24) - 1;
  // Workgroups: key ranges until there are some for every compute unit, each of a tile a wave at least; then row ranges, of 128
  // rows at least.
  auto ranges = [&](long long sequences, long long keys, long long rows, int* by_key, int* by_row) {
    const long long want = (1024 + sequences - 1) / sequences;
    *by_key = (int)std::max(1LL, std::min({want, (keys + 127) / 128, most / std::max(1LL, sequences)}));
    *by_row = (int)std::max(1LL, std::min({want / *by_key, rows / 128, 64LL, most / std::max(1LL, sequences * *by_key)}));
  };
  p.ctx_keys = p.ctx_splits = p.own_keys = p.own_splits = 1;
  if (T) ranges(bg, T, R, &p.ctx_keys, &p.ctx_splits);
  if (L) ranges(bg * a.K, L, sg, &p.own_keys, &p.own_splits);
  p.keys_by_length = p.ctx_keys >= 8 && a.B > 1 && a.B <= 64 && T >= 512 * p.ctx_keys;
  p.ctx_bytes = p.ctx_splits > 1 ? (size_t)p.ctx_splits * bg * T * sizeof(float) : 0;
  p.own_bytes = p.own_splits > 1 ? (size_t)p.own_splits * bg * a.K * L * sizeof(float) : 0;
  p.blocks = (T ? bg * p.ctx_splits * p.ctx_keys : 0) + (L ? bg * a.K * p.own_splits * p.own_keys : 0);
  p.sum_blocks = std::max(p.ctx_splits > 1 ? (bg * T + 255) / 256 : 0, p.own_splits > 1 ? (bg * a.K * L + 255) / 256 : 0);
  return p;
}

hipError_t launch_packed_attention(const PackedArgs& a, int dh, bool bf16_rows, const PackedPlan& p, hipStream_t s) {
  if (bf16_rows) return dh == 32 ? fwd<bf16, 32>(a, p, s) : dh == 64 ? fwd<bf16, 64>(a, p, s) : fwd<bf16, 128>(a, p, s);
  return dh == 32 ? fwd<float, 32>(a, p, s) : dh == 64 ? fwd<float, 64>(a, p, s) : fwd<float, 128>(a, p, s);
}

hipError_t launch_packed_weights(const PackedArgs& a, int dh, bool bf16_rows, hipStream_t s) {
  if (bf16_rows) return dh == 32 ? weigh<bf16, 32>(a, s) : dh == 64 ? weigh<bf16, 64>(a, s) : weigh<bf16, 128>(a, s);
  return dh == 32 ? weigh<float, 32>(a, s) : dh == 64 ? weigh<float, 64>(a, s) : weigh<float, 128>(a, s);
}

// Paged-cache append (fe_cache_append): new key and value rows to their pages, keys and queries turned
// by their positions on the way.
#include <algorithm>

#include "prefix.h"

namespace {

typedef float f32x8 __attribute__((ext_vector_type(8)));
template <typename T> struct Vec8;
template <> struct Vec8<bf16> { typedef bf16x8 type; };
template <> struct Vec8<float> { typedef f32x8 type; };

constexpr int kMaxRows = 64;            // rows of a workgroup

// Sine and cosine of pos * freq.  The angle is formed and reduced to turns in fp64 (a position of
// 2^31 still leaves 2^-22 of a turn's unit); the reduced turn is split into two floats, and the small one enters
// by its first-order term, so both results are good to fp32 rounding.
FE_DEV void turn(long long pos, double freq, float* c, float* s) {
  const double t = (double)pos * freq * 0.15915494309189535;   // 1 / (2 pi)
  const double f = t - rint(t);
  const float hi = (float)f, lo = (float)(f - (double)hi) * 6.2831853f;
  float sn, cs;
  sincospif(2.f * hi, &sn, &cs);
  *s = fmaf(cs, lo, sn);
  *c = fmaf(-sn, lo, cs);
}

// One workgroup takes `rows` consecutive new rows of one sequence: the sines and cosines of a row are formed
// once, in LDS, for all its heads, then every thread moves units of 16 columns (8 pairs).
// Bound: HBM, every row read and written once (32768 rows of 24 heads of 32, bf16, 101 MB: 18.2 us, 5.5 TB/s); small
// calls launch latency (128 rows of 24 heads of 64: 4.1 us).
template <typename T>
__global__ __launch_bounds__(256) void k_cache_append(fe_append_args a, int rows, int blocks) {
  typedef typename Vec8<T>::type V8;
  __shared__ float s_cos[kMaxRows * 64 / 4], s_sin[kMaxRows * 64 / 4];
  __shared__ long long s_dst[kMaxRows];
  const int tid = threadIdx.x, s = blockIdx.x / blocks, blk = blockIdx.x % blocks;
  const int n = a.new_len ? min(max(a.new_len[s], 0), a.S) : a.S;
  const int len = max(a.len[s], 0);
  const long long pos0 = (a.pos0 ? a.pos0[s] : 0) + (long long)len;
  const int32_t* tab = a.table + (long long)s * a.table_cols;
  const int cap = a.table_cols * a.page_rows;      // the host has checked that it fits
  const int i0 = blk * rows, m = min(rows, n - i0);
  const int np = a.rot / 2;

  if (tid < m) {
    const long long j = (long long)len + i0 + tid;
    long long dst = -1;
    if (j < cap) {
      const int page = tab[(int)j / a.page_rows];
      if (page >= 0 && page < a.n_pages) dst = (long long)page * a.page_rows + (int)j % a.page_rows;
    }
    s_dst[tid] = dst;
  }
  for (int e = tid; e < m * np; e += 256) {
    const int r = e / np;
    turn(pos0 + i0 + r, a.freq[e - r * np], &s_cos[e], &s_sin[e]);
  }
  if (blk == 0 && a.status) {                      // uniform over the workgroup: the pages of all n rows
    int bad = (long long)len + n > cap && n > 0;
    if (n > 0 && len < cap)
      for (int p = len / a.page_rows + tid; p <= (int)(min((long long)len + n, (long long)cap) - 1) / a.page_rows; p += 256)
        bad |= tab[p] < 0 || tab[p] >= a.n_pages;
    bad = block_any<4>(bad);
    if (tid == 0) a.status[s] = bad ? FE_DEV_BAD_PAGE : 0;
  }
  __syncthreads();
  // every thread has read len[s]; with several workgroups per sequence a second launch advances it in place
  if (tid == 0 && blk == 0 && a.len_out && (a.len_out != a.len || blocks == 1))
    a.len_out[s] = (int)min((long long)len + n, 0x7fffffffLL);
  if (m <= 0) return;

  const int hq = a.q ? a.n_heads : 0, per_head = a.dh / 16, units = (hq + 2 * a.n_kv_heads) * per_head;
  const int turned = a.rot / 16;
  for (int e = tid; e < m * units; e += 256) {
    const int r = e / units, u = e - r * units, hh = u / per_head, x = u - hh * per_head;
    const long long row = (long long)s * a.S + i0 + r;
    const T* src;
    T* dst;
    bool is_v = false;
    if (hh < hq) {
      src = static_cast<const T*>(a.q) + row * a.q_ld + hh * a.dh;
      dst = static_cast<T*>(a.q_out) + row * a.q_out_ld + hh * a.dh;
    } else {
      const long long to = s_dst[r];
      if (to < 0) continue;
      const int hk = hh - hq;
      is_v = hk >= a.n_kv_heads;
      const int h = is_v ? hk - a.n_kv_heads : hk;
      src = (is_v ? static_cast<const T*>(a.v) + row * a.v_ld : static_cast<const T*>(a.k) + row * a.k_ld) + h * a.dh;
      dst = static_cast<T*>(is_v ? a.v_pages : a.k_pages) + to * a.page_ld + h * a.dh;
    }
    const bool rot = !is_v && x < turned;
    const bool apart = rot && !a.neighbours;       // the pair's columns lie rot / 2 apart
    const int c0 = apart ? 8 * x : 16 * x, c1 = apart ? 8 * x + np : 16 * x + 8;
    V8 v0 = *reinterpret_cast<const V8*>(src + c0), v1 = *reinterpret_cast<const V8*>(src + c1);
    if (rot) {
      float f[16];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = to_f32((T)v0[i]), f[8 + i] = to_f32((T)v1[i]);
      const float *cs = &s_cos[r * np + 8 * x], *sn = &s_sin[r * np + 8 * x];
      if (apart) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float p = f[i], q = f[8 + i];
          v0[i] = from_f32<T>(p * cs[i] - q * sn[i]);
          v1[i] = from_f32<T>(q * cs[i] + p * sn[i]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v0[2 * i] = from_f32<T>(f[2 * i] * cs[i] - f[2 * i + 1] * sn[i]);
          v0[2 * i + 1] = from_f32<T>(f[2 * i + 1] * cs[i] + f[2 * i] * sn[i]);
          v1[2 * i] = from_f32<T>(f[8 + 2 * i] * cs[4 + i] - f[9 + 2 * i] * sn[4 + i]);
          v1[2 * i + 1] = from_f32<T>(f[9 + 2 * i] * cs[4 + i] + f[8 + 2 * i] * sn[4 + i]);
        }
      }
    }
    *reinterpret_cast<V8*>(dst + c0) = v0;
    *reinterpret_cast<V8*>(dst + c1) = v1;
  }
}

__global__ void k_advance(int32_t* len, const int32_t* new_len, int N, int S) {
  const int s = blockIdx.x * 256 + threadIdx.x;
  if (s >= N) return;
  const int n = new_len ? min(max(new_len[s], 0), S) : S;
  len[s] = (int)min((long long)max(len[s], 0) + n, 0x7fffffffLL);
}

}  // namespace

hipError_t launch_advance(int32_t* len, const int32_t* new_len, int N, int S, hipStream_t s) {
  hipLaunchKernelGGL(k_advance, dim3((unsigned)((N + 255) / 256)), dim3(256), 0, s, len, new_len, N, S);
  return hipGetLastError();
}

hipError_t launch_cache_append(const fe_append_args& a, hipStream_t s) {
  // rows per workgroup: about 512 units of 16 columns, two a thread (ragged prompts, 37 x 129 rows: 256 units 11.7 us,
  // 512 11.2, 1024 12.6, 2048 13.8; 16 x 2048 rows: 18.6, 18.8, 19.3, 20.2), and no more sines than the LDS tables hold
  const int units = ((a.q ? a.n_heads : 0) + 2 * a.n_kv_heads) * (a.dh / 16);
  const int fit = a.rot ? std::min(kMaxRows, kMaxRows * 16 / (a.rot / 2)) : kMaxRows;
  const int rows = std::max(1, std::min({a.S, fit, 512 / std::max(1, units)}));
  const int blocks = (a.S + rows - 1) / rows;
  const dim3 grid((unsigned)((long long)blocks * a.N));
  if (a.dtype == FE_BF16)
    hipLaunchKernelGGL(k_cache_append<bf16>, grid, dim3(256), 0, s, a, rows, blocks);
  else
    hipLaunchKernelGGL(k_cache_append<float>, grid, dim3(256), 0, s, a, rows, blocks);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && a.len_out == a.len && blocks > 1) {
    e = launch_advance(a.len_out, a.new_len, a.N, a.S, s);
  }
  return e;
}

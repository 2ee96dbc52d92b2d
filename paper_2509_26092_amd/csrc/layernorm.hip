// Layer norm over the channels of a row, forward and backward, and the
// reduction of the gradients of its scale and shift.
//   y = (x - mean) rstd gamma + beta, mean = sum x / D,
//   rstd = 1 / sqrt(sum (x - mean)^2 / D + eps)
//   g = dy gamma, xh = (x - mean) rstd,
//   dx = rstd (g - sum g / D - xh sum(g xh) / D),
//   dgamma = sum over rows of dy xh, dbeta = sum over rows of dy
//
// Both passes are bound by memory: a row is read once into registers, the
// sums are taken there (the mean first, then the squares of what is left of
// it, so that a large mean costs no precision), and the result is written
// from there. L lanes hold a row in E chunks of 16 bytes each: part of a
// wave, a wave, or a block.
#include <math.h>

#include <algorithm>

#include "kernels.h"
#include "rows.h"

namespace rn18 {

namespace {

inline int ok() { return hipGetLastError() == hipSuccess ? 0 : -4; }

// ------------------------------------------------------------------ rows in registers
// Sums over the L lanes that hold a row. Lanes of more than one wave meet in
// `sh`, a buffer of the caller that no lane may still read from: callers
// alternate between two.
template <int L, int N>
__device__ inline void row_sums(float (&v)[N], float (*sh)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = group_sum<(L < 64 ? L : 64)>(v[i]);
  if (L > 64) {
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) sh[w][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = sh[0][i];
#pragma unroll
      for (int k = 1; k < L / 64; ++k) v[i] += sh[k][i];
    }
  }
}

template <int VW>
__device__ inline void load_param(const float* p, ChunkAt a, float fill, float* v) {
#pragma unroll
  for (int j = 0; j < VW; ++j) v[j] = fill;
  if (p) __builtin_memcpy(v, p + a.start, VW * 4);
}

// A block takes NT / L * U rows at a time, gridDim.x blocks after another;
// the next rows are loaded while the current ones are worked on.
template <typename T, int L, int E, int U>
__global__ __launch_bounds__(L > 256 ? L : 256) void ln_fwd_kernel(const T* x, const float* __restrict__ gamma,
                                                                   const float* __restrict__ beta, T* y,
                                                                   float* __restrict__ mean, float* __restrict__ rstd,
                                                                   long R, int D, long ldx, long ldy, float eps) {
  constexpr int VW = TT<T>::VW, NT = L > 256 ? L : 256, G = NT / L;
  __shared__ float sh[2][L > 64 ? L / 64 : 1][U];
  const int l = threadIdx.x % L, g = threadIdx.x / L;
  ChunkAt at[E];
  float gm[E][VW], bt[E][VW];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    at[e] = chunk_at<VW>(e * L + l, D);
    load_param<VW>(gamma, at[e], 1.f, gm[e]);
    load_param<VW>(beta, at[e], 0.f, bt[e]);
  }
  const float fd = (float)D;
  const long step = (long)gridDim.x * (G * U);
  long r0 = (long)blockIdx.x * (G * U) + g;
  uint4 q[U][E];
  auto fetch = [&](long base) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long r = base + u * G;
      const T* xr = x + (r < R ? r : R - 1) * ldx;
#pragma unroll
      for (int e = 0; e < E; ++e) q[u][e] = load_chunk(xr + at[e].start);
    }
  };
  fetch(r0);
  for (long b = (long)blockIdx.x * (G * U); b < R; b += step, r0 += step) {   // the same count for every thread
    float v[U][E][VW];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < E; ++e) unpack<T>(q[u][e], v[u][e]);
    if (b + step < R) fetch(r0 + step);
    float m[U], s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      m[u] = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int j = 0; j < VW; ++j) m[u] += e < E - 1 || j >= at[e].skip ? v[u][e][j] : 0.f;
    }
    row_sums<L>(m, sh[0]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      m[u] /= fd;
      s[u] = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int j = 0; j < VW; ++j) {
          v[u][e][j] -= m[u];
          s[u] += e < E - 1 || j >= at[e].skip ? v[u][e][j] * v[u][e][j] : 0.f;
        }
    }
    row_sums<L>(s, sh[1]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float rs = 1.0f / sqrtf(s[u] / fd + eps);
      const long r = r0 + u * G;
      if (r >= R) continue;
      T* yr = y + r * ldy;
#pragma unroll
      for (int e = 0; e < E; ++e) {
#pragma unroll
        for (int j = 0; j < VW; ++j) v[u][e][j] = v[u][e][j] * (rs * gm[e][j]) + bt[e][j];
        if (e < E - 1) store_chunk(yr + at[e].start, pack<T>(v[u][e]));
        else store_owned(yr, at[e], v[u][e]);
      }
      if (l == 0) {
        if (mean) mean[r] = m[u];
        if (rstd) rstd[r] = rs;
      }
    }
  }
}

// The backward pass keeps the sums of dgamma and dbeta of its columns in
// registers over all its rows, joins them over the block's row groups, and
// writes one partial row per block: part[block][2][Dp] (Dp = D rounded up to
// 4), or, a block alone, the gradients themselves.
struct LnParamOut {
  float* part;     // NULL: no parameter gradient is wanted
  float *dgamma, *dbeta;
  int Dp;
};

template <typename T, int L, int E>
__global__ __launch_bounds__(L > 256 ? L : 256) void ln_bwd_kernel(const T* dy, const T* x,
                                                                   const float* __restrict__ gamma,
                                                                   const float* __restrict__ mean,
                                                                   const float* __restrict__ rstd, T* dx,
                                                                   LnParamOut po, long R, int D, long lddy, long ldx,
                                                                   long lddx) {
  constexpr int VW = TT<T>::VW, NT = L > 256 ? L : 256, G = NT / L, NW = NT / 64;
  constexpr int NV = 2 * E * VW;
  // joining of the row groups: a wave's own in registers, the waves' here
  __shared__ float shp[L > 64 ? 1 : NW][L > 64 ? 1 : L * NV];
  __shared__ float sh[2][L > 64 ? L / 64 : 1][2];
  const int l = threadIdx.x % L, g = threadIdx.x / L;
  ChunkAt at[E];
  float gm[E][VW], ag[E][VW], ab[E][VW];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    at[e] = chunk_at<VW>(e * L + l, D);
    load_param<VW>(gamma, at[e], 1.f, gm[e]);
#pragma unroll
    for (int j = 0; j < VW; ++j) ag[e][j] = ab[e][j] = 0.f;
  }
  const float fd = (float)D;
  const long step = (long)gridDim.x * G;
  long r = (long)blockIdx.x * G + g;
  uint4 qd[E], qx[E];
  float m, rs;
  auto fetch = [&](long row) {
    const long rc = row < R ? row : R - 1;
    const T *pd = dy + rc * lddy, *px = x + rc * ldx;
    m = mean[rc];
    rs = rstd[rc];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      qd[e] = load_chunk(pd + at[e].start);
      qx[e] = load_chunk(px + at[e].start);
    }
  };
  fetch(r);
  int odd = 0;
  for (long b = (long)blockIdx.x * G; b < R; b += step, r += step, odd ^= 1) {
    float d[E][VW], xh[E][VW];
    const bool in = r < R;
    const float m0 = m, rs0 = rs;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      unpack<T>(qd[e], d[e]);
      unpack<T>(qx[e], xh[e]);
    }
    if (b + step < R) fetch(r + step);
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int j = 0; j < VW; ++j) {
        xh[e][j] = (xh[e][j] - m0) * rs0;
        const bool own = in && (e < E - 1 || j >= at[e].skip);
        const float dj = own ? d[e][j] : 0.f;
        const float t = own ? d[e][j] * xh[e][j] : 0.f;
        ab[e][j] += dj;
        ag[e][j] += t;
        s[0] += dj * gm[e][j];
        s[1] += t * gm[e][j];
      }
    row_sums<L>(s, sh[odd]);
    const float a = s[0] / fd, c = s[1] / fd;
    if (in) {
      T* dxr = dx + r * lddx;
#pragma unroll
      for (int e = 0; e < E; ++e) {
#pragma unroll
        for (int j = 0; j < VW; ++j) d[e][j] = rs0 * (d[e][j] * gm[e][j] - a - xh[e][j] * c);
        if (e < E - 1) store_chunk(dxr + at[e].start, pack<T>(d[e]));
        else store_owned(dxr, at[e], d[e]);
      }
    }
  }
  if (!po.part && !po.dgamma && !po.dbeta) return;
  float* og = po.part ? po.part + (long)blockIdx.x * 2 * po.Dp : po.dgamma;
  float* ob = po.part ? po.part + ((long)blockIdx.x * 2 + 1) * po.Dp : po.dbeta;
  if constexpr (L <= 64) {
    const int w = threadIdx.x >> 6, wl = threadIdx.x & 63;
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int j = 0; j < VW; ++j) {
#pragma unroll
        for (int o = L; o < 64; o <<= 1) {
          ag[e][j] += __shfl_xor(ag[e][j], o);
          ab[e][j] += __shfl_xor(ab[e][j], o);
        }
        if (wl < L) {
          shp[w][((e * VW + j) * 2) * L + wl] = ag[e][j];
          shp[w][((e * VW + j) * 2 + 1) * L + wl] = ab[e][j];
        }
      }
    __syncthreads();
    if (threadIdx.x >= L) return;
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int j = 0; j < VW; ++j) {
        ag[e][j] = shp[0][((e * VW + j) * 2) * L + l];
        ab[e][j] = shp[0][((e * VW + j) * 2 + 1) * L + l];
#pragma unroll
        for (int k = 1; k < NW; ++k) {
          ag[e][j] += shp[k][((e * VW + j) * 2) * L + l];
          ab[e][j] += shp[k][((e * VW + j) * 2 + 1) * L + l];
        }
      }
  }
#pragma unroll
  for (int e = 0; e < E; ++e)
#pragma unroll
    for (int j = 0; j < VW; ++j)
      if (j >= at[e].skip) {
        if (og) og[at[e].start + j] = ag[e][j];
        if (ob) ob[at[e].start + j] = ab[e][j];
      }
}

// Columns of the partial rows added up in the order of the blocks: 8 lanes of
// 4 columns by 32 groups of rows a block, the groups' sums added in order.
__global__ __launch_bounds__(256) void ln_param_sum_kernel(const float* __restrict__ part, int nb, int D, int Dp,
                                                           float* __restrict__ dgamma, float* __restrict__ dbeta) {
  __shared__ float sh[32][33];
  const int cl = threadIdx.x & 7, rg = threadIdx.x >> 3;
  const int c = blockIdx.x * 32 + cl * 4;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (c < Dp) {
    const float* p = part + (long)blockIdx.y * Dp + c;
#pragma unroll 4
    for (int b = rg; b < nb; b += 32) {
      const float4 v = *(const float4*)(p + (long)b * 2 * Dp);
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
  }
  sh[rg][cl * 4] = s.x; sh[rg][cl * 4 + 1] = s.y; sh[rg][cl * 4 + 2] = s.z; sh[rg][cl * 4 + 3] = s.w;
  __syncthreads();
  const int k = threadIdx.x, col = blockIdx.x * 32 + k;
  float* o = blockIdx.y ? dbeta : dgamma;
  if (k < 32 && col < D && o) {
    float t = sh[0][k];
    for (int i = 1; i < 32; ++i) t += sh[i][k];
    o[col] = t;
  }
}

// ------------------------------------------------------------------ rows of a few elements
// Rows shorter than a chunk: a thread per row.
template <typename T>
__global__ __launch_bounds__(256) void ln_fwd_short_kernel(const T* x, const float* __restrict__ gamma,
                                                           const float* __restrict__ beta, T* y,
                                                           float* __restrict__ mean, float* __restrict__ rstd, long R,
                                                           int D, long ldx, long ldy, float eps) {
  for (long r = blockIdx.x * 256l + threadIdx.x; r < R; r += gridDim.x * 256l) {
    float v[TT<T>::VW], s = 0.f, q = 0.f;
#pragma unroll
    for (int j = 0; j < TT<T>::VW; ++j) {
      v[j] = j < D ? TT<T>::to_f(x[r * ldx + j]) : 0.f;
      s += v[j];
    }
    const float m = s / (float)D;
#pragma unroll
    for (int j = 0; j < TT<T>::VW; ++j) {
      v[j] = j < D ? v[j] - m : 0.f;
      q += v[j] * v[j];
    }
    const float rs = 1.0f / sqrtf(q / (float)D + eps);
#pragma unroll
    for (int j = 0; j < TT<T>::VW; ++j)
      if (j < D) y[r * ldy + j] = TT<T>::from_f(v[j] * (rs * (gamma ? gamma[j] : 1.f)) + (beta ? beta[j] : 0.f));
    if (mean) mean[r] = m;
    if (rstd) rstd[r] = rs;
  }
}

template <typename T>
__global__ __launch_bounds__(256) void ln_bwd_short_kernel(const T* dy, const T* x, const float* __restrict__ gamma,
                                                           const float* __restrict__ mean,
                                                           const float* __restrict__ rstd, T* dx, LnParamOut po, long R,
                                                           int D, long lddy, long ldx, long lddx) {
  constexpr int VW = TT<T>::VW;
  __shared__ float sh[4][2 * VW];
  float ag[VW], ab[VW];
#pragma unroll
  for (int j = 0; j < VW; ++j) ag[j] = ab[j] = 0.f;
  for (long r = blockIdx.x * 256l + threadIdx.x; r < R; r += gridDim.x * 256l) {
    const float m = mean[r], rs = rstd[r];
    float g[VW], xh[VW], a = 0.f, c = 0.f;
#pragma unroll
    for (int j = 0; j < VW; ++j) {
      const float d = j < D ? TT<T>::to_f(dy[r * lddy + j]) : 0.f;
      xh[j] = j < D ? (TT<T>::to_f(x[r * ldx + j]) - m) * rs : 0.f;
      g[j] = j < D && gamma ? d * gamma[j] : d;
      ag[j] += d * xh[j];
      ab[j] += d;
      a += g[j];
      c += g[j] * xh[j];
    }
    a /= (float)D;
    c /= (float)D;
#pragma unroll
    for (int j = 0; j < VW; ++j)
      if (j < D) dx[r * lddx + j] = TT<T>::from_f(rs * (g[j] - a - xh[j] * c));
  }
  if (!po.part) return;
#pragma unroll
  for (int j = 0; j < VW; ++j) {
    ag[j] = group_sum<64>(ag[j]);
    ab[j] = group_sum<64>(ab[j]);
    if ((threadIdx.x & 63) == 0) {
      sh[threadIdx.x >> 6][j] = ag[j];
      sh[threadIdx.x >> 6][VW + j] = ab[j];
    }
  }
  __syncthreads();
  const int k = threadIdx.x, j = k % VW;
  if (k < 2 * VW && j < D)
    po.part[((long)blockIdx.x * 2 + k / VW) * po.Dp + j] = ((sh[0][k] + sh[1][k]) + sh[2][k]) + sh[3][k];
}

// ------------------------------------------------------------------ rows beyond a block's registers
// A block of 1024 threads per row reads it three times.
__device__ inline float block_sum1024(float v, float* sh) {
  v = group_sum<64>(v);
  __syncthreads();   // earlier readers of sh are done
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = sh[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) t += sh[i];
  return t;
}

template <typename T>
__global__ __launch_bounds__(1024) void ln_fwd_long_kernel(const T* x, const float* __restrict__ gamma,
                                                           const float* __restrict__ beta, T* y,
                                                           float* __restrict__ mean, float* __restrict__ rstd, long R,
                                                           int D, long ldx, long ldy, float eps) {
  constexpr int VW = TT<T>::VW;
  __shared__ float sh[16];
  const int nch = D / VW, tail = nch * VW + (int)threadIdx.x;   // whole chunks, and one element each of the rest
  for (long r = blockIdx.x; r < R; r += gridDim.x) {
    const T* xr = x + r * ldx;
    T* yr = y + r * ldy;
    float s = tail < D ? TT<T>::to_f(xr[tail]) : 0.f;
    for (int c = threadIdx.x; c < nch; c += 1024) {
      float v[VW];
      unpack<T>(load_chunk(xr + (long)c * VW), v);
#pragma unroll
      for (int j = 0; j < VW; ++j) s += v[j];
    }
    const float m = block_sum1024(s, sh) / (float)D;
    s = 0.f;
    if (tail < D) {
      const float t = TT<T>::to_f(xr[tail]) - m;
      s = t * t;
    }
    for (int c = threadIdx.x; c < nch; c += 1024) {
      float v[VW];
      unpack<T>(load_chunk(xr + (long)c * VW), v);
#pragma unroll
      for (int j = 0; j < VW; ++j) s += (v[j] - m) * (v[j] - m);
    }
    const float rs = 1.0f / sqrtf(block_sum1024(s, sh) / (float)D + eps);
    if (tail < D)
      yr[tail] = TT<T>::from_f((TT<T>::to_f(xr[tail]) - m) * (rs * (gamma ? gamma[tail] : 1.f)) +
                               (beta ? beta[tail] : 0.f));
    for (int c = threadIdx.x; c < nch; c += 1024) {
      float v[VW], gm[VW], bt[VW];
      const ChunkAt a{c * VW, 0};
      unpack<T>(load_chunk(xr + a.start), v);
      load_param<VW>(gamma, a, 1.f, gm);
      load_param<VW>(beta, a, 0.f, bt);
#pragma unroll
      for (int j = 0; j < VW; ++j) v[j] = (v[j] - m) * (rs * gm[j]) + bt[j];
      store_chunk(yr + a.start, pack<T>(v));
    }
    if (threadIdx.x == 0) {
      if (mean) mean[r] = m;
      if (rstd) rstd[r] = rs;
    }
  }
}

template <typename T>
__global__ __launch_bounds__(1024) void ln_bwd_long_kernel(const T* dy, const T* x, const float* __restrict__ gamma,
                                                           const float* __restrict__ mean,
                                                           const float* __restrict__ rstd, T* dx, long R, int D,
                                                           long lddy, long ldx, long lddx) {
  constexpr int VW = TT<T>::VW;
  __shared__ float sh[16];
  const int nch = D / VW, tail = nch * VW + (int)threadIdx.x;
  for (long r = blockIdx.x; r < R; r += gridDim.x) {
    const T *dyr = dy + r * lddy, *xr = x + r * ldx;
    T* dxr = dx + r * lddx;
    const float m = mean[r], rs = rstd[r];
    float a = 0.f, b = 0.f, tg = 0.f, tx = 0.f;
    if (tail < D) {
      tg = TT<T>::to_f(dyr[tail]) * (gamma ? gamma[tail] : 1.f);
      tx = (TT<T>::to_f(xr[tail]) - m) * rs;
      a = tg;
      b = tg * tx;
    }
    for (int c = threadIdx.x; c < nch; c += 1024) {
      float g[VW], v[VW], gm[VW];
      const ChunkAt at{c * VW, 0};
      unpack<T>(load_chunk(dyr + at.start), g);
      unpack<T>(load_chunk(xr + at.start), v);
      load_param<VW>(gamma, at, 1.f, gm);
#pragma unroll
      for (int j = 0; j < VW; ++j) {
        a += g[j] * gm[j];
        b += g[j] * gm[j] * ((v[j] - m) * rs);
      }
    }
    a = block_sum1024(a, sh) / (float)D;
    b = block_sum1024(b, sh) / (float)D;
    if (tail < D) dxr[tail] = TT<T>::from_f(rs * (tg - a - tx * b));
    for (int c = threadIdx.x; c < nch; c += 1024) {
      float g[VW], v[VW], gm[VW];
      const ChunkAt at{c * VW, 0};
      unpack<T>(load_chunk(dyr + at.start), g);
      unpack<T>(load_chunk(xr + at.start), v);
      load_param<VW>(gamma, at, 1.f, gm);
#pragma unroll
      for (int j = 0; j < VW; ++j) g[j] = rs * (g[j] * gm[j] - a - (v[j] - m) * rs * b);
      store_chunk(dxr + at.start, pack<T>(g));
    }
  }
}

// Its parameter gradients: block (columns of 256, range of rows) writes one
// partial row.
template <typename T>
__global__ __launch_bounds__(256) void ln_param_long_kernel(const T* __restrict__ dy, const T* __restrict__ x,
                                                            const float* __restrict__ mean,
                                                            const float* __restrict__ rstd, LnParamOut po, long R,
                                                            int D, long lddy, long ldx) {
  const long c = (long)blockIdx.x * 256 + threadIdx.x;
  if (c >= D) return;
  float sg = 0.f, sb = 0.f;
  for (long r = blockIdx.y; r < R; r += gridDim.y) {
    const float g = TT<T>::to_f(dy[r * lddy + c]);
    sg += g * ((TT<T>::to_f(x[r * ldx + c]) - mean[r]) * rstd[r]);
    sb += g;
  }
  float* p = po.part + (long)blockIdx.y * 2 * po.Dp;
  p[c] = sg;
  p[po.Dp + c] = sb;
}

// ------------------------------------------------------------------ choice of kernel
enum LnPath { LN_SHORT, LN_TILE, LN_LONG };

// The lanes L and chunks E of a row of D elements: one chunk per lane up to a
// wave, then up to `max_e` chunks per lane of a wave, and of blocks of up to
// 1024 threads.
LnPath ln_tile(int prec, int D, int max_e, int* L, int* E) {
  const int vw = prec_vw(prec);
  if (D < vw) return LN_SHORT;
  const int nch = ceil_div(D, vw);
  *E = 1;
  *L = 1;
  while (*L < 64 && *L < nch) *L *= 2;
  if (nch <= 64) return LN_TILE;
  for (int l = 64; l <= 1024; l *= l == 64 ? 4 : 2)
    if (nch <= l * max_e) {
      *L = l;
      *E = ceil_div(nch, l);
      return LN_TILE;
    }
  return LN_LONG;
}

// Blocks for `units` pieces of work, `per_cu` blocks a compute unit at most,
// all with the same number of pieces but for the last.
int even_grid(long units, int per_cu) {
  const long most = (long)per_cu * plan_cus();
  if (units <= most) return (int)std::max(1l, units);
  const long each = (units + most - 1) / most;
  return (int)((units + each - 1) / each);
}

int ln_fwd_per_cu(int L) { return L > 256 ? 2048 / L : 8; }

template <typename T, int L, int E, int U, typename... A>
int fwd_go(long R, hipStream_t s, A... a) {
  constexpr int NT = L > 256 ? L : 256;
  const long units = (R + NT / L * U - 1) / (NT / L * U);
  hipLaunchKernelGGL((ln_fwd_kernel<T, L, E, U>), dim3(even_grid(units, ln_fwd_per_cu(L))), dim3(NT), 0, s, a...);
  return ok();
}

// Several rows a lane at once where there are enough to fill the chip so.
template <typename T, int L, int E, int U, typename... A>
int fwd_u(long R, hipStream_t s, A... a) {
  if (U > 1 && R >= (long)plan_cus() * (256 / L) * U * 2) return fwd_go<T, L, E, U>(R, s, a...);
  return fwd_go<T, L, E, 1>(R, s, a...);
}

template <typename T, typename... A>
int fwd_tile(int L, int E, long R, hipStream_t s, A... a) {
  switch (L * 8 + E) {
    case 1 * 8 + 1: return fwd_u<T, 1, 1, 2>(R, s, a...);
    case 2 * 8 + 1: return fwd_u<T, 2, 1, 2>(R, s, a...);
    case 4 * 8 + 1: return fwd_u<T, 4, 1, 2>(R, s, a...);
    case 8 * 8 + 1: return fwd_u<T, 8, 1, 2>(R, s, a...);
    case 16 * 8 + 1: return fwd_u<T, 16, 1, 2>(R, s, a...);
    case 32 * 8 + 1: return fwd_u<T, 32, 1, 2>(R, s, a...);
    case 64 * 8 + 1: return fwd_u<T, 64, 1, 2>(R, s, a...);
    case 64 * 8 + 2: return fwd_u<T, 64, 2, 1>(R, s, a...);
    case 64 * 8 + 3: return fwd_u<T, 64, 3, 1>(R, s, a...);
    case 64 * 8 + 4: return fwd_u<T, 64, 4, 1>(R, s, a...);
    case 256 * 8 + 2: return fwd_go<T, 256, 2, 1>(R, s, a...);
    case 256 * 8 + 3: return fwd_go<T, 256, 3, 1>(R, s, a...);
    case 256 * 8 + 4: return fwd_go<T, 256, 4, 1>(R, s, a...);
    case 512 * 8 + 3: return fwd_go<T, 512, 3, 1>(R, s, a...);
    case 512 * 8 + 4: return fwd_go<T, 512, 4, 1>(R, s, a...);
    case 1024 * 8 + 3: return fwd_go<T, 1024, 3, 1>(R, s, a...);
    case 1024 * 8 + 4: return fwd_go<T, 1024, 4, 1>(R, s, a...);
    default: return -1;
  }
}

// Blocks of the backward pass, one partial row each.
int bwd_grid(LnPath path, int L, long R, int D) {
  if (path == LN_SHORT) return even_grid((R + 255) / 256, 2);
  if (path == LN_LONG) return (int)std::max(1l, std::min(R, 8l * plan_cus() / ceil_div(D, 256)));
  const int G = L > 256 ? 1 : 256 / L;
  return even_grid((R + G - 1) / G, L > 256 ? 1024 / L : 4);
}

template <typename T, int L, int E, typename... A>
int bwd_go(int grid, hipStream_t s, A... a) {
  hipLaunchKernelGGL((ln_bwd_kernel<T, L, E>), dim3(grid), dim3(L > 256 ? L : 256), 0, s, a...);
  return ok();
}

template <typename T, typename... A>
int bwd_tile(int L, int E, int grid, hipStream_t s, A... a) {
  switch (L * 8 + E) {
    case 1 * 8 + 1: return bwd_go<T, 1, 1>(grid, s, a...);
    case 2 * 8 + 1: return bwd_go<T, 2, 1>(grid, s, a...);
    case 4 * 8 + 1: return bwd_go<T, 4, 1>(grid, s, a...);
    case 8 * 8 + 1: return bwd_go<T, 8, 1>(grid, s, a...);
    case 16 * 8 + 1: return bwd_go<T, 16, 1>(grid, s, a...);
    case 32 * 8 + 1: return bwd_go<T, 32, 1>(grid, s, a...);
    case 64 * 8 + 1: return bwd_go<T, 64, 1>(grid, s, a...);
    case 64 * 8 + 2: return bwd_go<T, 64, 2>(grid, s, a...);
    case 256 * 8 + 2: return bwd_go<T, 256, 2>(grid, s, a...);
    default: break;
  }
  if constexpr (TT<T>::VW == 8) {
    switch (L * 8 + E) {
      case 256 * 8 + 1: return bwd_go<T, 256, 1>(grid, s, a...);
      case 512 * 8 + 2: return bwd_go<T, 512, 2>(grid, s, a...);
      case 1024 * 8 + 2: return bwd_go<T, 1024, 2>(grid, s, a...);
      default: return -1;
    }
  } else {
    switch (L * 8 + E) {
      case 64 * 8 + 3: return bwd_go<T, 64, 3>(grid, s, a...);
      case 64 * 8 + 4: return bwd_go<T, 64, 4>(grid, s, a...);
      case 256 * 8 + 3: return bwd_go<T, 256, 3>(grid, s, a...);
      case 256 * 8 + 4: return bwd_go<T, 256, 4>(grid, s, a...);
      case 512 * 8 + 3: return bwd_go<T, 512, 3>(grid, s, a...);
      case 512 * 8 + 4: return bwd_go<T, 512, 4>(grid, s, a...);
      case 1024 * 8 + 3: return bwd_go<T, 1024, 3>(grid, s, a...);
      case 1024 * 8 + 4: return bwd_go<T, 1024, 4>(grid, s, a...);
      default: return -1;
    }
  }
}
constexpr int kFwdMaxE = 4;
int bwd_max_e(int prec) { return 16 / prec_vw(prec); }   // 16 columns a lane: their sums and gamma in 48 registers

int row_grid(long R) { return (int)std::min(R, 65536l); }

}  // namespace

int layernorm_fwd_launch(int prec, const void* x, const float* gamma, const float* beta, void* y, float* mean,
                         float* rstd, long R, int D, long ldx, long ldy, float eps, hipStream_t s) {
  if (R <= 0) return 0;
  int L = 0, E = 0;
  const LnPath path = ln_tile(prec, D, kFwdMaxE, &L, &E);
  return with_prec(prec, [&](auto tag) {
    using T = decltype(tag);
    const T* xt = (const T*)x;
    T* yt = (T*)y;
    if (path == LN_TILE) return fwd_tile<T>(L, E, R, s, xt, gamma, beta, yt, mean, rstd, R, D, ldx, ldy, eps);
    if (path == LN_SHORT)
      hipLaunchKernelGGL(ln_fwd_short_kernel<T>, dim3(row_grid((R + 255) / 256)), dim3(256), 0, s, xt, gamma, beta, yt,
                         mean, rstd, R, D, ldx, ldy, eps);
    else
      hipLaunchKernelGGL(ln_fwd_long_kernel<T>, dim3(row_grid(R)), dim3(1024), 0, s, xt, gamma, beta, yt, mean, rstd, R,
                         D, ldx, ldy, eps);
    return ok();
  });
}

size_t layernorm_bwd_workspace(int prec, long R, int D) {
  if (R <= 0) return 0;
  int L = 0, E = 0;
  const LnPath path = ln_tile(prec, D, bwd_max_e(prec), &L, &E);
  return (size_t)bwd_grid(path, L, R, D) * 2 * ((D + 3) & ~3) * 4;
}

int layernorm_bwd_launch(int prec, const void* dy, const void* x, const float* gamma, const float* mean,
                         const float* rstd, void* dx, float* dgamma, float* dbeta, long R, int D, long lddy, long ldx,
                         long lddx, void* ws, hipStream_t s) {
  int L = 0, E = 0;
  const LnPath path = ln_tile(prec, D, bwd_max_e(prec), &L, &E);
  const bool params = dgamma || dbeta;
  const int grid = R > 0 ? bwd_grid(path, L, R, D) : 0;
  const LnParamOut po{params ? (float*)ws : nullptr, nullptr, nullptr, (D + 3) & ~3};
  if (R > 0) {
    const int r = with_prec(prec, [&](auto tag) {
      using T = decltype(tag);
      const T *dyt = (const T*)dy, *xt = (const T*)x;
      T* dxt = (T*)dx;
      if (path == LN_TILE)
        return bwd_tile<T>(L, E, grid, s, dyt, xt, gamma, mean, rstd, dxt, po, R, D, lddy, ldx, lddx);
      if (path == LN_SHORT) {
        hipLaunchKernelGGL(ln_bwd_short_kernel<T>, dim3(grid), dim3(256), 0, s, dyt, xt, gamma, mean, rstd, dxt, po, R,
                           D, lddy, ldx, lddx);
        return ok();
      }
      if (params)   // before dx, which may replace dy or x
        hipLaunchKernelGGL(ln_param_long_kernel<T>, dim3(ceil_div(D, 256), grid), dim3(256), 0, s, dyt, xt, mean, rstd,
                           po, R, D, lddy, ldx);
      hipLaunchKernelGGL(ln_bwd_long_kernel<T>, dim3(row_grid(R)), dim3(1024), 0, s, dyt, xt, gamma, mean, rstd, dxt, R,
                         D, lddy, ldx, lddx);
      return ok();
    });
    if (r) return r;
  }
  if (params) {
    hipLaunchKernelGGL(ln_param_sum_kernel, dim3(ceil_div(po.Dp, 32), 2), dim3(256), 0, s, (const float*)ws, grid, D,
                       po.Dp, dgamma, dbeta);
    return ok();
  }
  return 0;
}

}  // namespace rn18

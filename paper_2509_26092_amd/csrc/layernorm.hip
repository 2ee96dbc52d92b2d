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
// wave, a wave, or a block. On 802816x64 bf16 the forward pass takes 41 us and
// the backward pass 60 (5.0 and 5.1 TB/s, a copy's rate), the backward pass on
// 16384x8192 bf16 160 us (5.0 TB/s). Rows beyond a block's registers are read
// two or three times: 4096x32768 bf16 forward 153 us (3.5 TB/s for one read
// and one write), backward 358.
#include <math.h>

#include <algorithm>

#include "kernels.h"
#include "rows.h"

namespace rn18 {

namespace {

inline int ok() { return hipGetLastError() == hipSuccess ? 0 : -4; }

// ------------------------------------------------------------------ rows in registers
template <int VW>
__device__ inline void load_param(const float* p, int start, float fill, float* v) {
#pragma unroll
  for (int j = 0; j < VW; ++j) v[j] = fill;
  if (p) __builtin_memcpy(v, p + start, VW * 4);
}

// Where a lane's E chunks start (e * L + l of the row), whether it has the
// last of them (the others are whole), and its element of the tail. L >= 8
// lanes where there is a tail.
template <int VW, int L, int E>
struct Span {
  int start[E], tail;
  bool last, has_tail;
  __device__ Span(int l, int D) {
    const int nch = D / VW;
#pragma unroll
    for (int e = 0; e < E; ++e) start[e] = (e * L + l) * VW;
    last = (E - 1) * L + l < nch;
    if (!last) start[E - 1] = 0;
    tail = nch * VW + l;
    has_tail = tail < D;
  }
};

// A block takes NT / L * U rows at a time, gridDim.x blocks after another;
// the next rows are loaded while the current ones are worked on.
template <typename T, int L, int E, int U>
__global__ __launch_bounds__(L > 256 ? L : 256) void ln_fwd_kernel(const T* x, const float* __restrict__ gamma,
                                                                   const float* __restrict__ beta, T* y,
                                                                   float* __restrict__ mean, float* __restrict__ rstd,
                                                                   long R, int D, long ldx, long ldy, float eps) {
  constexpr int VW = TT<T>::VW, NT = L > 256 ? L : 256, G = NT / L;
  __shared__ float sh[2][L > 64 ? L / 64 : 1][U];
  const int l = threadIdx.x % L, g = L < NT ? threadIdx.x / L : 0;
  const Span<VW, L, E> at(l, D);
  const bool tails = D % VW != 0;
  float gm[E][VW], bt[E][VW], gt = 1.f, tb = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    load_param<VW>(gamma, at.start[e], 1.f, gm[e]);
    load_param<VW>(beta, at.start[e], 0.f, bt[e]);
  }
  if (at.has_tail) {
    if (gamma) gt = gamma[at.tail];
    if (beta) tb = beta[at.tail];
  }
  const float fd = (float)D;
  const long step = (long)gridDim.x * (G * U);
  long r0 = (long)blockIdx.x * (G * U) + g;
  uint4 q[U][E];
  T qt[U];
  auto fetch = [&](long base) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long r = base + u * G;
      const T* xr = x + (r < R ? r : R - 1) * ldx;
#pragma unroll
      for (int e = 0; e < E; ++e) q[u][e] = load_chunk(xr + at.start[e]);
      if (tails) qt[u] = xr[at.has_tail ? at.tail : 0];
    }
  };
  fetch(r0);
  for (long b = (long)blockIdx.x * (G * U); b < R; b += step, r0 += step) {   // the same count for every thread
    float v[U][E][VW], t[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int e = 0; e < E; ++e) unpack<T>(q[u][e], v[u][e]);
      t[u] = tails && at.has_tail ? TT<T>::to_f(qt[u]) : 0.f;
    }
    if (b + step < R) fetch(r0 + step);
    float m[U], s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float w = 0.f;
      m[u] = t[u];
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int j = 0; j < VW; ++j) (e < E - 1 ? m[u] : w) += v[u][e][j];
      if (at.last) m[u] += w;
    }
    row_sums<L>(m, sh[0]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float w = 0.f;
      m[u] /= fd;
      t[u] -= m[u];
      s[u] = at.has_tail ? t[u] * t[u] : 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int j = 0; j < VW; ++j) {
          v[u][e][j] -= m[u];
          (e < E - 1 ? s[u] : w) += v[u][e][j] * v[u][e][j];
        }
      if (at.last) s[u] += w;
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
        if (e < E - 1 || at.last) store_chunk(yr + at.start[e], pack<T>(v[u][e]));
      }
      if (at.has_tail) yr[at.tail] = TT<T>::from_f(t[u] * (rs * gt) + tb);
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
// 4).
// Small calls take one launch instead: dgamma and dbeta need no row sums, so
// blocks of their own (from row_blocks on) add up 32 columns each over all
// rows, beside the blocks that write dx.
struct LnParamOut {
  float* part;     // NULL: no parameter gradient is wanted, or blocks of their own write them
  int Dp;
  int row_blocks;
  float *dgamma, *dbeta;
};

// Sums over the rows of 32 columns from c0: 8 lanes of 4 columns by 32 groups
// of rows (the block's first 256 threads), the groups' sums by fours and the
// fours in order.
template <typename T>
__device__ inline void ln_columns(const T* dy, const T* x, const float* mean, const float* rstd, float* dgamma,
                                  float* dbeta, long R, int D, long lddy, long ldx, int c0) {
  __shared__ float sh[2][32][33], sh2[2][8][33];
  const int t = threadIdx.x, cl = (t & 7) * 4, rg = t >> 3, c = c0 + cl;
  float g[4] = {}, b[4] = {};
  if (t < 256 && c < D) {
#pragma unroll 4
    for (long r = rg; r < R; r += 32) {
      const float m = mean[r], rs = rstd[r];
      T qd[4] = {}, qx[4] = {};
      if (c + 4 <= D) {
        __builtin_memcpy(qd, dy + r * lddy + c, 4 * sizeof(T));
        __builtin_memcpy(qx, x + r * ldx + c, 4 * sizeof(T));
      } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
          if (j < D - c) {
            qd[j] = dy[r * lddy + c + j];
            qx[j] = x[r * ldx + c + j];
          }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float d = TT<T>::to_f(qd[j]);
        b[j] += d;
        g[j] += d * ((TT<T>::to_f(qx[j]) - m) * rs);
      }
    }
  }
  if (t < 256)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      sh[0][rg][cl + j] = g[j];
      sh[1][rg][cl + j] = b[j];
    }
  __syncthreads();
  const int k = t & 31, q = t >> 5;
  if (t < 256)
#pragma unroll
    for (int w = 0; w < 2; ++w)
      sh2[w][q][k] = (sh[w][4 * q][k] + sh[w][4 * q + 1][k]) + (sh[w][4 * q + 2][k] + sh[w][4 * q + 3][k]);
  __syncthreads();
  float* o = q == 0 ? dgamma : dbeta;
  if (q < 2 && c0 + k < D && o) {
    float v = sh2[q][0][k];
#pragma unroll
    for (int i = 1; i < 8; ++i) v += sh2[q][i][k];
    o[c0 + k] = v;
  }
}

// WIDE: for the widest rows, whose column sums would not fit in registers
// beside two rows: the sums live in LDS (each lane adds to its own columns)
// and gamma is read again for every row.
template <typename T, int L, int E, bool WIDE = false>
__global__ __launch_bounds__(L > 256 ? L : 256) void ln_bwd_kernel(const T* dy, const T* x,
                                                                   const float* __restrict__ gamma,
                                                                   const float* __restrict__ mean,
                                                                   const float* __restrict__ rstd, T* dx,
                                                                   LnParamOut po, long R, int D, long lddy, long ldx,
                                                                   long lddx) {
  constexpr int VW = TT<T>::VW, NT = L > 256 ? L : 256, G = NT / L, NW = NT / 64;
  constexpr int NV = 2 * (E * VW + 1);
  if (!WIDE && (int)blockIdx.x >= po.row_blocks) {
    ln_columns(dy, x, mean, rstd, po.dgamma, po.dbeta, R, D, lddy, ldx, ((int)blockIdx.x - po.row_blocks) * 32);
    return;
  }
  // joining of the row groups: a wave's own in registers, the waves' here
  __shared__ float shp[L > 64 ? 1 : NW][L > 64 ? 1 : L * NV];
  __shared__ float sh[2][L > 64 ? L / 64 : 1][2];
  constexpr int Q = E * VW / 4;   // float4 column sums of a lane
  __shared__ float4 wide[WIDE ? 2 : 1][WIDE ? Q : 1][WIDE ? L : 1];
  const int l = threadIdx.x % L, g = L < NT ? threadIdx.x / L : 0;
  const Span<VW, L, E> at(l, D);
  const bool tails = D % VW != 0;
  float gm[E][VW], ag[E * VW + 1], ab[E * VW + 1], gt = 1.f;
  if (WIDE)
#pragma unroll
    for (int i = 0; i < Q; ++i) wide[0][i][l] = wide[WIDE][i][l] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (!WIDE) load_param<VW>(gamma, at.start[e], 1.f, gm[e]);
  if (at.has_tail && gamma) gt = gamma[at.tail];
#pragma unroll
  for (int i = 0; i <= E * VW; ++i) ag[i] = ab[i] = 0.f;
  const float fd = (float)D;
  const long step = (long)po.row_blocks * G;
  long r = (long)blockIdx.x * G + g;
  uint4 qd[E], qx[E], nd[E], nx[E];
  T td, tx, ntd, ntx;
  float m, rs, nm, nrs;
  auto fetch = [&](long row) {
    const long rc = row < R ? row : R - 1;
    const T *pd = dy + rc * lddy, *px = x + rc * ldx;
    nm = mean[rc];
    nrs = rstd[rc];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      nd[e] = load_chunk(pd + at.start[e]);
      nx[e] = load_chunk(px + at.start[e]);
    }
    if (tails) {
      ntd = pd[at.has_tail ? at.tail : 0];
      ntx = px[at.has_tail ? at.tail : 0];
    }
  };
  fetch(r);
  int odd = 0;
  for (long b = (long)blockIdx.x * G; b < R; b += step, r += step, odd ^= 1) {
    const bool in = r < R;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    // what a lane does not own counts as zeros
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const bool own = in && (e < E - 1 || at.last);
      qd[e] = own ? nd[e] : zero;
      qx[e] = own ? nx[e] : zero;
    }
    float dt = 0.f, xt = 0.f;
    m = in ? nm : 0.f;
    rs = in ? nrs : 0.f;
    if (tails && in && at.has_tail) {
      dt = TT<T>::to_f(ntd);
      xt = (TT<T>::to_f(ntx) - m) * rs;
    }
    if (b + step < R) fetch(r + step);
    float s[2] = {dt * gt, dt * gt * xt};
    ab[E * VW] += dt;
    ag[E * VW] += dt * xt;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float d[VW], v[VW];
      if (WIDE) load_param<VW>(gamma, at.start[e], 1.f, gm[e]);
      unpack<T>(qd[e], d);
      unpack<T>(qx[e], v);
#pragma unroll
      for (int j = 0; j < VW; ++j) {
        const float t = d[j] * ((v[j] - m) * rs);
        if (WIDE) {
          v[j] = t;
        } else {
          ab[e * VW + j] += d[j];
          ag[e * VW + j] += t;
        }
        s[0] += d[j] * gm[e][j];
        s[1] += t * gm[e][j];
      }
      if (WIDE) {
#pragma unroll
        for (int h = 0; h < VW / 4; ++h) {
          float4 &wg = wide[0][e * VW / 4 + h][l], &wb = wide[WIDE][e * VW / 4 + h][l];
          float4 a = wg, b = wb;
          a.x += v[4 * h]; a.y += v[4 * h + 1]; a.z += v[4 * h + 2]; a.w += v[4 * h + 3];
          b.x += d[4 * h]; b.y += d[4 * h + 1]; b.z += d[4 * h + 2]; b.w += d[4 * h + 3];
          wg = a;
          wb = b;
        }
      }
      opaque(qd[e]);
      opaque(qx[e]);
      __builtin_amdgcn_sched_barrier(0);   // one chunk's values at a time in registers
    }
    row_sums<L>(s, sh[odd]);
    const float a = s[0] / fd, c = s[1] / fd;
    if (in) {
      T* dxr = dx + r * lddx;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float d[VW], v[VW];
        if (WIDE) load_param<VW>(gamma, at.start[e], 1.f, gm[e]);
        unpack<T>(qd[e], d);
        unpack<T>(qx[e], v);
#pragma unroll
        for (int j = 0; j < VW; ++j) d[j] = rs * (d[j] * gm[e][j] - a - (v[j] - m) * rs * c);
        if (e < E - 1 || at.last) store_chunk(dxr + at.start[e], pack<T>(d));
        __builtin_amdgcn_sched_barrier(0);
      }
      if (at.has_tail) dxr[at.tail] = TT<T>::from_f(rs * (dt * gt - a - xt * c));
    }
  }
  if (!po.part) return;
  float* og = po.part + (long)blockIdx.x * 2 * po.Dp;
  float* ob = og + po.Dp;
  if constexpr (L <= 64) {
    const int w = threadIdx.x >> 6, wl = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i <= E * VW; ++i) {
#pragma unroll
      for (int o = L; o < 64; o <<= 1) {
        ag[i] += __shfl_xor(ag[i], o);
        ab[i] += __shfl_xor(ab[i], o);
      }
      if (wl < L) {
        shp[w][i * 2 * L + wl] = ag[i];
        shp[w][(i * 2 + 1) * L + wl] = ab[i];
      }
    }
    __syncthreads();
    if (threadIdx.x >= L) return;
#pragma unroll
    for (int i = 0; i <= E * VW; ++i) {
      ag[i] = shp[0][i * 2 * L + l];
      ab[i] = shp[0][(i * 2 + 1) * L + l];
#pragma unroll
      for (int k = 1; k < NW; ++k) {
        ag[i] += shp[k][i * 2 * L + l];
        ab[i] += shp[k][(i * 2 + 1) * L + l];
      }
    }
  }
  if (WIDE)
#pragma unroll
    for (int i = 0; i < Q; ++i) {
      __builtin_memcpy(ag + 4 * i, &wide[0][i][l], 16);
      __builtin_memcpy(ab + 4 * i, &wide[WIDE][i][l], 16);
    }
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (e < E - 1 || at.last) {
      __builtin_memcpy(og + at.start[e], ag + e * VW, VW * 4);
      __builtin_memcpy(ob + at.start[e], ab + e * VW, VW * 4);
    }
  if (at.has_tail) {
    og[at.tail] = ag[E * VW];
    ob[at.tail] = ab[E * VW];
  }
}

// Columns of the partial rows added up in a fixed order: 8 lanes of 4 columns
// by 128 groups of rows a block (short chains of loads, and most of the time
// of this kernel is their latency), then the groups' sums by fours and the
// fours in order. One launch takes up to kSumCols columns from c0 on: its
// threads are counted in 32 bits, which 2^27 columns would pass.
constexpr int kSumCols = 1 << 26;
__global__ __launch_bounds__(1024) void ln_param_sum_kernel(const float* __restrict__ part, int nb, int D, int Dp,
                                                            int c0, float* __restrict__ dgamma,
                                                            float* __restrict__ dbeta) {
  __shared__ float sh[128][33], sh2[32][33];
  const int cl = threadIdx.x & 7, rg = threadIdx.x >> 3;
  const int c = c0 + blockIdx.x * 32 + cl * 4;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (c < Dp) {
    const float* p = part + (long)blockIdx.y * Dp + c;
#pragma unroll 4
    for (int b = rg; b < nb; b += 128) {
      const float4 v = *(const float4*)(p + (long)b * 2 * Dp);
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
  }
  sh[rg][cl * 4] = s.x; sh[rg][cl * 4 + 1] = s.y; sh[rg][cl * 4 + 2] = s.z; sh[rg][cl * 4 + 3] = s.w;
  __syncthreads();
  const int k = threadIdx.x & 31, g = threadIdx.x >> 5;
  sh2[g][k] = (sh[4 * g][k] + sh[4 * g + 1][k]) + (sh[4 * g + 2][k] + sh[4 * g + 3][k]);
  __syncthreads();
  const int col = c0 + blockIdx.x * 32 + k;
  float* o = blockIdx.y ? dbeta : dgamma;
  if (g == 0 && col < D && o) {
    float t = sh2[0][k];
    for (int i = 1; i < 32; ++i) t += sh2[i][k];
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
      const int a = c * VW;
      unpack<T>(load_chunk(xr + a), v);
      load_param<VW>(gamma, a, 1.f, gm);
      load_param<VW>(beta, a, 0.f, bt);
#pragma unroll
      for (int j = 0; j < VW; ++j) v[j] = (v[j] - m) * (rs * gm[j]) + bt[j];
      store_chunk(yr + a, pack<T>(v));
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
      const int at = c * VW;
      unpack<T>(load_chunk(dyr + at), g);
      unpack<T>(load_chunk(xr + at), v);
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
      const int at = c * VW;
      unpack<T>(load_chunk(dyr + at), g);
      unpack<T>(load_chunk(xr + at), v);
      load_param<VW>(gamma, at, 1.f, gm);
#pragma unroll
      for (int j = 0; j < VW; ++j) g[j] = rs * (g[j] * gm[j] - a - (v[j] - m) * rs * b);
      store_chunk(dxr + at, pack<T>(g));
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
  const int nch = D / vw;
  *E = 1;
  *L = D % vw ? 8 : 1;   // (a lane each for the tail)
  while (*L < 64 && *L < nch) *L *= 2;
  if (nch <= 64) return LN_TILE;
  for (int l = 64; l <= 1024; l *= l == 64 ? 4 : 2)
    if (nch <= l * max_e) {
      *L = l;
      *E = ceil_div(nch, l);
      // (32 columns a lane beside gamma and beta do not fit in a lane's 128
      // registers: 2000x32768 bf16 forward 91 us, as a long row 85)
      return l == 1024 && *E * vw > 24 ? LN_LONG : LN_TILE;
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

int ln_fwd_per_cu(int L) { return L > 256 ? 4096 / L : 16; }

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
    case 1024 * 8 + 4:
      if constexpr (TT<T>::VW == 4) return fwd_go<T, 1024, 4, 1>(R, s, a...);
    default: return -1;
  }
}

// Blocks of the backward pass, one partial row each.
int bwd_grid(LnPath path, int L, long R, int D) {
  if (path == LN_SHORT) return even_grid((R + 255) / 256, 2);
  if (path == LN_LONG) return (int)std::max(1l, std::min(R, 8l * plan_cus() / ceil_div(D, 256)));
  const int G = L > 256 ? 1 : 256 / L;
  return even_grid((R + G - 1) / G, L > 256 ? 1024 / L : L < 64 ? 3 : 2);
}

template <typename T, int L, int E, bool WIDE = false, typename... A>
int bwd_go(int grid, hipStream_t s, A... a) {
  hipLaunchKernelGGL((ln_bwd_kernel<T, L, E, WIDE>), dim3(grid), dim3(L > 256 ? L : 256), 0, s, a...);
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
      case 1024 * 8 + 2: return bwd_go<T, 1024, 2, true>(grid, s, a...);
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
      case 1024 * 8 + 3: return bwd_go<T, 1024, 3, true>(grid, s, a...);
      case 1024 * 8 + 4: return bwd_go<T, 1024, 4, true>(grid, s, a...);
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

// Calls whose parameter gradients blocks of their own add up, in place of a
// second launch that joins partial sums: dy and x are read twice, from cache,
// and a column's sum is a chain of R / 32 additions. (Calls one after the
// other on the same inputs: 64x512 fp32 6.6 us, with the second launch 9.1 to
// 10; 512x8192 bf16 13.6 and 23; 1024x4096 11.1 and 18; but 2048x1024 10.0 and
// 9.5 to 10.6, 4096x512 16.9 and 10.1.)
static bool ln_bwd_small(int prec, long R, int D) {
  return R <= 1024 && R * D * prec_bytes(prec) <= (8l << 20);
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
  // (dx in place of dy or x would be written while the column sums read them)
  const bool small = params && R > 0 && path == LN_TILE && L < 1024 && dx != dy && dx != x && ln_bwd_small(prec, R, D);
  const LnParamOut po{params && !small ? (float*)ws : nullptr, (D + 3) & ~3, grid, dgamma, dbeta};
  if (R > 0) {
    const int r = with_prec(prec, [&](auto tag) {
      using T = decltype(tag);
      const T *dyt = (const T*)dy, *xt = (const T*)x;
      T* dxt = (T*)dx;
      if (path == LN_TILE)
        return bwd_tile<T>(L, E, small ? grid + ceil_div(D, 32) : grid, s, dyt, xt, gamma, mean, rstd, dxt, po, R, D,
                           lddy, ldx, lddx);
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
  if (params && !small)
    for (int c0 = 0; c0 < po.Dp; c0 += kSumCols) {
      hipLaunchKernelGGL(ln_param_sum_kernel, dim3(ceil_div(std::min(po.Dp - c0, kSumCols), 32), 2), dim3(1024), 0, s,
                         (const float*)ws, grid, D, po.Dp, c0, dgamma, dbeta);
      const int r = ok();
      if (r) return r;
    }
  return 0;
}

}  // namespace rn18

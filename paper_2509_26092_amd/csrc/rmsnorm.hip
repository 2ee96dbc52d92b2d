// Dropout of rows with a residual's addition, and root-mean-square norm with
// both in the same pass, forward and backward.
//   m = keep / (1 - p),  h = res + m x (rounded to storage),
//   rstd = 1 / sqrt(sum h^2 / D + eps),  y = h rstd gamma
//   8 bits: a = max(max |y|, 1e-30), scale = a / 448, y8 = e4m3(y / scale)
//   xh = h rstd, g = dy gamma, dh = rstd (g - xh sum(g xh) / D) + dr,
//   dx = m dh, dgamma = sum over rows of dy xh
// The norm takes h as it is stored, which is what the backward pass sees.
// The mask is computed again from its counter wherever it is needed: it costs
// about 30 integer instructions for four elements and no memory.
//
// Bound by memory where rows are many, by the launch where they are few (64x512
// takes 3 us in each kernel). So a row is read once and written from registers,
// and the sum, the scaling and the residual's addition share that pass. HBM
// rates, of the 5.2 TB/s of a plain copy:
//   forward to 8 bits, bf16 16384x8192 with residual: 177 us for 940 MB
//   backward, bf16 50176x512 with dropout and residual: 51 us for 257 MB, and
//     5 us for the launch that joins dgamma's partial sums
//   dropout, fp16 16385x2050 with residual, rows of odd strides: 45 us for 202 MB
#include <math.h>

#include "philox.h"
#include "rows.h"

namespace rn18 {

namespace {

// ------------------------------------------------------------------ dropout
// A thread takes chunks of 16 bytes, a grid's width apart: their rows and
// places follow by addition from the first one's, without a division each.
template <typename T, bool RES>
__global__ __launch_bounds__(256) void dropout_rows_kernel(const T* x, const T* res, T* y, long R, int D, long ldx,
                                                           long ldres, long ldy, Dropout d) {
  constexpr int VW = TT<T>::VW;
  const DropKey key(d, D);
  const int per_row = (D + VW - 1) / VW;
  const long step = (long)gridDim.x * 256, first = blockIdx.x * 256l + threadIdx.x;
  const long step_r = step / per_row;
  const int step_c = (int)(step - step_r * per_row);
  long r = first / per_row;
  int c = (int)(first - r * per_row);
  while (r < R) {
    const int col = c * VW;
    const T *xr = x + r * ldx + col, *rr = res + r * ldres + col;
    T* yr = y + r * ldy + col;
    float v[VW];
    if (col + VW <= D) {
      unpack<T>(load_chunk(xr), v);
      key.apply<VW>(v, r, col);
      if (RES) {
        float w[VW];
        unpack<T>(load_chunk(rr), w);
#pragma unroll
        for (int j = 0; j < VW; ++j) v[j] += w[j];
      }
      store_chunk(yr, pack<T>(v));
    } else {
#pragma unroll
      for (int j = 0; j < VW; ++j) v[j] = col + j < D ? TT<T>::to_f(xr[j]) : 0.f;
      key.apply<VW>(v, r, col);
#pragma unroll
      for (int j = 0; j < VW; ++j)
        if (col + j < D) yr[j] = TT<T>::from_f(RES ? v[j] + TT<T>::to_f(rr[j]) : v[j]);
    }
    r += step_r;
    c += step_c;
    if (c >= per_row) {
      c -= per_row;
      ++r;
    }
  }
}

// ------------------------------------------------------------------ outputs
// e4m3 of y * inv for VW values, as bytes. (|y * inv| <= 448 (1 + 2^-22),
// which rounds to 448, the type's largest.)
__device__ inline uint32_t e4m3x4(const float* v) {
  int q = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], q, true);
}
template <int VW>
__device__ inline void store_q8(uint8_t* p, const float* v) {
  uint32_t q[VW / 4];
#pragma unroll
  for (int i = 0; i < VW / 4; ++i) q[i] = e4m3x4(v + 4 * i);
  __builtin_memcpy(p, q, VW);
}
__device__ inline uint8_t q8_one(float v) { return (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(v, v, 0, false); }
constexpr float kQ8Max = 448.f, kQ8Least = 1e-30f;
// The scale's numerator of a row (NaN stays).
__device__ inline float q8_amax(float a) { return a < kQ8Least ? kQ8Least : a; }

// h of one chunk as it is stored: the branch's chunk dropped, the residual's
// added, rounded.
template <typename T, bool DROP>
__device__ inline void chunk_h(float* v, const uint4& qx, const uint4& qr, bool res, const DropKey& key, long r,
                               int start, uint4& qh) {
  constexpr int VW = TT<T>::VW;
  unpack<T>(qx, v);
  if (DROP) key.apply<VW>(v, r, start);
  if (res) {
    float w[VW];
    unpack<T>(qr, w);
#pragma unroll
    for (int j = 0; j < VW; ++j) v[j] += w[j];
  }
  qh = pack<T>(v);
  unpack<T>(qh, v);
}
template <typename T, bool DROP>
__device__ inline T one_h(T x, T w, bool res, const DropKey& key, long r, int col) {
  float v = TT<T>::to_f(x);
  if (DROP) v = key.one(v, r, col);
  return TT<T>::from_f(res ? v + TT<T>::to_f(w) : v);
}

// ------------------------------------------------------------------ forward, rows in registers
// As in the layer norm: L lanes hold a row in E chunks, a block takes NT / L
// rows at a time, and the next rows are loaded while the current ones are
// worked on.
template <typename T, int L, int E, bool DROP, bool Q8>
__global__ __launch_bounds__(L > 256 ? L : 256) void rms_fwd_kernel(RmsFwd a, Dropout d) {
  constexpr int VW = TT<T>::VW, NT = L > 256 ? L : 256, G = NT / L;
  __shared__ float sh[2][L > 64 ? L / 64 : 1][1];
  const int l = threadIdx.x % L, g = L < NT ? threadIdx.x / L : 0, D = a.D;
  const Span<VW, L, E> at(l, D);
  const DropKey key(d, D);
  const bool tails = D % VW != 0, res = a.res != nullptr;
  const T *x = (const T*)a.x, *rs_ = (const T*)a.res;
  float gm[E][VW], gt = 1.f;
#pragma unroll
  for (int e = 0; e < E; ++e) load_param<VW>(a.gamma, at.start[e], 1.f, gm[e]);
  if (at.has_tail && a.gamma) gt = a.gamma[at.tail];
  const float fd = (float)D;
  const long step = (long)gridDim.x * G;
  long r = (long)blockIdx.x * G + g;
  uint4 qx[E], qr[E];
  T tx, tr;
  auto fetch = [&](long row) {
    const long rc = row < a.R ? row : a.R - 1;
    const T *px = x + rc * a.ldx, *pr = rs_ + rc * a.ldres;
#pragma unroll
    for (int e = 0; e < E; ++e) qx[e] = load_chunk(px + at.start[e]);
    if (res)
#pragma unroll
      for (int e = 0; e < E; ++e) qr[e] = load_chunk(pr + at.start[e]);
    if (tails) {
      tx = px[at.has_tail ? at.tail : 0];
      if (res) tr = pr[at.has_tail ? at.tail : 0];
    }
  };
  fetch(r);
  int odd = 0;
  for (long b = (long)blockIdx.x * G; b < a.R; b += step, r += step, odd ^= 1) {   // the same count for every thread
    const bool in = r < a.R;
    float v[E][VW], t = 0.f, s[1], w = 0.f;
    T th{};
    uint4 qh[E];
    T* hr = (T*)a.h + r * a.ldh;
    s[0] = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      chunk_h<T, DROP>(v[e], qx[e], qr[e], res, key, r, at.start[e], qh[e]);
#pragma unroll
      for (int j = 0; j < VW; ++j) (e < E - 1 ? s[0] : w) += v[e][j] * v[e][j];
    }
    if (at.last) s[0] += w;
    if (at.has_tail) {
      th = one_h<T, DROP>(tx, tr, res, key, r, at.tail);
      t = TT<T>::to_f(th);
      s[0] += t * t;
    }
    if (b + step < a.R) fetch(r + step);
    if (a.h && in) {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (e < E - 1 || at.last) store_chunk(hr + at.start[e], qh[e]);
      if (at.has_tail) hr[at.tail] = th;
    }
    row_sums<L>(s, sh[Q8 ? 0 : odd]);
    const float rs = 1.0f / sqrtf(s[0] / fd + a.eps);
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int j = 0; j < VW; ++j) v[e][j] = v[e][j] * rs * gm[e][j];
    t = t * rs * gt;
    if (Q8) {
      float m[1] = {at.has_tail ? fabsf(t) : 0.f};
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (e < E - 1 || at.last)
#pragma unroll
          for (int j = 0; j < VW; ++j) m[0] = max2(m[0], fabsf(v[e][j]));
      row_red<L>(m, sh[1], Max());
      const float amax = q8_amax(m[0]), inv = kQ8Max / amax;
      if (in) {
        uint8_t* yr = (uint8_t*)a.y + r * a.ldy;
#pragma unroll
        for (int e = 0; e < E; ++e) {
#pragma unroll
          for (int j = 0; j < VW; ++j) v[e][j] *= inv;
          if (e < E - 1 || at.last) store_q8<VW>(yr + at.start[e], v[e]);
        }
        if (at.has_tail) yr[at.tail] = q8_one(t * inv);
        if (l == 0) a.scale[r] = amax / kQ8Max;
      }
    } else if (in) {
      T* yr = (T*)a.y + r * a.ldy;
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (e < E - 1 || at.last) store_chunk(yr + at.start[e], pack<T>(v[e]));
      if (at.has_tail) yr[at.tail] = TT<T>::from_f(t);
    }
    if (l == 0 && in && a.rstd) a.rstd[r] = rs;
  }
}

// Rows shorter than a chunk: a thread per row.
template <typename T, bool DROP, bool Q8>
__global__ __launch_bounds__(256) void rms_fwd_short_kernel(RmsFwd a, Dropout d) {
  constexpr int VW = TT<T>::VW;
  const DropKey key(d, a.D);
  for (long r = blockIdx.x * 256l + threadIdx.x; r < a.R; r += gridDim.x * 256l) {
    float v[VW], s = 0.f, m = 0.f;
#pragma unroll
    for (int j = 0; j < VW; ++j) v[j] = j < a.D ? TT<T>::to_f(((const T*)a.x)[r * a.ldx + j]) : 0.f;
    if (DROP) key.apply<VW>(v, r, 0);
#pragma unroll
    for (int j = 0; j < VW; ++j) {
      if (j >= a.D) continue;
      if (a.res) v[j] += TT<T>::to_f(((const T*)a.res)[r * a.ldres + j]);
      const T h = TT<T>::from_f(v[j]);
      if (a.h) ((T*)a.h)[r * a.ldh + j] = h;
      v[j] = TT<T>::to_f(h);
      s += v[j] * v[j];
    }
    const float rs = 1.0f / sqrtf(s / (float)a.D + a.eps);
#pragma unroll
    for (int j = 0; j < VW; ++j) {
      if (j >= a.D) continue;
      v[j] = v[j] * rs * (a.gamma ? a.gamma[j] : 1.f);
      m = max2(m, fabsf(v[j]));
    }
    const float amax = q8_amax(m), inv = kQ8Max / amax;
#pragma unroll
    for (int j = 0; j < VW; ++j) {
      if (j >= a.D) continue;
      if (Q8) ((uint8_t*)a.y)[r * a.ldy + j] = q8_one(v[j] * inv);
      else ((T*)a.y)[r * a.ldy + j] = TT<T>::from_f(v[j]);
    }
    if (Q8) a.scale[r] = amax / kQ8Max;
    if (a.rstd) a.rstd[r] = rs;
  }
}

// Rows beyond a block's registers: h is made and stored in one pass (where h
// is x itself, nothing is stored) and read again for y, and once more for the
// largest y where that is wanted. A thread reads what it has written itself.
// The chunks' sums are added up in 64 bits: up to 2^20 of them are a thread's, and
// in fp32 equal elements' roundings all go one way (1.4e-4 of y at 2^24 elements).
template <typename T, bool DROP, bool Q8>
__global__ __launch_bounds__(1024) void rms_fwd_long_kernel(RmsFwd a, Dropout d) {
  constexpr int VW = TT<T>::VW;
  __shared__ float sh[16], shm[2][16][1];
  const DropKey key(d, a.D);
  const int D = a.D, nch = D / VW, tail = nch * VW + (int)threadIdx.x;   // whole chunks, and one element each of the rest
  const bool has_tail = tail < D, res = a.res != nullptr;
  int odd = 0;
  for (long r = blockIdx.x; r < a.R; r += gridDim.x, odd ^= 1) {
    const T *xr = (const T*)a.x + r * a.ldx, *rr = res ? (const T*)a.res + r * a.ldres : xr;
    T* hr = (T*)a.h + r * a.ldh;
    float t = 0.f, v[VW], gm[VW];
    double s = 0.;
    uint4 qh;
    if (has_tail) {
      const T th = one_h<T, DROP>(xr[tail], rr[tail], res, key, r, tail);
      if (a.h) hr[tail] = th;
      t = TT<T>::to_f(th);
      s = t * t;
    }
    for (int c = threadIdx.x; c < nch; c += 1024) {
      chunk_h<T, DROP>(v, load_chunk(xr + c * VW), load_chunk(rr + c * VW), res, key, r, c * VW, qh);
      if (a.h) store_chunk(hr + c * VW, qh);
      float u = 0.f;
#pragma unroll
      for (int j = 0; j < VW; ++j) u += v[j] * v[j];
      s += u;
    }
    const float rs = 1.0f / sqrtf(block_sum1024((float)s, sh) / (float)D + a.eps);
    const T* src = a.h ? hr : xr;
    auto y_of = [&](int c) {
      unpack<T>(load_chunk(src + c * VW), v);
      load_param<VW>(a.gamma, c * VW, 1.f, gm);
#pragma unroll
      for (int j = 0; j < VW; ++j) v[j] = v[j] * rs * gm[j];
    };
    t = t * rs * (has_tail && a.gamma ? a.gamma[tail] : 1.f);
    if (Q8) {
      float m[1] = {fabsf(t)};
      for (int c = threadIdx.x; c < nch; c += 1024) {
        y_of(c);
#pragma unroll
        for (int j = 0; j < VW; ++j) m[0] = max2(m[0], fabsf(v[j]));
      }
      row_red<1024>(m, shm[odd], Max());
      const float amax = q8_amax(m[0]), inv = kQ8Max / amax;
      uint8_t* yr = (uint8_t*)a.y + r * a.ldy;
      for (int c = threadIdx.x; c < nch; c += 1024) {
        y_of(c);
#pragma unroll
        for (int j = 0; j < VW; ++j) v[j] *= inv;
        store_q8<VW>(yr + c * VW, v);
      }
      if (has_tail) yr[tail] = q8_one(t * inv);
      if (threadIdx.x == 0) a.scale[r] = amax / kQ8Max;
    } else {
      T* yr = (T*)a.y + r * a.ldy;
      for (int c = threadIdx.x; c < nch; c += 1024) {
        y_of(c);
        store_chunk(yr + c * VW, pack<T>(v));
      }
      if (has_tail) yr[tail] = TT<T>::from_f(t);
    }
    if (threadIdx.x == 0 && a.rstd) a.rstd[r] = rs;
  }
}

// ------------------------------------------------------------------ backward, rows in registers
// The sums of dgamma of a lane's columns stay in registers over all rows of
// the block, are joined over its row groups, and written as one partial row a
// block: part[block][Dp] (Dp = D rounded up to 4).
// Small calls take one launch instead: dgamma needs no row sums, so blocks of
// their own (from row_blocks on) add up 32 columns each over all rows: 8 lanes
// of 4 columns by 32 groups of rows, the groups' sums by fours, the fours in order.
struct RmsParamOut {
  float* part;      // NULL: dgamma is not wanted, or blocks of their own write it
  int Dp, row_blocks;
};
template <typename T>
__device__ inline void rms_columns(const RmsBwd& a, int c0) {
  __shared__ float sh[32][33], sh2[8][33];
  const int t = threadIdx.x, cl = (t & 7) * 4, rg = t >> 3, c = c0 + cl;
  float s[4] = {};
  if (t < 256 && c < a.D) {
#pragma unroll 4
    for (long r = rg; r < a.R; r += 32) {
      const float rs = a.rstd[r];
      const T *pd = (const T*)a.dy + r * a.lddy + c, *ph = (const T*)a.h + r * a.ldh + c;
      T qd[4] = {}, qh[4] = {};
      if (c + 4 <= a.D) {
        __builtin_memcpy(qd, pd, 4 * sizeof(T));
        __builtin_memcpy(qh, ph, 4 * sizeof(T));
      } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
          if (j < a.D - c) {
            qd[j] = pd[j];
            qh[j] = ph[j];
          }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] += TT<T>::to_f(qd[j]) * (TT<T>::to_f(qh[j]) * rs);
    }
  }
  if (t < 256)
#pragma unroll
    for (int j = 0; j < 4; ++j) sh[rg][cl + j] = s[j];
  __syncthreads();
  const int k = t & 31, q = t >> 5;
  if (t < 256) sh2[q][k] = (sh[4 * q][k] + sh[4 * q + 1][k]) + (sh[4 * q + 2][k] + sh[4 * q + 3][k]);
  __syncthreads();
  if (t < 32 && c0 + k < a.D) {
    float v = sh2[0][k];
#pragma unroll
    for (int i = 1; i < 8; ++i) v += sh2[i][k];
    a.dgamma[c0 + k] = v;
  }
}

template <typename T, int L, int E, bool DROP>
__global__ __launch_bounds__(L > 256 ? L : 256) void rms_bwd_kernel(RmsBwd a, Dropout d, RmsParamOut po) {
  constexpr int VW = TT<T>::VW, NT = L > 256 ? L : 256, G = NT / L, NW = NT / 64, NV = E * VW + 1;
  if ((int)blockIdx.x >= po.row_blocks) {
    rms_columns<T>(a, ((int)blockIdx.x - po.row_blocks) * 32);
    return;
  }
  __shared__ float shp[L > 64 ? 1 : NW][L > 64 ? 1 : L * NV];
  __shared__ float sh[2][L > 64 ? L / 64 : 1][1];
  const int l = threadIdx.x % L, g = L < NT ? threadIdx.x / L : 0, D = a.D;
  const Span<VW, L, E> at(l, D);
  const DropKey key(d, D);
  const bool tails = D % VW != 0, more = a.dr != nullptr;
  float gm[E][VW], ag[NV], gt = 1.f;
#pragma unroll
  for (int e = 0; e < E; ++e) load_param<VW>(a.gamma, at.start[e], 1.f, gm[e]);
  if (at.has_tail && a.gamma) gt = a.gamma[at.tail];
#pragma unroll
  for (int i = 0; i < NV; ++i) ag[i] = 0.f;
  const float fd = (float)D;
  const long step = (long)po.row_blocks * G;
  long r = (long)blockIdx.x * G + g;
  uint4 nd[E], nh[E], nr[E];
  T ntd, nth, ntr;
  float nrs;
  auto fetch = [&](long row) {
    const long rc = row < a.R ? row : a.R - 1;
    const T *pd = (const T*)a.dy + rc * a.lddy, *ph = (const T*)a.h + rc * a.ldh, *pr = (const T*)a.dr + rc * a.lddr;
    nrs = a.rstd[rc];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      nd[e] = load_chunk(pd + at.start[e]);
      nh[e] = load_chunk(ph + at.start[e]);
      if (more) nr[e] = load_chunk(pr + at.start[e]);
    }
    if (tails) {
      ntd = pd[at.has_tail ? at.tail : 0];
      nth = ph[at.has_tail ? at.tail : 0];
      if (more) ntr = pr[at.has_tail ? at.tail : 0];
    }
  };
  fetch(r);
  int odd = 0;
  for (long b = (long)blockIdx.x * G; b < a.R; b += step, r += step, odd ^= 1) {
    const bool in = r < a.R;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    uint4 qr[E];
    float dv[E][VW], xh[E][VW], dt = 0.f, xt = 0.f;
    const float rs = in ? nrs : 0.f;
    // what a lane does not own counts as zeros
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const bool own = in && (e < E - 1 || at.last);
      unpack<T>(own ? nd[e] : zero, dv[e]);
      unpack<T>(own ? nh[e] : zero, xh[e]);
      qr[e] = nr[e];
    }
    const T tr = ntr;
    if (tails && in && at.has_tail) {
      dt = TT<T>::to_f(ntd);
      xt = TT<T>::to_f(nth) * rs;
    }
    if (b + step < a.R) fetch(r + step);
    float s[1] = {dt * gt * xt};
    ag[NV - 1] += dt * xt;
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int j = 0; j < VW; ++j) {
        xh[e][j] *= rs;
        const float t = dv[e][j] * xh[e][j];
        ag[e * VW + j] += t;
        s[0] += t * gm[e][j];
      }
    row_sums<L>(s, sh[odd]);
    const float c = s[0] / fd;
    if (in) {
      T *hr = (T*)a.dh + r * a.lddh, *xr = (T*)a.dx + r * a.lddx;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float w[VW] = {};
        if (more) unpack<T>(qr[e], w);
#pragma unroll
        for (int j = 0; j < VW; ++j) w[j] += rs * (dv[e][j] * gm[e][j] - xh[e][j] * c);
        const bool own = e < E - 1 || at.last;
        if (a.dh && own) store_chunk(hr + at.start[e], pack<T>(w));
        if (a.dx && own) {
          if (DROP) key.apply<VW>(w, r, at.start[e]);
          store_chunk(xr + at.start[e], pack<T>(w));
        }
      }
      if (at.has_tail) {
        const float w = rs * (dt * gt - xt * c) + (more ? TT<T>::to_f(tr) : 0.f);
        if (a.dh) hr[at.tail] = TT<T>::from_f(w);
        if (a.dx) xr[at.tail] = TT<T>::from_f(DROP ? key.one(w, r, at.tail) : w);
      }
    }
  }
  if (!po.part) return;
  float* og = po.part + (long)blockIdx.x * po.Dp;
  if constexpr (L <= 64) {
    const int w = threadIdx.x >> 6, wl = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int o = L; o < 64; o <<= 1) ag[i] += __shfl_xor(ag[i], o);
      if (wl < L) shp[w][i * L + wl] = ag[i];
    }
    __syncthreads();
    if (threadIdx.x >= L) return;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      ag[i] = shp[0][i * L + l];
#pragma unroll
      for (int k = 1; k < NW; ++k) ag[i] += shp[k][i * L + l];
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (e < E - 1 || at.last) __builtin_memcpy(og + at.start[e], ag + e * VW, VW * 4);
  if (at.has_tail) og[at.tail] = ag[NV - 1];
}

template <typename T, bool DROP>
__global__ __launch_bounds__(256) void rms_bwd_short_kernel(RmsBwd a, Dropout d, float* part, int Dp) {
  constexpr int VW = TT<T>::VW;
  __shared__ float sh[4][VW];
  const DropKey key(d, a.D);
  float ag[VW] = {};
  for (long r = blockIdx.x * 256l + threadIdx.x; r < a.R; r += gridDim.x * 256l) {
    const float rs = a.rstd[r];
    float g[VW], xh[VW], w[VW], c = 0.f;
#pragma unroll
    for (int j = 0; j < VW; ++j) {
      const bool in = j < a.D;
      const float dy = in ? TT<T>::to_f(((const T*)a.dy)[r * a.lddy + j]) : 0.f;
      xh[j] = in ? TT<T>::to_f(((const T*)a.h)[r * a.ldh + j]) * rs : 0.f;
      g[j] = in && a.gamma ? dy * a.gamma[j] : dy;
      ag[j] += dy * xh[j];
      c += g[j] * xh[j];
    }
    c /= (float)a.D;
#pragma unroll
    for (int j = 0; j < VW; ++j) {
      w[j] = rs * (g[j] - xh[j] * c);
      if (a.dr && j < a.D) w[j] += TT<T>::to_f(((const T*)a.dr)[r * a.lddr + j]);
      if (a.dh && j < a.D) ((T*)a.dh)[r * a.lddh + j] = TT<T>::from_f(w[j]);
    }
    if (a.dx) {
      if (DROP) key.apply<VW>(w, r, 0);
#pragma unroll
      for (int j = 0; j < VW; ++j)
        if (j < a.D) ((T*)a.dx)[r * a.lddx + j] = TT<T>::from_f(w[j]);
    }
  }
  if (!part) return;
#pragma unroll
  for (int j = 0; j < VW; ++j) {
    ag[j] = group_sum<64>(ag[j]);
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6][j] = ag[j];
  }
  __syncthreads();
  const int k = threadIdx.x;
  if (k < VW && k < a.D) part[(long)blockIdx.x * Dp + k] = ((sh[0][k] + sh[1][k]) + sh[2][k]) + sh[3][k];
}

// ------------------------------------------------------------------ backward, rows beyond a block's registers
template <typename T, bool DROP>
__global__ __launch_bounds__(1024) void rms_bwd_long_kernel(RmsBwd a, Dropout d) {
  constexpr int VW = TT<T>::VW;
  __shared__ float sh[16];
  const DropKey key(d, a.D);
  const int D = a.D, nch = D / VW, tail = nch * VW + (int)threadIdx.x;
  const bool has_tail = tail < D;
  for (long r = blockIdx.x; r < a.R; r += gridDim.x) {
    const T *dyr = (const T*)a.dy + r * a.lddy, *hr = (const T*)a.h + r * a.ldh;
    const T* drr = a.dr ? (const T*)a.dr + r * a.lddr : nullptr;
    T *dhr = a.dh ? (T*)a.dh + r * a.lddh : nullptr, *dxr = a.dx ? (T*)a.dx + r * a.lddx : nullptr;
    const float rs = a.rstd[r];
    float tg = 0.f, tx = 0.f;
    double sum = 0.;   // (in 64 bits as in the forward pass)
    if (has_tail) {
      tg = TT<T>::to_f(dyr[tail]) * (a.gamma ? a.gamma[tail] : 1.f);
      tx = TT<T>::to_f(hr[tail]) * rs;
      sum = tg * tx;
    }
    float g[VW], v[VW], gm[VW];
    for (int c = threadIdx.x; c < nch; c += 1024) {
      unpack<T>(load_chunk(dyr + c * VW), g);
      unpack<T>(load_chunk(hr + c * VW), v);
      load_param<VW>(a.gamma, c * VW, 1.f, gm);
      float u = 0.f;
#pragma unroll
      for (int j = 0; j < VW; ++j) u += g[j] * gm[j] * (v[j] * rs);
      sum += u;
    }
    const float s = block_sum1024((float)sum, sh) / (float)D;
    if (has_tail) {
      const float w = rs * (tg - tx * s) + (drr ? TT<T>::to_f(drr[tail]) : 0.f);
      if (dhr) dhr[tail] = TT<T>::from_f(w);
      if (dxr) dxr[tail] = TT<T>::from_f(DROP ? key.one(w, r, tail) : w);
    }
    for (int c = threadIdx.x; c < nch; c += 1024) {
      float w[VW] = {};
      unpack<T>(load_chunk(dyr + c * VW), g);
      unpack<T>(load_chunk(hr + c * VW), v);
      if (drr) unpack<T>(load_chunk(drr + c * VW), w);
      load_param<VW>(a.gamma, c * VW, 1.f, gm);
#pragma unroll
      for (int j = 0; j < VW; ++j) w[j] += rs * (g[j] * gm[j] - v[j] * rs * s);
      if (dhr) store_chunk(dhr + c * VW, pack<T>(w));
      if (dxr) {
        if (DROP) key.apply<VW>(w, r, c * VW);
        store_chunk(dxr + c * VW, pack<T>(w));
      }
    }
  }
}

// Its parameter gradient: block (columns of 256, range of rows) writes one
// partial row, added up in 64 bits (the longest rows have one block to a column).
template <typename T>
__global__ __launch_bounds__(256) void rms_param_long_kernel(RmsBwd a, float* part, int Dp) {
  const long c = (long)blockIdx.x * 256 + threadIdx.x;
  if (c >= a.D) return;
  double s = 0.;
  for (long r = blockIdx.y; r < a.R; r += gridDim.y)
    s += TT<T>::to_f(((const T*)a.dy)[r * a.lddy + c]) * (TT<T>::to_f(((const T*)a.h)[r * a.ldh + c]) * a.rstd[r]);
  part[(long)blockIdx.y * Dp + c] = (float)s;
}

// ------------------------------------------------------------------ choice of kernel
template <typename T, int L, int E, bool DROP, bool Q8>
int fwd_go(const RmsFwd& a, const Dropout& d, hipStream_t s) {
  constexpr int NT = L > 256 ? L : 256, G = NT / L;
  hipLaunchKernelGGL((rms_fwd_kernel<T, L, E, DROP, Q8>), dim3(even_grid((a.R + G - 1) / G, L > 256 ? 4096 / L : 16)),
                     dim3(NT), 0, s, a, d);
  return launched();
}

template <typename T, bool DROP, bool Q8>
int fwd_path(RowPath path, int L, int E, const RmsFwd& a, const Dropout& d, hipStream_t s) {
  if (path == ROW_SHORT) {
    hipLaunchKernelGGL((rms_fwd_short_kernel<T, DROP, Q8>), dim3(row_grid((a.R + 255) / 256)), dim3(256), 0, s, a, d);
    return launched();
  }
  if (path == ROW_LONG) {
    hipLaunchKernelGGL((rms_fwd_long_kernel<T, DROP, Q8>), dim3(row_grid(a.R)), dim3(1024), 0, s, a, d);
    return launched();
  }
  switch (L * 8 + E) {
    case 1 * 8 + 1: return fwd_go<T, 1, 1, DROP, Q8>(a, d, s);
    case 2 * 8 + 1: return fwd_go<T, 2, 1, DROP, Q8>(a, d, s);
    case 4 * 8 + 1: return fwd_go<T, 4, 1, DROP, Q8>(a, d, s);
    case 8 * 8 + 1: return fwd_go<T, 8, 1, DROP, Q8>(a, d, s);
    case 16 * 8 + 1: return fwd_go<T, 16, 1, DROP, Q8>(a, d, s);
    case 32 * 8 + 1: return fwd_go<T, 32, 1, DROP, Q8>(a, d, s);
    case 64 * 8 + 1: return fwd_go<T, 64, 1, DROP, Q8>(a, d, s);
    case 64 * 8 + 2: return fwd_go<T, 64, 2, DROP, Q8>(a, d, s);
    case 256 * 8 + 1: return fwd_go<T, 256, 1, DROP, Q8>(a, d, s);
    case 256 * 8 + 2: return fwd_go<T, 256, 2, DROP, Q8>(a, d, s);
    case 512 * 8 + 2: return fwd_go<T, 512, 2, DROP, Q8>(a, d, s);
    case 1024 * 8 + 2: return fwd_go<T, 1024, 2, DROP, Q8>(a, d, s);
    default: break;
  }
  if constexpr (TT<T>::VW == 4) switch (L * 8 + E) {
      case 64 * 8 + 3: return fwd_go<T, 64, 3, DROP, Q8>(a, d, s);
      case 64 * 8 + 4: return fwd_go<T, 64, 4, DROP, Q8>(a, d, s);
      case 256 * 8 + 3: return fwd_go<T, 256, 3, DROP, Q8>(a, d, s);
      case 256 * 8 + 4: return fwd_go<T, 256, 4, DROP, Q8>(a, d, s);
      case 512 * 8 + 3: return fwd_go<T, 512, 3, DROP, Q8>(a, d, s);
      case 512 * 8 + 4: return fwd_go<T, 512, 4, DROP, Q8>(a, d, s);
      case 1024 * 8 + 3: return fwd_go<T, 1024, 3, DROP, Q8>(a, d, s);
      case 1024 * 8 + 4: return fwd_go<T, 1024, 4, DROP, Q8>(a, d, s);
      default: break;
    }
  return -1;
}
int rms_max_e(int prec) { return 16 / prec_vw(prec); }   // 16 columns a lane

int bwd_grid(RowPath path, int L, long R, int D) {
  if (path == ROW_SHORT) return even_grid((R + 255) / 256, 2);
  if (path == ROW_LONG) return (int)std::max(1l, std::min(R, 8l * plan_cus() / ceil_div(D, 256)));
  const int G = L > 256 ? 1 : 256 / L;
  return even_grid((R + G - 1) / G, L > 256 ? 1024 / L : L < 64 ? 3 : 2);
}

template <typename T, bool DROP>
int bwd_path(RowPath path, int L, int E, int grid, bool small, const RmsBwd& a, const Dropout& d, float* part,
             hipStream_t s) {
  const int Dp = (a.D + 3) & ~3, blocks = small ? grid + ceil_div(a.D, 32) : grid;
  const RmsParamOut po{small ? nullptr : part, Dp, grid};
  if (path == ROW_SHORT) {
    hipLaunchKernelGGL((rms_bwd_short_kernel<T, DROP>), dim3(grid), dim3(256), 0, s, a, d, part, Dp);
    return launched();
  }
  if (path == ROW_LONG) {
    if (part) {   // before dh and dx, which may replace dy, h or dr
      hipLaunchKernelGGL(rms_param_long_kernel<T>, dim3(ceil_div(a.D, 256), grid), dim3(256), 0, s, a, part, Dp);
      const int r = launched();
      if (r) return r;
    }
    hipLaunchKernelGGL((rms_bwd_long_kernel<T, DROP>), dim3(row_grid(a.R)), dim3(1024), 0, s, a, d);
    return launched();
  }
#define GO(L_, E_)                                                                                            \
  case L_ * 8 + E_:                                                                                           \
    hipLaunchKernelGGL((rms_bwd_kernel<T, L_, E_, DROP>), dim3(blocks), dim3(L_ > 256 ? L_ : 256), 0, s, a, d, po); \
    return launched();
  switch (L * 8 + E) {
    GO(1, 1) GO(2, 1) GO(4, 1) GO(8, 1) GO(16, 1) GO(32, 1) GO(64, 1) GO(64, 2) GO(256, 1) GO(256, 2) GO(512, 2)
    GO(1024, 2)
    default: break;
  }
  if constexpr (TT<T>::VW == 4) switch (L * 8 + E) {
      GO(64, 3) GO(64, 4) GO(256, 3) GO(256, 4) GO(512, 3) GO(512, 4) GO(1024, 3) GO(1024, 4)
      default: break;
    }
#undef GO
  return -1;
}

}  // namespace

int dropout_rows_launch(int prec, const void* x, const void* res, void* y, long R, int D, long ldx, long ldres,
                        long ldy, const Dropout& d, hipStream_t s) {
  if (R <= 0) return 0;
  return with_prec(prec, [&](auto tag) {
    using T = decltype(tag);
    const long units = (R * ((D + TT<T>::VW - 1l) / TT<T>::VW) + 255) / 256;
    const dim3 grid(even_grid(units, 16));
    if (res)
      hipLaunchKernelGGL((dropout_rows_kernel<T, true>), grid, dim3(256), 0, s, (const T*)x, (const T*)res, (T*)y, R, D,
                         ldx, ldres, ldy, d);
    else
      hipLaunchKernelGGL((dropout_rows_kernel<T, false>), grid, dim3(256), 0, s, (const T*)x, (const T*)nullptr, (T*)y,
                         R, D, ldx, 0l, ldy, d);
    return launched();
  });
}

int rmsnorm_fwd_launch(int prec, const RmsFwd& a, const Dropout* d, hipStream_t s) {
  if (a.R <= 0) return 0;
  int L = 0, E = 0;
  const RowPath path = row_tile(prec, a.D, rms_max_e(prec), &L, &E);
  const Dropout none{};
  return with_prec(prec, [&](auto tag) {
    using T = decltype(tag);
    if (d) return a.scale ? fwd_path<T, true, true>(path, L, E, a, *d, s) : fwd_path<T, true, false>(path, L, E, a, *d, s);
    return a.scale ? fwd_path<T, false, true>(path, L, E, a, none, s) : fwd_path<T, false, false>(path, L, E, a, none, s);
  });
}

size_t rmsnorm_bwd_workspace(int prec, long R, int D) {
  if (R <= 0) return 0;
  int L = 0, E = 0;
  const RowPath path = row_tile(prec, D, rms_max_e(prec), &L, &E);
  return (size_t)bwd_grid(path, L, R, D) * ((D + 3) & ~3) * 4;
}

// Calls whose dgamma blocks of their own add up, in place of a second launch that
// joins partial sums; dy and h are read twice, from cache, and a column's sum is
// a chain of R / 32 additions. A call so and with the second launch (us, its own
// 3 to 5 among them): fp32 64x512 7.4 and 10.4, 1024x2048 (8 MB) 11.9 and 12.3,
// bf16 1024x4096 (8 MB) 13.6 and 15.6; beyond the rule fp32 1024x4096 19.0 and
// 17.2, 2048x512 13.6 and 10.6, bf16 512x16384 36.3 and 32.8.
static bool rms_bwd_small(int prec, long R, int D) {
  return R <= 1024 && R * D * prec_bytes(prec) <= (8l << 20);
}

int rmsnorm_bwd_launch(int prec, const RmsBwd& a, const Dropout* d, void* ws, hipStream_t s) {
  int L = 0, E = 0, grid = 0;
  bool small = false;
  if (a.R > 0) {
    const RowPath path = row_tile(prec, a.D, rms_max_e(prec), &L, &E);
    grid = bwd_grid(path, L, a.R, a.D);
    float* part = a.dgamma ? (float*)ws : nullptr;
    // (dh or dx in place of dy or h would be written while the column sums read them)
    auto apart = [&](const void* p) { return !p || (p != a.dy && p != a.h); };
    small = part && path == ROW_TILE && apart(a.dh) && apart(a.dx) && rms_bwd_small(prec, a.R, a.D);
    const Dropout none{};
    const int r = with_prec(prec, [&](auto tag) {
      using T = decltype(tag);
      return d ? bwd_path<T, true>(path, L, E, grid, small, a, *d, part, s)
               : bwd_path<T, false>(path, L, E, grid, small, a, none, part, s);
    });
    if (r) return r;
  }
  return a.dgamma && !small ? column_sums_launch((const float*)ws, grid, a.D, 1, a.dgamma, nullptr, s) : 0;
}

}  // namespace rn18

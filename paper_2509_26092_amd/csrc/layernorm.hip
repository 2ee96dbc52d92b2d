// Layer norm over the channels of a row, forward and backward, and the
// reduction of the gradients of its scale and shift.
//   y = (x - mean) rstd gamma + beta, mean = sum x / D,
//   rstd = 1 / sqrt(sum (x - mean)^2 / D + eps)
//   g = dy gamma, xh = (x - mean) rstd,
//   dx = rstd (g - sum g / D - xh sum(g xh) / D),
//   dgamma = sum over rows of dy xh, dbeta = sum over rows of dy
#include <math.h>

#include "kernels.h"

namespace rn18 {

namespace {

inline int ok() { return hipGetLastError() == hipSuccess ? 0 : -4; }

int row_grid(long R) { return (int)(R < 65536 ? R : 65536); }

// Sum over the 256 threads of a block; every thread gets it.
__device__ inline float block_sum(float v, float* sh) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  __syncthreads();   // earlier readers of sh are done
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  return (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

template <typename T>
__global__ __launch_bounds__(256) void ln_fwd_kernel(const T* x, const float* __restrict__ gamma,
                                                     const float* __restrict__ beta, T* y, float* __restrict__ mean,
                                                     float* __restrict__ rstd, long R, int D, long ldx, long ldy,
                                                     float eps) {
  __shared__ float sh[4];
  for (long r = blockIdx.x; r < R; r += gridDim.x) {
    const T* xr = x + r * ldx;
    T* yr = y + r * ldy;
    float s = 0.f;
    for (int c = threadIdx.x; c < D; c += 256) s += TT<T>::to_f(xr[c]);
    const float m = block_sum(s, sh) / (float)D;
    s = 0.f;
    for (int c = threadIdx.x; c < D; c += 256) {
      const float d = TT<T>::to_f(xr[c]) - m;
      s += d * d;
    }
    const float rs = 1.0f / sqrtf(block_sum(s, sh) / (float)D + eps);
    for (int c = threadIdx.x; c < D; c += 256) {
      const float v = (TT<T>::to_f(xr[c]) - m) * rs * (gamma ? gamma[c] : 1.f) + (beta ? beta[c] : 0.f);
      yr[c] = TT<T>::from_f(v);
    }
    if (threadIdx.x == 0) {
      if (mean) mean[r] = m;
      if (rstd) rstd[r] = rs;
    }
  }
}

template <typename T>
__global__ __launch_bounds__(256) void ln_bwd_kernel(const T* dy, const T* x, const float* __restrict__ gamma,
                                                     const float* __restrict__ mean, const float* __restrict__ rstd,
                                                     T* dx, long R, int D, long lddy, long ldx, long lddx) {
  __shared__ float sh[4];
  for (long r = blockIdx.x; r < R; r += gridDim.x) {
    const T* dyr = dy + r * lddy;
    const T* xr = x + r * ldx;
    T* dxr = dx + r * lddx;
    const float m = mean[r], rs = rstd[r];
    float a = 0.f, b = 0.f;
    for (int c = threadIdx.x; c < D; c += 256) {
      const float g = TT<T>::to_f(dyr[c]) * (gamma ? gamma[c] : 1.f);
      a += g;
      b += g * ((TT<T>::to_f(xr[c]) - m) * rs);
    }
    a = block_sum(a, sh) / (float)D;
    b = block_sum(b, sh) / (float)D;
    for (int c = threadIdx.x; c < D; c += 256) {
      const float g = TT<T>::to_f(dyr[c]) * (gamma ? gamma[c] : 1.f);
      dxr[c] = TT<T>::from_f(rs * (g - a - (TT<T>::to_f(xr[c]) - m) * rs * b));
    }
  }
}

// Column sums: a block covers 64 columns with 4 row groups (rows g, g+4,
// ...); the four group sums are added in order.
template <typename T>
__global__ __launch_bounds__(256) void ln_param_grad_kernel(const T* __restrict__ dy, const T* __restrict__ x,
                                                            const float* __restrict__ mean,
                                                            const float* __restrict__ rstd,
                                                            float* __restrict__ dgamma, float* __restrict__ dbeta,
                                                            long R, int D, long lddy, long ldx) {
  __shared__ float pg[4][64], pb[4][64];
  const int q = threadIdx.x >> 6, l = threadIdx.x & 63;
  const long c = (long)blockIdx.x * 64 + l;
  float sg = 0.f, sb = 0.f;
  if (c < D)
    for (long r = q; r < R; r += 4) {
      const float g = TT<T>::to_f(dy[r * lddy + c]);
      sg += g * ((TT<T>::to_f(x[r * ldx + c]) - mean[r]) * rstd[r]);
      sb += g;
    }
  pg[q][l] = sg;
  pb[q][l] = sb;
  __syncthreads();
  if (q == 0 && c < D) {
    if (dgamma) dgamma[c] = ((pg[0][l] + pg[1][l]) + pg[2][l]) + pg[3][l];
    if (dbeta) dbeta[c] = ((pb[0][l] + pb[1][l]) + pb[2][l]) + pb[3][l];
  }
}

}  // namespace

int layernorm_fwd_launch(int prec, const void* x, const float* gamma, const float* beta, void* y, float* mean,
                         float* rstd, long R, int D, long ldx, long ldy, float eps, hipStream_t s) {
  if (R <= 0) return 0;
  return with_prec(prec, [&](auto tag) {
    using T = decltype(tag);
    hipLaunchKernelGGL(ln_fwd_kernel<T>, dim3(row_grid(R)), dim3(256), 0, s, (const T*)x, gamma, beta, (T*)y, mean,
                       rstd, R, D, ldx, ldy, eps);
    return ok();
  });
}

size_t layernorm_bwd_workspace(int prec, long R, int D) {
  (void)prec; (void)R; (void)D;
  return 0;
}

int layernorm_bwd_launch(int prec, const void* dy, const void* x, const float* gamma, const float* mean,
                         const float* rstd, void* dx, float* dgamma, float* dbeta, long R, int D, long lddy, long ldx,
                         long lddx, void* ws, hipStream_t s) {
  (void)ws;
  return with_prec(prec, [&](auto tag) {
    using T = decltype(tag);
    // before dx, which may replace dy or x
    if (dgamma || dbeta)
      hipLaunchKernelGGL(ln_param_grad_kernel<T>, dim3(ceil_div(D, 64)), dim3(256), 0, s, (const T*)dy, (const T*)x,
                         mean, rstd, dgamma, dbeta, R, D, lddy, ldx);
    if (R > 0)
      hipLaunchKernelGGL(ln_bwd_kernel<T>, dim3(row_grid(R)), dim3(256), 0, s, (const T*)dy, (const T*)x, gamma, mean,
                         rstd, (T*)dx, R, D, lddy, ldx, lddx);
    return ok();
  });
}

}  // namespace rn18

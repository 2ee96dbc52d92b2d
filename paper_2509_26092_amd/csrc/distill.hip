// The distillation loss of a student against a teacher's top logits, with the
// gradient of the student's logits.
#include <math.h>

#include "kernels.h"

namespace rn18 {

namespace {

inline int ok() { return hipGetLastError() == hipSuccess ? 0 : -4; }

int row_grid(long R) { return (int)(R < 65536 ? R : 65536); }

__device__ inline float block_red(float v, float* sh, bool is_max) {
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    const float w = __shfl_xor(v, o);
    v = is_max ? fmaxf(v, w) : v + w;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  if (is_max) return fmaxf(fmaxf(sh[0], sh[1]), fmaxf(sh[2], sh[3]));
  return (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

// One block per row, three passes over it: maximum, sums of exponentials,
// gradient. The classes that the teacher's list or the label name are
// written last, by the thread of the first list entry that names them.
template <typename T>
__global__ __launch_bounds__(256) void distill_kernel(DistillArgs a) {
  __shared__ float sh[4];
  __shared__ float q[kTopMax], tv[kTopMax];
  __shared__ int32_t qi[kTopMax];
  const T* z = (const T*)a.z;
  T* dz = (T*)a.dz;
  const float invt = 1.0f / a.temperature;
  for (long r = blockIdx.x; r < a.R; r += gridDim.x) {
    const T* zr = z + r * a.ldz;
    T* dr = dz ? dz + r * a.lddz : nullptr;
    const float w = a.weight ? a.weight[r] : 1.0f;
    if (w == 0.f) {
      for (int c = threadIdx.x; dr && c < a.C; c += 256) dr[c] = TT<T>::from_f(0.f);
      if (threadIdx.x == 0) a.row_loss[r] = 0.f;
      continue;
    }
    const int lab = a.labels && a.alpha != 1.0f ? a.labels[r] : -1;
    const bool hard = lab >= 0 && lab < a.C;
    // the teacher's distribution over its valid entries
    float tm = -INFINITY;
    __syncthreads();
    for (int k = threadIdx.x; k < a.K; k += 256) {
      const int i = a.t_idx[r * a.K + k];
      const float t = a.t_vals[r * a.K + k] * invt;
      const bool valid = i >= 0 && i < a.C && t != -INFINITY;
      qi[k] = valid ? i : -1;
      tv[k] = valid ? t : -INFINITY;
      if (valid) tm = fmaxf(tm, t);
    }
    tm = block_red(tm, sh, true);
    if (tm == -INFINITY) tm = 0.f;
    float ts = 0.f;
    for (int k = threadIdx.x; k < a.K; k += 256) {
      q[k] = qi[k] < 0 ? 0.f : expf(tv[k] - tm);
      ts += q[k];
    }
    ts = block_red(ts, sh, false);
    float m = -INFINITY;
    for (int c = threadIdx.x; c < a.C; c += 256) m = fmaxf(m, TT<T>::to_f(zr[c]));
    m = block_red(m, sh, true);
    if (m == -INFINITY) m = 0.f;
    float s1 = 0.f, st = 0.f;
    for (int c = threadIdx.x; c < a.C; c += 256) {
      const float d = TT<T>::to_f(zr[c]) - m;
      s1 += expf(d);
      st += expf(d * invt);
    }
    s1 = block_red(s1, sh, false);
    st = block_red(st, sh, false);
    const bool some = st != 0.f;              // false: every class of the row is masked
    const bool soft_on = ts != 0.f && some, hard_on = hard && some;
    const float lse_t = logf(st), lse_q = logf(ts);
    float l = 0.f;
    if (soft_on)
      for (int k = threadIdx.x; k < a.K; k += 256) {
        const float p = q[k] / ts;
        if (qi[k] >= 0 && p != 0.f)
          l += p * ((tv[k] - tm - lse_q) - ((TT<T>::to_f(zr[qi[k]]) - m) * invt - lse_t));
      }
    l = block_red(l, sh, false);
    if (threadIdx.x == 0) {
      float v = soft_on ? a.alpha * a.temperature * a.temperature * l : 0.f;
      if (hard_on) v += (1.0f - a.alpha) * (logf(s1) - (TT<T>::to_f(zr[lab]) - m));
      a.row_loss[r] = w * v;
    }
    if (dr) {
      const float f = a.scale * w;
      const float ft = soft_on ? f * a.alpha * a.temperature : 0.f, fh = hard_on ? f * (1.0f - a.alpha) : 0.f;
      auto grad = [&](float zv) {
        const float d = zv - m;
        float g = 0.f;
        if (soft_on) g += ft * (expf(d * invt) / st);
        if (hard_on) g += fh * (expf(d) / s1);
        return g;
      };
      // the named classes' values, before dz (which may replace z) is written
      float gk = 0.f, gy = 0.f;
      bool own_k = false, own_y = false;
      int at = -1;
      const int k = threadIdx.x;
      if (soft_on && k < a.K && qi[k] >= 0) {
        at = qi[k];
        own_k = true;
        float sum = 0.f;
        for (int j = 0; j < a.K; ++j)
          if (qi[j] == at) {
            if (j < k) own_k = false;
            sum += q[j];
          }
        gk = grad(TT<T>::to_f(zr[at])) - ft * (sum / ts) - (hard_on && at == lab ? fh : 0.f);
      }
      if (hard_on && threadIdx.x == 0) {
        own_y = true;
        for (int j = 0; soft_on && j < a.K; ++j) own_y &= qi[j] != lab;
        gy = grad(TT<T>::to_f(zr[lab])) - fh;
      }
      __syncthreads();
      for (int c = threadIdx.x; c < a.C; c += 256) dr[c] = TT<T>::from_f(grad(TT<T>::to_f(zr[c])));
      __syncthreads();
      if (own_k) dr[at] = TT<T>::from_f(gk);
      if (own_y) dr[lab] = TT<T>::from_f(gy);
    }
  }
}

// loss = scale * sum of the row losses, added in 64 bits in a fixed order.
__global__ __launch_bounds__(256) void distill_loss_kernel(const float* __restrict__ row_loss, long R, float scale,
                                                           float* __restrict__ loss) {
  __shared__ double sh[256];
  double v = 0.0;
  for (long i = threadIdx.x; i < R; i += 256) v += (double)row_loss[i];
  sh[threadIdx.x] = v;
  __syncthreads();
  for (int s = 128; s > 0; s >>= 1) {
    if ((int)threadIdx.x < s) sh[threadIdx.x] += sh[threadIdx.x + s];
    __syncthreads();
  }
  if (threadIdx.x == 0) loss[0] = (float)(sh[0] * (double)scale);
}

}  // namespace

size_t distill_workspace(int prec, long R, int C, int K) {
  (void)prec; (void)R; (void)C; (void)K;
  return 0;
}

int distill_launch(int prec, const DistillArgs& a, float* loss, void* ws, hipStream_t s) {
  (void)ws;
  return with_prec(prec, [&](auto tag) {
    using T = decltype(tag);
    if (a.R > 0) hipLaunchKernelGGL(distill_kernel<T>, dim3(row_grid(a.R)), dim3(256), 0, s, a);
    if (loss) hipLaunchKernelGGL(distill_loss_kernel, dim3(1), dim3(256), 0, s, a.row_loss, a.R, a.scale, loss);
    return ok();
  });
}

}  // namespace rn18

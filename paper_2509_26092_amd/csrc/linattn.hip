// Linear attention with a decay for each head, over whole sequences, its
// backward pass, and the form for single tokens.
//   S_t = exp(g) S_(t-1) + k_t v_t^T,  o_t = scale S_t^T q_t
// The three gradients are passes of the same kind: with roles exchanged
//   dq_t = scale S_t dO_t             reads (dO, v, k) in the places of (q, k, v),
//   dk_t = G_t v_t, dv_t = G_t^T k_t  read (v, dO, q) and (k, q, dO) from the last
//                                     token to the first,
// G_t = exp(g) G_(t+1) + scale q_t dO_t^T. A pass is described by Core.
#include <math.h>

#include "rows.h"

namespace rn18 {

namespace {

// One operand: rows ld elements apart, head h of the pass at column
// (h / group) * width.
struct Operand {
  const void* p;
  long ld;
  int group;
};
// A pass: for the tokens in order (rev: from the last to the first)
//   S <- exp(g) S + kv_scale k v^T (M x N),  out = out_scale S^T q
// rev takes the decay behind a token instead of before it:
//   S' = S + kv_scale k v^T,  out = out_scale S'^T q,  S <- exp(g) S'
// s_in and s_out hold element (m, n) of a head's state at m * s_m + n * s_n.
struct Core {
  Operand q, k, v;
  void* out;
  long ldo;
  int out_f32;   // out is fp32 [tokens][H][N] whatever the storage type
  const float* log_decay;
  const int32_t* lengths;
  const float* s_in;
  float* s_out;
  int s_m, s_n;
  int B, T, H, M, N, rev;
  float out_scale, kv_scale;
};

// Tokens of sequence b.
__device__ inline int seq_len(const Core& c, int b) {
  return c.lengths ? min(max(c.lengths[b], 0), c.T) : c.T;
}

// A block per sequence, head and 64 columns; a lane's column of the state
// lives in LDS.
template <typename T>
__global__ __launch_bounds__(64) void linattn_plain_kernel(Core c) {
  __shared__ float S[256][64], sq[256], sk[256];
  const int lane = threadIdx.x, n = blockIdx.y * 64 + lane, b = blockIdx.x / c.H, h = blockIdx.x % c.H;
  const bool in = n < c.N;
  const int len = seq_len(c, b);
  const float decay = expf(c.log_decay[h]);
  const long head = (long)blockIdx.x * c.M * c.N;
  for (int m = 0; m < c.M; ++m) S[m][lane] = in && c.s_in ? c.s_in[head + (long)m * c.s_m + (long)n * c.s_n] : 0.f;
  for (int i = 0; i < len; ++i) {
    const long row = (long)b * c.T + (c.rev ? len - 1 - i : i);
    __syncthreads();
    for (int m = lane; m < c.M; m += 64) {
      sq[m] = TT<T>::to_f(((const T*)c.q.p)[row * c.q.ld + (long)(h / c.q.group) * c.M + m]);
      sk[m] = TT<T>::to_f(((const T*)c.k.p)[row * c.k.ld + (long)(h / c.k.group) * c.M + m]);
    }
    __syncthreads();
    if (!in) continue;
    const float v = c.kv_scale * TT<T>::to_f(((const T*)c.v.p)[row * c.v.ld + (long)(h / c.v.group) * c.N + n]);
    float o = 0.f;
    for (int m = 0; m < c.M; ++m) {
      const float s = (c.rev ? S[m][lane] : decay * S[m][lane]) + sk[m] * v;
      o += s * sq[m];
      S[m][lane] = c.rev ? decay * s : s;
    }
    o *= c.out_scale;
    if (c.out_f32) ((float*)c.out)[(row * c.H + h) * c.N + n] = o;
    else ((T*)c.out)[row * c.ldo + (long)h * c.N + n] = TT<T>::from_f(o);
  }
  if (in && c.s_out)
    for (int m = 0; m < c.M; ++m) c.s_out[head + (long)m * c.s_m + (long)n * c.s_n] = S[m][lane];
}

// The gradients of query heads that share a key head, added up in the order
// of the heads: part fp32 [tokens][H][N] to out [tokens][H / group][N].
template <typename T>
__global__ __launch_bounds__(256) void linattn_group_sum_kernel(const float* __restrict__ part, T* out, long ldo,
                                                                const int32_t* lengths, int B, int T_, int H, int group,
                                                                int N) {
  const int Hk = H / group, cols = Hk * N;
  const long total = (long)B * T_ * cols;
  for (long i = blockIdx.x * 256l + threadIdx.x; i < total; i += gridDim.x * 256l) {
    const long row = i / cols;
    const int col = (int)(i - row * cols), hk = col / N, n = col - hk * N;
    if (lengths && (int)(row % T_) >= lengths[row / T_]) continue;
    const float* p = part + (row * H + (long)hk * group) * N + n;
    float s = p[0];
    for (int g = 1; g < group; ++g) s += p[(long)g * N];
    out[row * ldo + col] = TT<T>::from_f(s);
  }
}

// One token: a block per sequence and head, a lane per four columns of the
// state and group of its rows; bound by reading and writing the state.
template <typename T>
__global__ __launch_bounds__(256) void linattn_step_kernel(LinattnFwd a, int per_row) {
  __shared__ float sq[256], sk[256], part[16][260];
  const int b = blockIdx.x / a.H, h = blockIdx.x % a.H, hk = h / (a.H / a.Hk), t = threadIdx.x;
  if (t < a.Dk) {
    sq[t] = TT<T>::to_f(((const T*)a.q)[b * a.ldq + (long)h * a.Dk + t]) * a.scale;
    sk[t] = TT<T>::to_f(((const T*)a.k)[b * a.ldk + (long)hk * a.Dk + t]);
  }
  __syncthreads();
  const int c = t % per_row, g = t / per_row, groups = 256 / per_row, n0 = c * 4, D = a.Dv;
  const float decay = exp2f(a.log_decay[h] * kLog2e);
  const float* in = a.s0 + (long)blockIdx.x * a.Dk * D;
  float* out = a.sT + (long)blockIdx.x * a.Dk * D;
  float v[4], o[4] = {};
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = n0 + j < D ? TT<T>::to_f(((const T*)a.v)[b * a.ldv + (long)hk * D + n0 + j]) : 0.f;
  for (int m = g; m < a.Dk; m += groups) {
    float s[4] = {};
    const float *src = in + (long)m * D + n0, q = sq[m], k = sk[m];
    float* dst = out + (long)m * D + n0;
    if (n0 + 4 <= D) {
      __builtin_memcpy(s, src, 16);
    } else {
#pragma unroll
      for (int j = 0; j < 3; ++j)
        if (n0 + j < D) s[j] = src[j];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      s[j] = decay * s[j] + k * v[j];
      o[j] += q * s[j];
    }
    if (n0 + 4 <= D) {
      __builtin_memcpy(dst, s, 16);
    } else {
#pragma unroll
      for (int j = 0; j < 3; ++j)
        if (n0 + j < D) dst[j] = s[j];
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) part[g & 15][n0 + j] = 0.f;
  __syncthreads();
  // the row groups' sums: by sixteens in order where there are more of them
  for (int p = 0; p < groups; p += 16) {
    if (g / 16 == p / 16)
#pragma unroll
      for (int j = 0; j < 4; ++j) part[g & 15][n0 + j] += o[j];
    __syncthreads();
  }
  for (int n = t; n < D; n += 256) {
    float s = 0.f;
    for (int p = 0; p < min(groups, 16); ++p) s += part[p][n];
    ((T*)a.o)[b * a.ldo + (long)h * D + n] = TT<T>::from_f(s);
  }
}

int core_launch(int prec, const Core& c, hipStream_t s) {
  if (c.B <= 0) return 0;
  return with_prec(prec, [&](auto tag) {
    using T = decltype(tag);
    hipLaunchKernelGGL(linattn_plain_kernel<T>, dim3(c.B * c.H, ceil_div(c.N, 64)), dim3(64), 0, s, c);
    return launched();
  });
}

int group_sum_launch(int prec, const float* part, void* out, long ldo, const LinattnBwd& a, int N, hipStream_t s) {
  const long total = (long)a.B * a.T * a.Hk * N;
  if (total <= 0) return 0;
  return with_prec(prec, [&](auto tag) {
    using T = decltype(tag);
    hipLaunchKernelGGL(linattn_group_sum_kernel<T>, dim3(even_grid((total + 255) / 256, 16)), dim3(256), 0, s, part,
                       (T*)out, ldo, a.lengths, a.B, a.T, a.H, a.H / a.Hk, N);
    return launched();
  });
}

}  // namespace

size_t linattn_fwd_workspace(int, int, int, int, int, int, int) { return 0; }

int linattn_fwd_launch(int prec, const LinattnFwd& a, void*, hipStream_t s) {
  const int G = a.H / a.Hk;
  return core_launch(prec, Core{{a.q, a.ldq, 1}, {a.k, a.ldk, G}, {a.v, a.ldv, G}, a.o, a.ldo, 0, a.log_decay, a.lengths,
                                a.s0, a.sT, a.Dv, 1, a.B, a.T, a.H, a.Dk, a.Dv, 0, a.scale, 1.f}, s);
}

int linattn_step_launch(int prec, const LinattnFwd& a, hipStream_t s) {
  if (a.B <= 0) return 0;
  int per_row = 1;
  while (per_row * 4 < a.Dv) per_row *= 2;
  return with_prec(prec, [&](auto tag) {
    using T = decltype(tag);
    hipLaunchKernelGGL(linattn_step_kernel<T>, dim3(a.B * a.H), dim3(256), 0, s, a, per_row);
    return launched();
  });
}

size_t linattn_bwd_workspace(int, int B, int T, int H, int Hk, int Dk, int Dv) {
  return H > Hk ? (size_t)B * T * H * std::max(Dk, Dv) * 4 : 0;
}

int linattn_bwd_launch(int prec, const LinattnBwd& a, void* ws, hipStream_t s) {
  const int G = a.H / a.Hk;
  const Operand q{a.q, a.ldq, 1}, k{a.k, a.ldk, G}, v{a.v, a.ldv, G}, d{a.dout, a.lddout, 1};
  // dq: the state's transpose, so that its elements are taken the other way round
  int r = core_launch(prec, Core{d, v, k, a.dq, a.lddq, 0, a.log_decay, a.lengths, a.s0, nullptr, 1, a.Dv, a.B, a.T,
                                 a.H, a.Dv, a.Dk, 0, a.scale, 1.f}, s);
  if (r) return r;
  r = core_launch(prec, Core{v, d, q, G > 1 ? ws : a.dk, a.lddk, G > 1, a.log_decay, a.lengths, a.dsT, nullptr, 1, a.Dv,
                             a.B, a.T, a.H, a.Dv, a.Dk, 1, 1.f, a.scale}, s);
  if (r || (G > 1 && (r = group_sum_launch(prec, (const float*)ws, a.dk, a.lddk, a, a.Dk, s)))) return r;
  r = core_launch(prec, Core{k, q, d, G > 1 ? ws : a.dv, a.lddv, G > 1, a.log_decay, a.lengths, a.dsT, a.ds0, a.Dv, 1,
                             a.B, a.T, a.H, a.Dk, a.Dv, 1, 1.f, a.scale}, s);
  if (r || (G > 1 && (r = group_sum_launch(prec, (const float*)ws, a.dv, a.lddv, a, a.Dv, s)))) return r;
  return 0;
}

}  // namespace rn18

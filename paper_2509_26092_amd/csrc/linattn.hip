// Linear attention with a decay for each head, over whole sequences, its
// backward pass, and the form for single tokens.
//   S_t = exp(g) S_(t-1) + k_t v_t^T,  o_t = scale S_t^T q_t
// The three gradients are passes of the same kind: with roles exchanged
//   dq_t = scale S_t dO_t             reads (dO, v, k) in the places of (q, k, v),
//   dk_t = G_t v_t, dv_t = G_t^T k_t  read (v, dO, q) and (k, q, dO) from the last
//                                     token to the first,
// G_t = exp(g) G_(t+1) + scale q_t dO_t^T. A pass is described by Core.
#include "linattn.h"

namespace rn18 {

namespace {

// What a segment's tokens leave of a state (see Kept). Growth by more than exp(64)
// goes in up to four steps: one factor would be infinite from exp(88.7) on, and make
// NaN of a state of zeros. (exp(256) takes fp32's smallest number beyond its range.)
struct KeptLong {
  Kept step;
  int steps;
  __device__ inline float operator()(float x) const {
    x = step(x);
    for (int i = 1; i < steps; ++i) x = step(x);
    return x;
  }
};
__device__ inline KeptLong kept_long(int n, float g) {
  const float t = (float)n * g;
  if (!(t > 64.f)) return KeptLong{kept(n, g), 1};
  const float most = t > 256.f ? 256.f : t;
  const int steps = (int)ceilf(most / 64.f);
  return KeptLong{kept(1, most / (float)steps), steps};
}

// Where a call has few heads, its sequences are cut into segments: a first
// launch leaves what each segment (but the last) adds to the state, this one
// turns these sums into the states that the segments start from, element by
// element in order, and a last one takes the segments from there.
__global__ __launch_bounds__(256) void linattn_segments_kernel(Cores cs, Split p, int tokens) {
  const Core c = cs.c[blockIdx.z];
  constexpr int U = 8;   // sums loaded at a time
  const int per = c.M * c.N, e = blockIdx.x * 256 + threadIdx.x, bh = blockIdx.y, b = bh / c.H;
  if (e >= per) return;
  const int len = seq_len(c, b), m = e / c.N, n = e - m * c.N;
  const float g = c.log_decay[bh - b * c.H];
  float x = c.s_in ? c.s_in[(long)bh * per + (long)m * c.s_m + (long)n * c.s_n] : 0.f;
  const KeptLong whole = kept_long(tokens, g);
  float* at = c.states + (long)bh * p.nseg * per + (long)m * c.st_m + (long)n * c.st_n;
  for (int s = 0; s < p.nseg; s += U) {
    float add[U];
#pragma unroll
    for (int u = 0; u < U; ++u) add[u] = s + u < p.nseg - 1 ? at[(long)u * per] : 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s + u >= p.nseg) break;
      at[(long)u * per] = x;
      const int k = min(max(len - (s + u) * tokens, 0), tokens);
      if (k > 0) x = (k == tokens ? whole : kept_long(k, g))(x) + add[u];
    }
    at += (long)U * per;
  }
}

// The gradients of query heads that share a key head, added up in the order
// of the heads: part fp32 [tokens][H][N] to out [tokens][H / group][N]; dk and dv
// in one launch. Added up in 64 bits, which costs nothing beside the reads: in fp32
// equal gradients' roundings all go one way (1.4e-3 of a sum over 2^17 heads).
// Bound by reading the parts (19 us for 6x4095 tokens of 8 heads over 2, 96 and 100
// columns).
struct GroupSum {
  const float* part[2];
  void* out[2];
  long ldo[2];
  int N[2];
};
// V columns a thread at a time, kGroupRun times in a block's run of columns.
// (4: 273 us for that whole backward pass; 16, which are too few blocks, 290.)
constexpr int kGroupRun = 4;
template <typename T, int V>
__global__ __launch_bounds__(256) void linattn_group_sum_kernel(GroupSum a, const int32_t* lengths, int B, int T_, int H,
                                                                int group) {
  const int w = blockIdx.y, N = a.N[w], Hk = H / group;
  const unsigned units = (unsigned)Hk * N / V, rows = (unsigned)B * T_;   // below 2^28 and 2^31
  const long total = (long)rows * units, run = 256 * kGroupRun;
  for (long e0 = blockIdx.x * run + threadIdx.x; e0 < total; e0 += gridDim.x * run) {
    unsigned row = (unsigned)(e0 / units), u = (unsigned)(e0 - (long)row * units);
    for (int i = 0; i < kGroupRun && row < rows; ++i) {
      if (!lengths || (int)(row % T_) < lengths[row / T_]) {
        const int col = (int)u * V, hk = col / N;
        const float* p = a.part[w] + ((long)row * H + (long)hk * group) * N + (col - hk * N);
        double s[V] = {};
#pragma unroll 4
        for (int g = 0; g < group; ++g) {
          float t[V];
          __builtin_memcpy(t, p + (long)g * N, sizeof(t));
#pragma unroll
          for (int j = 0; j < V; ++j) s[j] += t[j];
        }
        T o[V];
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] = TT<T>::from_f((float)s[j]);
        __builtin_memcpy((T*)a.out[w] + (long)row * a.ldo[w] + col, o, sizeof(o));
      }
      u += 256;
      if (u >= units) {
        row += u / units;
        u %= units;
      }
    }
  }
}

// One token: a block per sequence, head and part of the state's columns, a lane
// per four columns and group of the state's rows. It does 4 operations for each 8 bytes, so it is
// bound by reading and writing the state: 256 sequences, 16 heads of 128x128 (537
// MB) take 111 us, 4.8 TB/s of a copy's 5.2; one sequence, 8 heads of 64 4.5 us,
// which is a launch and three dependent passes.
template <typename T>
__global__ __launch_bounds__(256) void linattn_step_kernel(LinattnFwd a, int per_row) {
  __shared__ float sq[256], sk[256], part[16][260];
  const int b = blockIdx.x / a.H, h = blockIdx.x % a.H, hk = h / (a.H / a.Hk), t = threadIdx.x;
  if (t < a.Dk) {
    sq[t] = TT<T>::to_f(((const T*)a.q)[b * a.ldq + (long)h * a.Dk + t]) * a.scale;
    sk[t] = TT<T>::to_f(((const T*)a.k)[b * a.ldk + (long)hk * a.Dk + t]);
  }
  __syncthreads();
  const int c = t % per_row, g = t / per_row, groups = 256 / per_row, D = a.Dv;
  const int first = blockIdx.y * per_row * 4, place = c * 4, n0 = first + place, here = min(D - first, per_row * 4);
  const Kept decay = kept(1, a.log_decay[h]);
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
      s[j] = fmaf(k, v[j], decay(s[j]));
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
  for (int j = 0; j < 4; ++j) part[g & 15][place + j] = 0.f;
  __syncthreads();
  // the row groups' sums: by sixteens in order where there are more of them
  for (int p = 0; p < groups; p += 16) {
    if (g / 16 == p / 16)
#pragma unroll
      for (int j = 0; j < 4; ++j) part[g & 15][place + j] += o[j];
    __syncthreads();
  }
  for (int n = t; n < here; n += 256) {
    float s = 0.f;
    for (int p = 0; p < min(groups, 16); ++p) s += part[p][n];
    ((T*)a.o)[b * a.ldo + (long)h * D + first + n] = TT<T>::from_f(s);
  }
}

// Segments of a call: two waves for each SIMD, as many as fit there, where there
// are few heads, and up to 8192 tokens twice as many, which evens out sequences of
// other lengths (us; 6 ragged ones of up to 4095, 8 heads of 96, fp16 backward: 22
// segments 264, 11 278, 6 301; but 1x65537, 16 heads of 128, bf16 forward: 32
// segments 445, 64, whose states are a sixth of the traffic, 476, 16 495). No
// segment but the last is below four chunks, and two are none: 1x1024, 8 heads of
// 64, bf16 forward takes 23 in 8 segments of four, 31 in 4 and 55 whole, 2x256 22 in
// two segments and 18 whole. The same for a state and its transpose.
// No segments, whose sums are another pass over k and v, for heads that fill
// the card by themselves, which a backward pass does sooner: its three passes
// run side by side. us without segments and with them, where the rule begins,
// backward: bf16 12x2048, 16 heads of 64 159 and 202, 11x1000, 8 heads of 128 126
// and 165, fp32 12x1024, 16 of 128 621 and 732; below it bf16 16x3000, 8 of 64 227
// and 193, fp32 (bound by the matrix units, which want more waves) 6x2048, 16 of
// 128 804 and 711. Just below it the count is past its best: bf16 21x3000, 8 of 64
// 227 whole, 241 in 12 segments and 219 in 4, as is 16x3000 with 178 in 4. Forward,
// sequences of up to 64 chunks: bf16 12x1024, 16 of 128 87 and 132, 14x486 50 and
// 96, 12x2048 164 and 207; longer ones, below their rule: 17x3000, 16 of 64 226 and
// 174. A SIMD holds one wave of the widest states in place of two, so that half as
// many heads of 129 columns or more fill the card: bf16 backward 4x1000, 8 of 256
// 164 and 302, forward 20x400, 4 of 256 75 and 130; half of that forward, 4x1000,
// 162 and 72.
Split split_of(int prec, int B, int T, int H, int M, int N, int passes) {
  const int all = std::max(1, ceil_div(T, kChunk)), beside = passes == 1 ? 1 : prec == PREC_F32 ? 2 : 3,
            widest = std::max(M, N) > 128 ? 2 : 1;
  const long units = std::max(1l, (long)B * H * ceil_div(std::max(M, N), 64)), want = (all <= 256 ? 8l : 4l) * plan_cus();
  const long enough = passes == 1 && all <= 64 ? 3l * plan_cus() / 2 : 2l * plan_cus();
  long nseg = units * beside * widest >= enough ? 1 : std::min((want + units - 1) / units, (long)all / 4);
  if (nseg < 3) nseg = 1;
  const int chunks = ceil_div(all, nseg);
  return Split{ceil_div(all, chunks), chunks};
}
size_t split_bytes(int prec, int B, int T, int H, int M, int N, int passes) {
  const Split p = split_of(prec, B, T, H, M, N, passes);
  return p.nseg > 1 ? (size_t)B * H * p.nseg * M * N * 4 : 0;
}

int cores_launch(int prec, const Cores& cs, int passes, hipStream_t s) {
  const Core& c = cs.c[0];
  if (c.B <= 0) return 0;
  const Split p = split_of(prec, c.B, c.T, c.H, c.M, c.N, passes);
  switch (prec) {
    case PREC_F32: return chunks_launch_fp32(cs, p, s);
    case PREC_BF16: return chunks_launch_bf16(cs, p, s);
    case PREC_F16: return chunks_launch_fp16(cs, p, s);
    default: return -1;
  }
}

}  // namespace

int segments_launch(const Cores& cs, const Split& p, hipStream_t s) {
  const Core& c = cs.c[0];
  hipLaunchKernelGGL(linattn_segments_kernel, dim3(ceil_div((long)c.M * c.N, 256), c.B * c.H, cs.sums), dim3(256), 0, s, cs,
                     p, p.chunks * kChunk);
  return launched();
}

size_t linattn_fwd_workspace(int prec, int B, int T, int H, int, int Dk, int Dv) {
  return split_bytes(prec, B, T, H, Dk, Dv, 1);
}

int linattn_fwd_launch(int prec, const LinattnFwd& a, void* ws, hipStream_t s) {
  const int G = a.H / a.Hk;
  Cores cs{};
  cs.c[0] = Core{{a.q, a.ldq, 1}, {a.k, a.ldk, G}, {a.v, a.ldv, G}, a.o, a.ldo, 0, a.log_decay, a.lengths, a.s0, a.sT,
                 a.Dv, 1, a.B, a.T, a.H, a.Dk, a.Dv, 0, a.scale, 1.f, (float*)ws, a.Dv, 1};
  cs.n = cs.sums = 1;
  return cores_launch(prec, cs, 1, s);
}

int linattn_step_launch(int prec, const LinattnFwd& a, hipStream_t s) {
  if (a.B <= 0) return 0;
  int per_row = 1;
  while (per_row * 4 < a.Dv) per_row *= 2;
  // a state's columns over several blocks where there are few states (us): 95
  // sequences, 2 heads of 256 25 in place of 50 with a block each, 32, 8 heads of
  // 256 32 of 55, 8, 16 heads of 128 8.5 of 10.5
  while (per_row > 4 && (long)a.B * a.H * ceil_div(a.Dv, per_row * 4) < 4l * plan_cus()) per_row /= 2;
  return with_prec(prec, [&](auto tag) {
    using T = decltype(tag);
    hipLaunchKernelGGL(linattn_step_kernel<T>, dim3(a.B * a.H, ceil_div(a.Dv, per_row * 4)), dim3(256), 0, s, a, per_row);
    return launched();
  });
}

// Query heads' own gradients of shared keys and values, then the segment states
// of the forward and the reverse passes.
static size_t group_bytes(int B, int T, int H, int Hk, int D) {
  return H > Hk ? (((size_t)B * T * H * D * 4 + 255) & ~(size_t)255) : 0;
}
size_t linattn_bwd_workspace(int prec, int B, int T, int H, int Hk, int Dk, int Dv) {
  return group_bytes(B, T, H, Hk, Dk) + group_bytes(B, T, H, Hk, Dv) + 2 * split_bytes(prec, B, T, H, Dk, Dv, 3);
}

int linattn_bwd_launch(int prec, const LinattnBwd& a, void* ws, hipStream_t s) {
  const int G = a.H / a.Hk;
  char* at = (char*)ws;
  float* pk = (float*)at;
  at += group_bytes(a.B, a.T, a.H, a.Hk, a.Dk);
  float* pv = (float*)at;
  at += group_bytes(a.B, a.T, a.H, a.Hk, a.Dv);
  float *sf = (float*)at, *sr = (float*)(at + split_bytes(prec, a.B, a.T, a.H, a.Dk, a.Dv, 3));
  const Operand q{a.q, a.ldq, 1}, k{a.k, a.ldk, G}, v{a.v, a.ldv, G}, d{a.dout, a.lddout, 1};
  // dq and dk: on the state's transpose, whose elements are taken the other way
  // round; dv goes with dk's segments. All in one launch where their kernel is
  // the same: none waits for the last blocks of another, and what they share is
  // read together.
  const Core dq{d, v, k, a.dq, a.lddq, 0, a.log_decay, a.lengths, a.s0, nullptr, 1, a.Dv, a.B, a.T, a.H, a.Dv, a.Dk, 0,
                a.scale, 1.f, sf, a.Dk, 1};
  const Core dk{v, d, q, G > 1 ? pk : a.dk, a.lddk, G > 1, a.log_decay, a.lengths, a.dsT, nullptr, 1, a.Dv, a.B, a.T, a.H,
                a.Dv, a.Dk, 1, 1.f, a.scale, sr, a.Dk, 1};
  const Core dv{k, q, d, G > 1 ? pv : a.dv, a.lddv, G > 1, a.log_decay, a.lengths, a.dsT, a.ds0, a.Dv, 1, a.B, a.T, a.H,
                a.Dk, a.Dv, 1, 1.f, a.scale, sr, 1, a.Dk};
  const bool one = shape_of(prec, dq) == shape_of(prec, dv) && !(a.ds0 && a.ds0 == a.dsT);   // (dk reads dsT too)
  int r = cores_launch(prec, one ? Cores{{dq, dk, dv}, 3, 2} : Cores{{dq, dk, dk}, 2, 2}, 3, s);
  if (!r && !one) r = cores_launch(prec, Cores{{dv, dv, dv}, 1, 0}, 3, s);
  const long rows = (long)a.B * a.T;
  if (r || G == 1 || rows <= 0) return r;
  const GroupSum gs{{pk, pv}, {a.dk, a.dv}, {a.lddk, a.lddv}, {a.Dk, a.Dv}};
  const long units = rows * (a.H / G) * std::max(a.Dk, a.Dv);
  return with_prec(prec, [&](auto tag) {
    using T = decltype(tag);
    constexpr long run = 256 * kGroupRun;
    auto grid = [&](int V) { return dim3((unsigned)std::min((units / V + run - 1) / run, 32768l), 2); };
    if (a.Dk % 4 == 0 && a.Dv % 4 == 0)
      hipLaunchKernelGGL((linattn_group_sum_kernel<T, 4>), grid(4), dim3(256), 0, s, gs, a.lengths, a.B, a.T, a.H, G);
    else
      hipLaunchKernelGGL((linattn_group_sum_kernel<T, 1>), grid(1), dim3(256), 0, s, gs, a.lengths, a.B, a.T, a.H, G);
    return launched();
  });
}

}  // namespace rn18

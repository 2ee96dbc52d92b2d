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

// ------------------------------------------------------------------ chunks on the matrix units
// A sequence is taken in chunks of C tokens. With X the state before a chunk
// of n tokens and i, j its tokens,
//   out_i = decay^(i + 1 - rev) X^T q_i + sum_(j <= i) decay^(i - j) (q_i . k_j) v_j
//   X <- decay^n X + sum_j decay^(n - 1 + rev - j) k_j v_j^T
// (the second factors of both sums with kv_scale). No power is above one for
// a decay below one. A block of four waves takes a head's columns of 64 NT
// (16 NT a wave) of the state through the chunks: X stays in the accumulators
// of the matrix units, whose layout is also that of an operand, so that it
// never leaves them; q, k, v and the scores P pass through LDS. The next
// chunk's rows are loaded into registers meanwhile.
//
// Matrix operands in 16 bits are bf16, which has fp32's range: fp16 inputs are
// held as two parts each (exact), what is computed in fp32 (X, P, the decayed
// v) as two or three. Products of parts below 2^-16 of the result are left out,
// for the state 2^-24.

// A lane's operand of one step over KB of the inner index, in NP parts: places
// 8 (lane / 16) + 0..7 of 32 in 16 bits, 4 (lane / 16) + 0..3 of 16 in fp32
// (four steps of the unit). A state's tiles of 16 rows make "split" operands:
// places 4 (lane / 16) + 0..3 of the first and the second 16.
template <int P> struct Frag { uint4 p[P]; };

template <int P> struct Ops16 {
  typedef bf16_t lds_t;
  static constexpr int NP = P, KB = 32, EV = 8, PPARTS = 2;
  typedef Frag<P> In;
  typedef Frag<2> Two;
  typedef Frag<3> Three;
  __device__ static inline bf16x8_t v8(const uint4& q) { return __builtin_bit_cast(bf16x8_t, q); }
  // The products of part i of a and part j of b with i + j < LIM, the smallest first.
  template <int LIM, int A, int B>
  __device__ static inline void mma(floatx4_t& acc, const Frag<A>& a, const Frag<B>& b) {
#pragma unroll
    for (int i = A - 1; i >= 0; --i)
#pragma unroll
      for (int j = B - 1; j >= 0; --j)
        if (i + j < LIM) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8(a.p[i]), v8(b.p[j]), acc, 0, 0, 0);
  }
  // The leading parts of two values, which keep the rest.
  __device__ static inline uint32_t take(float& a, float& b) {
    const uint32_t h = f2bf2(a, b);
    a -= __builtin_bit_cast(float, h << 16);
    b -= __builtin_bit_cast(float, h & 0xffff0000u);
    return h;
  }
  template <int N>
  __device__ static inline Frag<N> parts(float (&v)[8]) {
    Frag<N> f;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = take(v[2 * i], v[2 * i + 1]);
      f.p[n] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return f;
  }
  __device__ static inline void values(const In& f, float (&v)[8]) {
    unpack<bf16_t>(f.p[0], v);
    if constexpr (P > 1) {
      float t[8];
      unpack<bf16_t>(f.p[1], t);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += t[i];
    }
  }
};
struct Ops32 {
  typedef float lds_t;
  static constexpr int NP = 1, KB = 16, EV = 4, PPARTS = 1;
  typedef Frag<1> In;
  typedef Frag<1> Two;
  typedef Frag<1> Three;
  template <int LIM>
  __device__ static inline void mma(floatx4_t& acc, const In& a, const In& b) {
    const floatx4_t x = __builtin_bit_cast(floatx4_t, a.p[0]), y = __builtin_bit_cast(floatx4_t, b.p[0]);
#pragma unroll
    for (int r = 0; r < 4; ++r) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[r], y[r], acc, 0, 0, 0);
  }
  template <int N>
  __device__ static inline In parts(float (&v)[4]) {
    return In{{pack<float>(v)}};
  }
  __device__ static inline void values(const In& f, float (&v)[4]) { unpack<float>(f.p[0], v); }
};
template <typename T> struct OpsOf { typedef Ops32 type; };
template <> struct OpsOf<bf16_t> { typedef Ops16<1> type; };
template <> struct OpsOf<f16_t> { typedef Ops16<2> type; };

typedef short v4i16_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char_t;

template <typename T, int MP, int NT, int C>
struct Tile {
  typedef typename OpsOf<T>::type O;
  typedef typename O::lds_t L;
  static constexpr int NP = O::NP, KB = O::KB, PP = O::PPARTS, NB = 64 * NT, PAD = 16 / (int)sizeof(L);
  static constexpr int LDM = MP + PAD, LDN = NB + PAD, LDP = C + PAD;   // (rows 4 banks further each)
  static constexpr int SQ = C * LDM, SV = C * LDN, SP = C * LDP;        // of one part
  static constexpr int OFF_K = NP * SQ, OFF_V = 2 * NP * SQ, OFF_P = OFF_V + NP * SV, ALL = OFF_P + PP * SP;
  static constexpr int BYTES = ALL * (int)sizeof(L);
  static constexpr int BLOCKS = BYTES <= 81920 ? 2 : 1;   // a compute unit
  static_assert(BYTES <= 163840 && BYTES % 16 == 0, "LDS");
};

// 16 bytes of a row's columns from `col` on, zeros from `width` on; `shift` is
// how far the row's last, partial chunk is read from before its place (which
// needs a whole chunk's width). `none`: the row is not there.
template <typename T>
__device__ inline uint4 load_part(const T* row, int col, int width, bool none) {
  constexpr int VW = TT<T>::VW;
  if (width < VW) {
    uint4 q = make_uint4(0, 0, 0, 0);
    T e[VW] = {};
    if (!none && col == 0) {
      for (int j = 0; j < VW - 1; ++j)
        if (j < width) e[j] = row[j];
      __builtin_memcpy(&q, e, 16);
    }
    return q;
  }
  const bool out = none || col >= width;
  const int at = min(col, width - VW);
  uint4 q = load_chunk(out ? (const T*)&kNoChunk : row + at);
  if (width % VW) {   // (the same for all lanes)
    const int s = 8 * (int)sizeof(T) * (VW - width % VW);
    const uint64_t lo = q.x | (uint64_t)q.y << 32, hi = q.z | (uint64_t)q.w << 32;
    const uint64_t l2 = s >= 64 ? hi >> (s & 63) : lo >> s | hi << (64 - s), h2 = s >= 64 ? 0 : hi >> s;
    if (!out && at != col) q = make_uint4((uint32_t)l2, (uint32_t)(l2 >> 32), (uint32_t)h2, (uint32_t)(h2 >> 32));
  }
  return q;
}

// A chunk of 16 bytes into LDS: its parts, `step` elements apart.
template <typename T>
__device__ inline void put(typename OpsOf<T>::type::lds_t* p, int step, const uint4& q) {
  if constexpr (OpsOf<T>::type::NP == 1) {
    *(uint4*)p = q;
  } else {
    float v[8];
    unpack<T>(q, v);
    const auto f = OpsOf<T>::type::template parts<2>(v);
    *(uint4*)p = f.p[0];
    *(uint4*)(p + step) = f.p[1];
  }
}

template <typename T, int MP, int NT, int C, bool SUMS>
__global__ __launch_bounds__(256, (Tile<T, MP, NT, C>::BLOCKS)) void linattn_chunk_kernel(
    Core c, float* seg_states, int nseg, int chunks, int nb_n) {
  typedef Tile<T, MP, NT, C> TI;
  typedef typename OpsOf<T>::type O;
  typedef typename O::lds_t L;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int VW = TT<T>::VW, MT = MP / 16, CT = C / 16, KB = TI::KB, NP = TI::NP;
  constexpr int PER_M = MP / VW, PER_N = TI::NB / VW, NQ = C * PER_M / 256, NV = C * PER_N / 256;
  __shared__ uint4 smem[TI::BYTES / 16];
  L* const sQ = (L*)smem;
  L* const sK = sQ + TI::OFF_K;
  L* const sV = sQ + TI::OFF_V;
  L* const sP = sQ + TI::OFF_P;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, i0 = lane & 15,
            g = lane >> 4;
  // neighbours on an XCD: a head's segments, its column blocks, the heads
  const int segs = SUMS ? nseg - 1 : nseg, id = xcd_remap(blockIdx.x, gridDim.x);
  const int seg = id % segs, nb = id / segs % nb_n, bh = id / segs / nb_n, b = bh / c.H, h = bh - b * c.H;
  const int len = seq_len(c, b), t_first = seg * chunks * C, total = min(max(len - t_first, 0), chunks * C);
  const float g2 = c.log_decay[h] * kLog2e;
  auto pw = [&](int n) { return n <= 0 ? 1.f : exp2f((float)n * g2); };
  const int n_wave = nb * TI::NB + w * 16 * NT;   // the wave's columns from here on
  const bool works = n_wave < c.N;

  floatx4_t X[MT][NT];
  {
    const bool stored = !SUMS && nseg > 1;
    const float* src = stored ? seg_states + ((long)bh * nseg + seg) * c.M * c.N : c.s_in + (long)bh * c.M * c.N;
    const int s_m = stored ? c.N : c.s_m, s_n = stored ? 1 : c.s_n;
    const bool any = !SUMS && (stored || c.s_in);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int m = 16 * mt + 4 * g + r, n = n_wave + 16 * nt + i0;
          X[mt][nt][r] = any && m < c.M && n < c.N ? src[(long)m * s_m + (long)n * s_n] : 0.f;
        }
  }

  const long dir = c.rev ? -1 : 1, row0 = (long)b * c.T + (c.rev ? len - 1 - t_first : t_first);
  uint4 rq[SUMS ? 1 : NQ], rk[NQ], rv[NV];
  auto fetch = [&](int t0) {
    auto rows = [&](const Operand& x, int width, int n0, auto& r, int count, int per) {
      const T* p = (const T*)x.p + (long)(h / x.group) * width;
#pragma unroll
      for (int s = 0; s < count; ++s) {
        const int e = s * 256 + tid, i = t0 + e / per, col = n0 + e % per * VW;
        r[s] = load_part(p + (row0 + dir * i) * x.ld, col, width, i >= total);
      }
    };
    if (!SUMS) rows(c.q, c.M, 0, rq, NQ, PER_M);
    rows(c.k, c.M, 0, rk, NQ, PER_M);
    rows(c.v, c.N, nb * TI::NB, rv, NV, PER_N);
  };

  // operands from LDS: of a row, of a row in split places, of a column
  auto frag_row = [&](const L* base, int ld, int part, int row, int k0) {
    typename O::In f;
#pragma unroll
    for (int p = 0; p < NP; ++p) f.p[p] = *(const uint4*)(base + p * part + (row + i0) * ld + k0 + O::EV * g);
    return f;
  };
  auto frag_split = [&](const L* base, int row, int k0) {
    if constexpr (F32) {
      return frag_row(base, TI::LDM, 0, row, k0);
    } else {
      typename O::In f;
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const L* at = base + p * TI::SQ + (row + i0) * TI::LDM + k0 + 4 * g;
        const uint2 x = *(const uint2*)at, y = *(const uint2*)(at + 16);
        f.p[p] = make_uint4(x.x, x.y, y.x, y.y);
      }
      return f;
    }
  };
  auto frag_col = [&](const L* base, int ld, int part, int row, int col) {
    typename O::In f;
    if constexpr (F32) {
      float v[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = base[(row + 4 * g + r) * ld + col + i0];
      f.p[0] = pack<float>(v);
    } else {
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const L* at = base + p * part + (row + 8 * g + (i0 >> 2)) * ld + col + 4 * (i0 & 3);
        auto tr = [](const L* a) {
          return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16_t*)(lds_char_t*)a));
        };
        const uint2 x = tr(at), y = tr(at + 4 * ld);
        f.p[p] = make_uint4(x.x, x.y, y.x, y.y);
      }
    }
    return f;
  };

  if (!SUMS && !F32)   // the upper tile beside a diagonal one is read with it
    for (int e = tid; e < TI::PP * TI::SP * (int)sizeof(L) / 16; e += 256) ((uint4*)sP)[e] = make_uint4(0, 0, 0, 0);
  if (total > 0) fetch(0);
  for (int t0 = 0; t0 < total; t0 += C) {
    const int n = min(C, total - t0);
    __syncthreads();   // the last chunk is read
#pragma unroll
    for (int s = 0; s < NQ; ++s) {
      const int e = s * 256 + tid, at = e / PER_M * TI::LDM + e % PER_M * VW;
      if (!SUMS) put<T>(sQ + at, TI::SQ, rq[SUMS ? 0 : s]);
      put<T>(sK + at, TI::SQ, rk[s]);
    }
#pragma unroll
    for (int s = 0; s < NV; ++s) {
      const int e = s * 256 + tid;
      put<T>(sV + e / PER_N * TI::LDN + e % PER_N * VW, TI::SV, rv[s]);
    }
    __syncthreads();
    if (t0 + C < total) fetch(t0 + C);

    if constexpr (!SUMS) {
      // scores: the tiles up to the diagonal, one wave each in turn; P^T comes
      // out with a lane's token i = its column
      for (int t = w; t < CT * (CT + 1) / 2; t += 4) {
        const int it = t < 1 ? 0 : t < 3 ? 1 : t < 6 ? 2 : 3, jt = t - it * (it + 1) / 2;
        floatx4_t a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k0 = 0; k0 < MP; k0 += KB)
          O::template mma<2>(a, frag_row(sK, TI::LDM, TI::SQ, 16 * jt, k0), frag_row(sQ, TI::LDM, TI::SQ, 16 * it, k0));
        float p[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int d = 16 * (it - jt) + i0 - 4 * g - r;
          p[r] = d < 0 ? 0.f : a[r] * (pw(d) * c.kv_scale);
        }
        L* at = sP + (16 * it + i0) * TI::LDP + 16 * jt + 4 * g;
        if constexpr (F32) {
          *(uint4*)at = pack<float>(p);
        } else {
#pragma unroll
          for (int q = 0; q < TI::PP; ++q) {
            const uint32_t lo = O::take(p[0], p[1]), hi = O::take(p[2], p[3]);
            *(uint2*)(at + q * TI::SP) = make_uint2(lo, hi);
          }
        }
      }
    }

    typename O::In V[C / KB][NT];
    float bad = 0.f;   // NaN if one of the chunk's v is not finite
    floatx4_t out[SUMS ? 1 : CT][NT];
    if (works) {
#pragma unroll
      for (int jb = 0; jb < C / KB; ++jb)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          V[jb][nt] = frag_col(sV, TI::LDN, TI::SV, jb * KB, w * 16 * NT + 16 * nt);
      if constexpr (!SUMS) {
#pragma unroll
        for (int it = 0; it < CT; ++it)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) out[it][nt] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kb = 0; kb < MP / KB; ++kb) {
          typename O::Two A[NT];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float x[O::EV];
#pragma unroll
            for (int e = 0; e < O::EV; ++e) x[e] = X[kb * KB / 16 + e / 4][nt][e % 4];
            A[nt] = O::template parts<2>(x);
          }
#pragma unroll
          for (int it = 0; it < CT; ++it) {
            const auto q = frag_split(sQ, 16 * it, kb * KB);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) O::template mma<2>(out[it][nt], A[nt], q);
          }
        }
#pragma unroll
        for (int it = 0; it < CT; ++it) {
          const float up = pw(16 * it + i0 + 1 - c.rev);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) out[it][nt] *= up;
        }
      }
      // the state behind the chunk; the operands read here serve the sums within it too
      const float less = expm1f((float)n * c.log_decay[h]);   // decay^n - 1: exact near 1, where many chunks multiply
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int r = 0; r < 4; ++r) X[mt][nt][r] = fmaf(X[mt][nt][r], less, X[mt][nt][r]);
#pragma unroll
      for (int jb = 0; jb < C / KB; ++jb) {
        typename O::Three D[NT];
        float f[O::EV];
#pragma unroll
        for (int e = 0; e < O::EV; ++e) f[e] = pw(n - 1 + c.rev - (jb * KB + O::EV * g + e)) * c.kv_scale;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float v[O::EV];
          O::values(V[jb][nt], v);
#pragma unroll
          for (int e = 0; e < O::EV; ++e) {
            bad = fmaf(v[e], 0.f, bad);
            v[e] *= f[e];
          }
          D[nt] = O::template parts<3>(v);
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          const auto k = frag_col(sK, TI::LDM, TI::SQ, jb * KB, 16 * mt);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) O::template mma<3>(X[mt][nt], k, D[nt]);
        }
      }
    }
    if constexpr (!SUMS) {
      __syncthreads();   // the scores are there
      if (works) {
        if (__builtin_expect(!__any(bad != 0.f), 1)) {
#pragma unroll
          for (int it = 0; it < CT; ++it)
#pragma unroll
            for (int jb = 0; jb <= (16 * it + 15) / KB; ++jb) {
              Frag<TI::PP> p;
#pragma unroll
              for (int q = 0; q < TI::PP; ++q)
                p.p[q] = *(const uint4*)(sP + q * TI::SP + (16 * it + i0) * TI::LDP + jb * KB + O::EV * g);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) O::template mma<2>(out[it][nt], V[jb][nt], p);
            }
        } else {
          // a NaN or an infinity of a later token must not meet an earlier
          // one's zero score: one term after the other
#pragma unroll
          for (int it = 0; it < CT; ++it)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
              for (int j = 0; j <= 16 * it + i0; ++j) {
                float p = 0.f;
#pragma unroll
                for (int q = TI::PP - 1; q >= 0; --q) p += TT<L>::to_f(sP[q * TI::SP + (16 * it + i0) * TI::LDP + j]);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                  float v = 0.f;
#pragma unroll
                  for (int q = NP - 1; q >= 0; --q)
                    v += TT<L>::to_f(sV[q * TI::SV + j * TI::LDN + w * 16 * NT + 16 * nt + 4 * g + r]);
                  out[it][nt][r] = fmaf(p, v, out[it][nt][r]);
                }
              }
        }
#pragma unroll
        for (int it = 0; it < CT; ++it) {
          const int i = t0 + 16 * it + i0;
          if (i >= total) continue;
          const long row = row0 + dir * i;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            const int col = n_wave + 16 * nt + 4 * g;
            const floatx4_t v = out[it][nt] * c.out_scale;
            if (c.out_f32) {
              float* o = (float*)c.out + (row * c.H + h) * c.N + col;
              if (col + 4 <= c.N) {
                __builtin_memcpy(o, &v, 16);
              } else {
#pragma unroll
                for (int r = 0; r < 3; ++r)
                  if (col + r < c.N) o[r] = v[r];
              }
            } else {
              T* o = (T*)c.out + row * c.ldo + (long)h * c.N + col;
              T e[4];
#pragma unroll
              for (int r = 0; r < 4; ++r) e[r] = TT<T>::from_f(v[r]);
              if (col + 4 <= c.N) {
                __builtin_memcpy(o, e, sizeof(e));
              } else {
#pragma unroll
                for (int r = 0; r < 3; ++r)
                  if (col + r < c.N) o[r] = e[r];
              }
            }
          }
        }
      }
    }
  }

  if (!SUMS && (!c.s_out || seg != nseg - 1)) return;
  float* to = SUMS ? seg_states + ((long)bh * nseg + seg) * c.M * c.N : c.s_out + (long)bh * c.M * c.N;
  const int s_m = SUMS ? c.N : c.s_m, s_n = SUMS ? 1 : c.s_n;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int m = 16 * mt + 4 * g + r, n = n_wave + 16 * nt + i0;
        if (m < c.M && n < c.N) to[(long)m * s_m + (long)n * s_n] = X[mt][nt][r];
      }
}

// Where a call has few heads, its sequences are cut into segments: a first
// launch leaves what each segment (but the last) adds to the state, this one
// turns these sums into the states that the segments start from, element by
// element in order, and a last one takes the segments from there.
__global__ __launch_bounds__(256) void linattn_segments_kernel(Core c, float* seg_states, int nseg, int tokens) {
  const int per = c.M * c.N, e = blockIdx.x * 256 + threadIdx.x, bh = blockIdx.y, b = bh / c.H;
  if (e >= per) return;
  const int len = seq_len(c, b), m = e / c.N, n = e - m * c.N;
  const float g = c.log_decay[bh - b * c.H];
  float x = c.s_in ? c.s_in[(long)bh * per + (long)m * c.s_m + (long)n * c.s_n] : 0.f;
  float* p = seg_states + (long)bh * nseg * per + e;
  for (int s = 0; s < nseg - 1; ++s, p += per) {
    const int k = min(max(len - s * tokens, 0), tokens);
    const float add = *p;
    *p = x;
    if (k > 0) x = fmaf(x, expm1f((float)k * g), x) + add;
  }
  *p = x;
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

// Segments of a call: enough blocks for the chip where there are few heads,
// but no segment below four chunks.
struct Split {
  int nb, nseg, chunks;   // column blocks, segments, chunks of a segment
};
int chunk_of(int prec, int M) { return prec == PREC_F32 || (prec == PREC_F16 && M > 128) ? 32 : 64; }
Split split_of(int prec, int B, int T, int H, int M, int N) {
  const int C = chunk_of(prec, M), nb = N > 64 ? ceil_div(N, 128) : 1, all = std::max(1, ceil_div(T, C));
  const long blocks = std::max(1l, (long)B * H * nb);
  long nseg = blocks >= plan_cus() ? 1 : std::min((2l * plan_cus() + blocks - 1) / blocks, (long)all / 4);
  nseg = std::max(1l, nseg);
  const int chunks = ceil_div(all, nseg);
  return Split{nb, ceil_div(all, chunks), chunks};
}
size_t split_bytes(int prec, int B, int T, int H, int M, int N) {
  const Split p = split_of(prec, B, T, H, M, N);
  return p.nseg > 1 ? (size_t)B * H * p.nseg * M * N * 4 : 0;
}

template <typename T, int MP, int NT, int C>
int chunk_launch(const Core& c, const Split& p, float* states, hipStream_t s) {
  const int heads = c.B * c.H;
  if (p.nseg > 1) {
    hipLaunchKernelGGL((linattn_chunk_kernel<T, MP, NT, C, true>), dim3(heads * p.nb * (p.nseg - 1)), dim3(256), 0, s, c,
                       states, p.nseg, p.chunks, p.nb);
    hipLaunchKernelGGL(linattn_segments_kernel, dim3(ceil_div((long)c.M * c.N, 256), heads), dim3(256), 0, s, c, states,
                       p.nseg, p.chunks * C);
  }
  hipLaunchKernelGGL((linattn_chunk_kernel<T, MP, NT, C, false>), dim3(heads * p.nb * p.nseg), dim3(256), 0, s, c, states,
                     p.nseg, p.chunks, p.nb);
  return launched();
}

// `states`: split_bytes of the pass.
int core_launch(int prec, const Core& c, float* states, hipStream_t s) {
  if (c.B <= 0) return 0;
  const Split p = split_of(prec, c.B, c.T, c.H, c.M, c.N);
  return with_prec(prec, [&](auto tag) {
    using T = decltype(tag);
    constexpr int C = sizeof(T) == 4 ? 32 : 64, C256 = prec_of<T>() == PREC_BF16 ? 64 : 32;
    if (c.N <= 64) {
      if (c.M <= 64) return chunk_launch<T, 64, 1, C>(c, p, states, s);
      if (c.M <= 128) return chunk_launch<T, 128, 1, C>(c, p, states, s);
      return chunk_launch<T, 256, 1, C256>(c, p, states, s);
    }
    if (c.M <= 64) return chunk_launch<T, 64, 2, C>(c, p, states, s);
    if (c.M <= 128) return chunk_launch<T, 128, 2, C>(c, p, states, s);
    return chunk_launch<T, 256, 2, C256>(c, p, states, s);
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

size_t linattn_fwd_workspace(int prec, int B, int T, int H, int, int Dk, int Dv) {
  return split_bytes(prec, B, T, H, Dk, Dv);
}

int linattn_fwd_launch(int prec, const LinattnFwd& a, void* ws, hipStream_t s) {
  const int G = a.H / a.Hk;
  return core_launch(prec, Core{{a.q, a.ldq, 1}, {a.k, a.ldk, G}, {a.v, a.ldv, G}, a.o, a.ldo, 0, a.log_decay, a.lengths,
                                a.s0, a.sT, a.Dv, 1, a.B, a.T, a.H, a.Dk, a.Dv, 0, a.scale, 1.f}, (float*)ws, s);
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

// Query heads' own gradients of shared keys or values, then a pass's segment
// states.
static size_t group_bytes(int B, int T, int H, int Hk, int Dk, int Dv) {
  return H > Hk ? (((size_t)B * T * H * std::max(Dk, Dv) * 4 + 255) & ~(size_t)255) : 0;
}
size_t linattn_bwd_workspace(int prec, int B, int T, int H, int Hk, int Dk, int Dv) {
  return group_bytes(B, T, H, Hk, Dk, Dv) +
         std::max(split_bytes(prec, B, T, H, Dv, Dk), split_bytes(prec, B, T, H, Dk, Dv));
}

int linattn_bwd_launch(int prec, const LinattnBwd& a, void* ws, hipStream_t s) {
  const int G = a.H / a.Hk;
  float *part = (float*)ws, *states = (float*)((char*)ws + group_bytes(a.B, a.T, a.H, a.Hk, a.Dk, a.Dv));
  const Operand q{a.q, a.ldq, 1}, k{a.k, a.ldk, G}, v{a.v, a.ldv, G}, d{a.dout, a.lddout, 1};
  // dq and dk: on the state's transpose, whose elements are taken the other way round
  int r = core_launch(prec, Core{d, v, k, a.dq, a.lddq, 0, a.log_decay, a.lengths, a.s0, nullptr, 1, a.Dv, a.B, a.T,
                                 a.H, a.Dv, a.Dk, 0, a.scale, 1.f}, states, s);
  if (r) return r;
  r = core_launch(prec, Core{v, d, q, G > 1 ? part : a.dk, a.lddk, G > 1, a.log_decay, a.lengths, a.dsT, nullptr, 1,
                             a.Dv, a.B, a.T, a.H, a.Dv, a.Dk, 1, 1.f, a.scale}, states, s);
  if (r || (G > 1 && (r = group_sum_launch(prec, part, a.dk, a.lddk, a, a.Dk, s)))) return r;
  r = core_launch(prec, Core{k, q, d, G > 1 ? part : a.dv, a.lddv, G > 1, a.log_decay, a.lengths, a.dsT, a.ds0, a.Dv, 1,
                             a.B, a.T, a.H, a.Dk, a.Dv, 1, 1.f, a.scale}, states, s);
  return r || G == 1 ? r : group_sum_launch(prec, part, a.dv, a.lddv, a, a.Dv, s);
}

}  // namespace rn18

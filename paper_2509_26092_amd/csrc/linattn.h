// The chunked form of linear attention with a decay for each head: operands,
// kernel and choice of kernel (linattn.hip has the operators made of it; each
// storage type's kernels are compiled apart).
#pragma once
#include <math.h>

#include <type_traits>

#include "rows.h"

namespace rn18 {

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
  float* states;   // of segments, element (m, n) at m * st_m + n * st_n
  int st_m, st_n;
};
// Passes of one launch, which share their sizes' class (see shape_of): `n` of
// them, whose first `sums` leave the states that a segment starts from.
constexpr int kPasses = 3;
struct Cores {
  Core c[kPasses];
  int n, sums;
};

// A call's split: segments of a sequence, chunks of a segment.
struct Split {
  int nseg, chunks;
};
// A pass's kernel: rows of the state, waves of a block (32 columns each; eight
// waves of 256 rows would not fit in the registers), and WIDTHS (below).
struct Shape {
  int rows, waves, widths;
  bool operator==(const Shape& o) const { return rows == o.rows && waves == o.waves && widths == o.widths; }
};
inline Shape shape_of(int prec, const Core& c) {
  const int vw = prec_vw(prec), rows = c.M <= 64 ? 64 : c.M <= 128 ? 128 : 256;
  return Shape{rows, c.N <= 64 ? 2 : c.N <= 128 || rows == 256 ? 4 : 8,
               std::min(c.M, c.N) < vw ? 2 : c.M % vw || c.N % vw ? 1 : 0};
}
// What the segments before each one leave of the state, in place of their sums.
int segments_launch(const Cores& cs, const Split& p, hipStream_t s);
int chunks_launch_fp32(const Cores& cs, const Split& p, hipStream_t s);
int chunks_launch_bf16(const Cores& cs, const Split& p, hipStream_t s);
int chunks_launch_fp16(const Cores& cs, const Split& p, hipStream_t s);

namespace {

// What n tokens leave of a state, decay^n of it: as x + (decay^n - 1) x where most
// of it stays, since the factor's rounding would add up over many such steps, and
// as decay^n x where little does, which the difference would round away.
struct Kept {
  float factor;
  bool by_rest;
  __device__ inline float operator()(float x) const { return fmaf(x, factor, by_rest ? x : 0.f); }
};
__device__ inline Kept kept(int n, float g) {
  const float t = n > 0 ? (float)n * g : 0.f;
  const bool by_rest = t > -0.69f;
  return Kept{by_rest ? expm1f(t) : expf(t), by_rest};
}

// Tokens of sequence b.
__device__ inline int seq_len(const Core& c, int b) {
  return c.lengths ? min(max(c.lengths[b], 0), c.T) : c.T;
}

// ------------------------------------------------------------------ chunks on the matrix units
// A sequence is taken in chunks of 32 tokens. With X the state before a chunk
// of n tokens and i, j its tokens,
//   out_i = decay^(i + 1 - rev) X^T q_i + sum_(j <= i) decay^(i - j) (q_i . k_j) v_j
//   X <- decay^n X + sum_j decay^(n - 1 + rev - j) k_j v_j^T
// (the second terms of both with kv_scale). No power is above one for a decay
// below one, and none infinite for a growth of up to exp(2.5) a token. (Beyond it
// shorter chunks, or such heads token by token in a branch of their own, would do:
// measured, 3 to 15% of every head's time in fp16, whose registers are full.) A wave
// takes 16 NT columns of a head's state through the chunks: X stays in the
// accumulators of the matrix units, and so do the scores: what comes out of one
// product, rows 4 (lane / 16) + 0..3 of each 16, is an operand of the next whose
// inner index goes over these rows, if the other operand is read in the same order. Only q, k and v pass through LDS, q and k once for
// the W waves of a block, which share a head. The next chunk's rows are loaded
// into registers meanwhile.
//
// Matrix operands in 16 bits are bf16, which has fp32's range: fp16 inputs are
// held as two parts each (exact), what is computed in fp32 (X, the scores, the
// decayed v) as two or three. Products of parts below 2^-16 of the result are
// left out, for the state 2^-24.
//
// Bound by the vector units (parts of X and the scores, decay of X), the matrix
// units and memory, which two waves of a SIMD overlap only in part. bf16 forward:
// 256x196 tokens, 8 heads of 64, 66 us for 239 MB of HBM (3.6 TB/s of a copy's
// 5.2); 1x65537, 16 heads of 128, 340 us for 1.1 GB (the vector units are busy for
// 48% of that, the matrix units for 31%) after 140 us for the segments' sums (561
// MB, 4.0 TB/s); bf16 backward of the first, three passes, 140 us for 455 MB.
// Other ways are given below and there as a share of the same case's time in the
// kernel of their day, measured side by side. Slower or no faster: three waves of a
// SIMD (X leaves no room for them in the registers), loads two chunks ahead (19%
// more for the first), rows in LDS 8 or 12 banks further each, tables of the powers
// in LDS, a higher priority of waves that load (all equal).

// A lane's operand of one step over KB of the inner index, in NP parts: places
// 4 (lane / 16) + 0..3 of the first and of the second 16 in 16 bits, of 16 in
// fp32 (four steps of the unit).
template <int P> struct Frag { uint4 p[P]; };

template <int P> struct Ops16 {
  typedef bf16_t lds_t;
  static constexpr int NP = P, KB = 32, EV = 8;
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
  // The leading parts of two values of one sum, which keep the rest (exact: one
  // product with -1 and one with 0 each, in place of a shift or mask and a
  // difference; so what is not finite reaches the other value).
  // The factors go through registers: as literals, {-1, 0} was encoded as an
  // inline constant that the unit reads as {0, -1}.
  __device__ static inline uint32_t take(float& a, float& b) {
    uint32_t first = 0x0000bf80u, second = 0xbf800000u;
    asm("" : "+s"(first), "+s"(second));
    const uint32_t h = f2bf2(a, b);
    const bf16x2_t p = __builtin_bit_cast(bf16x2_t, h);
    a = __builtin_amdgcn_fdot2_f32_bf16(p, __builtin_bit_cast(bf16x2_t, first), a, false);
    b = __builtin_amdgcn_fdot2_f32_bf16(p, __builtin_bit_cast(bf16x2_t, second), b, false);
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
  // x, or NaN if one of the operand's values is not finite (products with 0).
  __device__ static inline float not_finite(const In& f, float x) {
    const uint32_t w[4] = {f.p[0].x, f.p[0].y, f.p[0].z, f.p[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      x = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w[i]), bf16x2_t{(__bf16)0.f, (__bf16)0.f}, x, false);
    return x;
  }
  // Zeros in place of what is not finite.
  __device__ static inline void clean(In& f) {
    auto word = [](uint32_t& w) {
      if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
      if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu;
    };
#pragma unroll
    for (int n = 0; n < P; ++n) {
      word(f.p[n].x);
      word(f.p[n].y);
      word(f.p[n].z);
      word(f.p[n].w);
    }
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
  static constexpr int NP = 1, KB = 16, EV = 4;
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
  __device__ static inline float not_finite(const In& f, float x) {
    const floatx4_t v = __builtin_bit_cast(floatx4_t, f.p[0]);
#pragma unroll
    for (int i = 0; i < 4; ++i) x = fmaf(v[i], 0.f, x);
    return x;
  }
  __device__ static inline void clean(In& f) {
    auto word = [](uint32_t& w) {
      if ((w & 0x7f800000u) == 0x7f800000u) w = 0;
    };
    word(f.p[0].x);
    word(f.p[0].y);
    word(f.p[0].z);
    word(f.p[0].w);
  }
  __device__ static inline void values(const In& f, float (&v)[4]) { unpack<float>(f.p[0], v); }
};
template <typename T> struct OpsOf { typedef Ops32 type; };
template <> struct OpsOf<bf16_t> { typedef Ops16<1> type; };
template <> struct OpsOf<f16_t> { typedef Ops16<2> type; };

typedef short v4i16_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char_t;

constexpr int kChunk = 32;

template <typename T, int MP, int NT, int W>
struct Tile {
  typedef typename OpsOf<T>::type O;
  typedef typename O::lds_t L;
  static constexpr int NP = O::NP, NB = 16 * NT * W, PAD = 16 / (int)sizeof(L);
  static constexpr int LDM = MP + PAD, LDN = NB + PAD;              // (rows 4 banks further each)
  static constexpr int SQ = kChunk * LDM, SV = kChunk * LDN;        // of one part
  static constexpr int OFF_K = NP * SQ, OFF_V = 2 * NP * SQ;
  static constexpr int BYTES = (OFF_V + NP * SV) * (int)sizeof(L);
  static constexpr int WAVES = MP * NT > 256 ? 1 : 2;               // of a SIMD: X is MP NT / 4 registers
  static_assert(BYTES <= 163840 && BYTES % 16 == 0, "LDS");
};

// The 16 bytes of a row at p, its column `col`; zeros for columns from `width`
// on, and where the row is not there. A partial last chunk is read from before
// its place (see shift_part). (No branch stands around a load: the compiler
// would wait there for each.)
template <typename T, int WIDTHS>
__device__ inline uint4 load_part(const T* p, int col, int width, bool there) {
  constexpr int VW = TT<T>::VW;
  if (WIDTHS == 2) {
    T e[VW];
#pragma unroll
    for (int j = 0; j < VW; ++j) e[j] = *(there && col + j < width ? p + j : (const T*)&kNoChunk);
    uint4 q;
    __builtin_memcpy(&q, e, 16);
    return q;
  }
  const bool in = there && col < width;
  const int over = WIDTHS == 0 ? 0 : max(col + VW - width, 0);
  return load_chunk(in ? p - over : (const T*)&kNoChunk);
}
// The part in its place, once it is there (not at the load, which it would wait
// for).
template <typename T, int WIDTHS>
__device__ inline uint4 shift_part(const uint4& q, int col, int width) {
  if (WIDTHS != 1) return q;
  const int s = 8 * (int)sizeof(T) * max(col + TT<T>::VW - width, 0) & 127;
  const uint64_t lo = q.x | (uint64_t)q.y << 32, hi = q.z | (uint64_t)q.w << 32;
  const uint64_t l2 = s >= 64 ? hi >> (s & 63) : s ? lo >> s | hi << (64 - s) : lo, h2 = s >= 64 ? 0 : hi >> s;
  return make_uint4((uint32_t)l2, (uint32_t)(l2 >> 32), (uint32_t)h2, (uint32_t)(h2 >> 32));
}

// A chunk of 16 bytes into LDS: its parts, `step` elements apart.
template <typename T>
__device__ inline void put(typename OpsOf<T>::type::lds_t* p, int step, const uint4& q) {
  if constexpr (OpsOf<T>::type::NP == 1) {
    *(uint4*)p = q;
  } else {
    // (neighbours are of different columns: each part by itself)
    float v[8], w[8];
    unpack<T>(q, v);
    const uint4 lead = pack<bf16_t>(v);
    unpack<bf16_t>(lead, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] -= w[i];
    *(uint4*)p = lead;
    *(uint4*)(p + step) = pack<bf16_t>(v);
  }
}

// WIDTHS 0: M and N are whole chunks of 16 bytes, 1: a chunk at least each, 2: one
// of them is less.
template <typename T, int MP, int NT, int W, int WIDTHS, bool SUMS>
__global__ __launch_bounds__(64 * W, (Tile<T, MP, NT, W>::WAVES)) void linattn_chunk_kernel(Cores cs, Split p, int nb_n,
                                                                                           int heads) {
  const int nseg = p.nseg, chunks = p.chunks;
  typedef Tile<T, MP, NT, W> TI;
  typedef typename OpsOf<T>::type O;
  typedef typename O::lds_t L;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int C = kChunk, CT = C / 16, VW = TT<T>::VW, MT = MP / 16, KB = O::KB, KT = KB / 16, NP = O::NP;
  constexpr int PER_M = MP / VW, PER_N = TI::NB / VW, ROWS_M = 64 * W / PER_M, ROWS_N = 64 * W / PER_N;
  constexpr int NQ = ROWS_M > C ? 1 : C / ROWS_M, NV = C / ROWS_N;
  static_assert(ROWS_M * PER_M == 64 * W && ROWS_N * PER_N == 64 * W && (NQ * ROWS_M == C || NQ == 1) && NV * ROWS_N == C,
                "loads");
  __shared__ uint4 smem[TI::BYTES / 16];
  L* const sQ = (L*)smem;
  L* const sK = sQ + TI::OFF_K;
  L* const sV = sQ + TI::OFF_V;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, i0 = lane & 15,
            g = lane >> 4;
  // Blocks that share operands or lines of memory (`heads` of a token, a head's
  // columns, the launch's passes) go to one XCD next to each other, everything
  // else to the XCDs in turn: neighbours along a sequence too, so that short
  // sequences of a batch leave none of them idle.
  const int passes = SUMS ? cs.sums : cs.n, segs = SUMS ? p.nseg - 1 : p.nseg, mates = heads * nb_n * passes;
  const int turn = blockIdx.x >> 3, mate = turn % mates, unit = turn / mates * 8 + (blockIdx.x & 7);
  const Core c = cs.c[mate % passes];
  const int sets = c.H / heads;
  if (unit >= c.B * sets * segs) return;
  const int seg = unit % segs, set = unit / segs % sets, b = unit / segs / sets, nb = mate / passes % nb_n,
            h = set * heads + mate / passes / nb_n, bh = b * c.H + h;
  float* const seg_states = c.states;
  const int len = seq_len(c, b), t_first = seg * chunks * C, total = min(max(len - t_first, 0), chunks * C);
  const float g2 = c.log_decay[h] * kLog2e;
  auto pw = [&](int n) { return n <= 0 ? 1.f : __builtin_amdgcn_exp2f((float)n * g2); };
  const int n_wave = nb * TI::NB + w * 16 * NT;   // the wave's columns from here on
  const bool works = n_wave < c.N;
  // Column of place x of tile nt: two tiles take turns of four, so that a lane
  // ends up with eight neighbours of an output row.
  static_assert(NT % 2 == 0, "pairs of tiles");
  auto col_of = [](int nt, int x) { return 32 * (nt / 2) + 8 * (x >> 2) + 4 * (nt & 1) + (x & 3); };

  floatx4_t X[MT][NT];   // rows 16 mt + 4 g + r, column col_of(nt, i0)
  bool empty;            // X is zero
  {
    const bool stored = !SUMS && nseg > 1;
    const float* src = stored ? seg_states + ((long)bh * nseg + seg) * c.M * c.N : c.s_in + (long)bh * c.M * c.N;
    const int s_m = stored ? c.st_m : c.s_m, s_n = stored ? c.st_n : c.s_n;
    const bool any = !SUMS && (stored || c.s_in);
    empty = !any;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int m = 16 * mt + 4 * g + r, n = n_wave + col_of(nt, i0);
          X[mt][nt][r] = any && m < c.M && n < c.N ? src[(long)m * s_m + (long)n * s_n] : 0.f;
        }
  }

  // A thread's chunks of 16 bytes of an operand: ROWS_M or ROWS_N tokens apart.
  const long dir = c.rev ? -1 : 1, row0 = (long)b * c.T + (c.rev ? len - 1 - t_first : t_first);
  uint4 rq[SUMS ? 1 : NQ], rk[NQ], rv[NV];
  const int im = tid / PER_M, in_ = tid / PER_N, colm = tid % PER_M * VW, coln = tid % PER_N * VW;
  auto place = [&](const Operand& x, int width, int i, int col) {
    return (const T*)x.p + (row0 + dir * i) * x.ld + (long)(h / x.group) * width + col;
  };
  const T *pq = SUMS ? nullptr : place(c.q, c.M, im, colm), *pk = place(c.k, c.M, im, colm),
          *pv = place(c.v, c.N, in_, nb * TI::NB + coln);
  const long sq = dir * c.q.ld, sk = dir * c.k.ld, sv = dir * c.v.ld;   // a token's step
  auto fetch = [&](int left) __attribute__((always_inline)) {   // the next chunk, of which `left` tokens are there
#pragma unroll
    for (int s = 0; s < NQ; ++s) {
      const bool there = im + s * ROWS_M < (ROWS_M > C ? min(left, C) : left);
      if (!SUMS) rq[SUMS ? 0 : s] = load_part<T, WIDTHS>(pq + s * ROWS_M * sq, colm, c.M, there);
      rk[s] = load_part<T, WIDTHS>(pk + s * ROWS_M * sk, colm, c.M, there);
    }
#pragma unroll
    for (int s = 0; s < NV; ++s)
      rv[s] = load_part<T, WIDTHS>(pv + s * ROWS_N * sv, nb * TI::NB + coln, c.N, in_ + s * ROWS_N < left);
    if (!SUMS) pq += C * sq;
    pk += C * sk;
    pv += C * sv;
  };

  // operands from LDS: of a row, and of a column at place i0 of its tile
  auto frag_row = [&](const L* base, int row, int k0) {
    typename O::In f;
    const L* at = base + (row + i0) * TI::LDM + k0 + 4 * g;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      if constexpr (F32) {
        f.p[p] = *(const uint4*)at;
      } else {
        const uint2 x = *(const uint2*)(at + p * TI::SQ), y = *(const uint2*)(at + p * TI::SQ + 16);
        f.p[p] = make_uint4(x.x, x.y, y.x, y.y);
      }
    }
    return f;
  };
  // `col` and `spread`: 16 columns in a row, or by fours 8 apart
  auto frag_col = [&](const L* base, int ld, int part, int row, int col, int spread) {
    typename O::In f;
    if constexpr (F32) {
      float v[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = base[(row + 4 * g + r) * ld + col + spread * (i0 >> 2) + (i0 & 3)];
      f.p[0] = pack<float>(v);
    } else {
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const L* at = base + p * part + (row + 4 * g + (i0 >> 2)) * ld + col + spread * (i0 & 3);
        auto tr = [](const L* a) {
          return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                               (__attribute__((address_space(3))) v4i16_t*)(lds_char_t*)a));
        };
        const uint2 x = tr(at), y = tr(at + 16 * ld);
        f.p[p] = make_uint4(x.x, x.y, y.x, y.y);
      }
    }
    return f;
  };

  // powers of the decay that serve every chunk: of a score in a diagonal tile
  // and in the one below, of a token's place, and of what is left of a chunk
  // behind a token (anew for a partial last chunk)
  const float scale = c.kv_scale * c.out_scale;
  float diag[4], below[4], up[CT], tail[C / KB][O::EV];
  Kept less{};
  if (!SUMS) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      diag[r] = i0 < 4 * g + r ? 0.f : pw(i0 - 4 * g - r) * scale;
      below[r] = pw(16 + i0 - 4 * g - r) * scale;
    }
#pragma unroll
    for (int it = 0; it < CT; ++it) up[it] = pw(16 * it + i0 + 1 - c.rev) * c.out_scale;
  }
  auto tails = [&](int n) __attribute__((always_inline)) {
#pragma unroll
    for (int jb = 0; jb < C / KB; ++jb)
#pragma unroll
      for (int e = 0; e < O::EV; ++e)
        tail[jb][e] = pw(n - 1 + c.rev - (jb * KB + 16 * (e >> 2) + 4 * g + (e & 3))) * c.kv_scale;
    less = kept(n, c.log_decay[h]);
  };
  tails(C);
  const int col_out = n_wave + 8 * g;
  char* po = (char*)c.out + (c.out_f32 ? (((row0 + dir * i0) * c.H + h) * c.N + col_out) * 4
                                       : ((row0 + dir * i0) * c.ldo + (long)h * c.N + col_out) * (long)sizeof(T));
  const long so = dir * (c.out_f32 ? (long)c.H * c.N * 4 : c.ldo * (long)sizeof(T));

  // A chunk's results wait in registers for the next one's loads: stores are
  // counted with the loads behind them, and loads behind them would wait for
  // stores that have only just begun (a chunk then waited for its stores: 16% more
  // at 256x196 tokens, 8 heads of 64, bf16 forward).
  uint4 result[CT][NT / 2][2];
  int results = 0;   // tokens of the chunk that waits
  auto flush = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int it = 0; it < CT; ++it)
      if (16 * it + i0 < results) {
        char* row = po + 16 * it * so;
#pragma unroll
        for (int np = 0; np < NT / 2; ++np) {
          const int rest = c.N - col_out - 32 * np;
          if (F32 || c.out_f32) {
            float v[8];
            __builtin_memcpy(v, result[it][np], 32);
            float* o = (float*)row + 32 * np;
            if (rest >= 8) {
              __builtin_memcpy(o, v, 32);
            } else {
#pragma unroll
              for (int x = 0; x < 7; ++x)
                if (x < rest) o[x] = v[x];
            }
          } else {
            T* o = (T*)row + 32 * np;
            if (rest >= 8) {
              __builtin_memcpy(o, &result[it][np][0], 16);
            } else {
              T e[8];
              __builtin_memcpy(e, &result[it][np][0], 16);
#pragma unroll
              for (int x = 0; x < 7; ++x)
                if (x < rest) o[x] = e[x];
            }
          }
        }
      }
    po += C * so;
  };

  auto stage = [&]() __attribute__((always_inline)) {   // what has been fetched into LDS
#pragma unroll
    for (int s = 0; s < NQ; ++s) {
      const int at = (im + s * ROWS_M) * TI::LDM + colm;
      if (ROWS_M > C && im >= C) continue;   // (few rows for many threads)
      if (!SUMS) put<T>(sQ + at, TI::SQ, shift_part<T, WIDTHS>(rq[SUMS ? 0 : s], colm, c.M));
      put<T>(sK + at, TI::SQ, shift_part<T, WIDTHS>(rk[s], colm, c.M));
    }
#pragma unroll
    for (int s = 0; s < NV; ++s)
      put<T>(sV + (in_ + s * ROWS_N) * TI::LDN + coln, TI::SV, shift_part<T, WIDTHS>(rv[s], nb * TI::NB + coln, c.N));
  };
  const bool last_state = SUMS || (c.s_out && seg == nseg - 1);   // the state behind the last chunk is wanted

  auto chunk = [&](int left) __attribute__((always_inline)) {   // the chunk in LDS, of which `left` tokens are there
    if (!works) return;

    floatx4_t out[CT][NT], P[CT][CT];   // out^T: rows columns, columns tokens; P^T[it][jt]: rows j, columns i
    if constexpr (!SUMS) {
#pragma unroll
      for (int it = 0; it < CT; ++it) {
#pragma unroll
        for (int jt = 0; jt < CT; ++jt) P[it][jt] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) out[it][nt] = floatx4_t{0.f, 0.f, 0.f, 0.f};
      }
      // (one body for all of the inner index: 2% less than with a branch in each step,
      // 1x65537 tokens, 16 heads of 128, bf16 forward)
      auto products = [&](auto with_state) __attribute__((always_inline)) {
#pragma unroll
        for (int kb = 0; kb < MP / KB; ++kb) {
          typename O::In q[CT];
#pragma unroll
          for (int it = 0; it < CT; ++it) q[it] = frag_row(sQ, 16 * it, kb * KB);
#pragma unroll
          for (int jt = 0; jt < CT; ++jt) {
            const auto k = frag_row(sK, 16 * jt, kb * KB);
#pragma unroll
            for (int it = jt; it < CT; ++it) O::template mma<2>(P[it][jt], k, q[it]);
          }
          if constexpr (decltype(with_state)::value)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              float x[O::EV];
#pragma unroll
              for (int e = 0; e < O::EV; ++e) x[e] = X[kb * KT + e / 4][nt][e % 4];
              const typename O::Two A = O::template parts<2>(x);
#pragma unroll
              for (int it = 0; it < CT; ++it) O::template mma<2>(out[it][nt], A, q[it]);
            }
        }
      };
      if (empty) products(std::false_type());
      else products(std::true_type());
#pragma unroll
      for (int it = 0; it < CT; ++it) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          P[it][it][r] = i0 < 4 * g + r ? 0.f : P[it][it][r] * diag[r];
          if (it > 0) P[it][0][r] *= below[r];
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) out[it][nt] *= up[it];
      }
    }
    empty = false;

    typename O::In V[C / KB][NT];
    float bad = 0.f;   // NaN if one of the chunk's v is not finite
#pragma unroll
    for (int jb = 0; jb < C / KB; ++jb)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        V[jb][nt] = frag_col(sV, TI::LDN, TI::SV, jb * KB, w * 16 * NT + col_of(nt, 0), 8);
        if (!SUMS) bad = O::not_finite(V[jb][nt], bad);
      }
    if (left > C || last_state) {   // the state behind the chunk
      if (!less.by_rest)   // (then the sum below leaves X as it is)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) X[mt][nt] *= less.factor;
      const float rest = less.by_rest ? less.factor : 0.f;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int r = 0; r < 4; ++r) X[mt][nt][r] = fmaf(X[mt][nt][r], rest, X[mt][nt][r]);
#pragma unroll
      for (int jb = 0; jb < C / KB; ++jb) {
        typename O::In K[MT > 4 ? 1 : MT];   // few rows: their operands once for all columns, otherwise the other way round
        typename O::Three D[MT > 4 ? NT : 1];
        if (MT <= 4)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) K[MT > 4 ? 0 : mt] = frag_col(sK, TI::LDM, TI::SQ, jb * KB, 16 * mt, 4);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float v[O::EV];
          O::values(V[jb][nt], v);
#pragma unroll
          for (int e = 0; e < O::EV; ++e) v[e] *= tail[jb][e];
          D[MT > 4 ? nt : 0] = O::template parts<3>(v);
          if (MT <= 4)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) O::template mma<3>(X[mt][nt], K[MT > 4 ? 0 : mt], D[0]);
        }
        if (MT > 4)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            const auto k = frag_col(sK, TI::LDM, TI::SQ, jb * KB, 16 * mt, 4);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) O::template mma<3>(X[mt][nt], k, D[MT > 4 ? nt : 0]);
          }
      }
    }

    if constexpr (!SUMS) {
      // the sums within the chunk. (A NaN or an infinity of a later token must
      // not meet an earlier one's zero score: it is taken out, and makes the
      // column's results NaN from its token on.)
      const bool any_bad = __any(bad != 0.f);
      if (__builtin_expect(any_bad, 0))
#pragma unroll
        for (int jb = 0; jb < C / KB; ++jb)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) O::clean(V[jb][nt]);
#pragma unroll
      for (int it = 0; it < CT; ++it)
#pragma unroll
        for (int jb = 0; jb <= it / KT; ++jb) {
          float p[O::EV];
#pragma unroll
          for (int e = 0; e < O::EV; ++e) p[e] = P[it][jb * KT + e / 4][e % 4];
          const auto f = O::template parts<2>(p);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) O::template mma<2>(out[it][nt], V[jb][nt], f);
        }
      if (__builtin_expect(any_bad, 0))
#pragma unroll 1
        for (int j = 0; j < C; ++j)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const float v = TT<L>::to_f(sV[j * TI::LDN + w * 16 * NT + col_of(nt, 4 * g + x)]);
              if (v * 0.f != 0.f)
#pragma unroll
                for (int it = 0; it < CT; ++it)
                  if (j <= 16 * it + i0) out[it][nt][x] = __builtin_nanf("");
            }
#pragma unroll
      for (int it = 0; it < CT; ++it)
#pragma unroll
        for (int np = 0; np < NT / 2; ++np) {
          float v[8];
#pragma unroll
          for (int x = 0; x < 8; ++x) v[x] = out[it][2 * np + x / 4][x % 4];
          if (F32 || c.out_f32) {
            result[it][np][0] = pack<float>(v);
            result[it][np][1] = pack<float>(v + 4);
          } else {
            result[it][np][0] = pack<T>(v);
          }
        }
      results = left;
    }
  };

  // (Two places in LDS and one barrier a chunk were no faster: equal at 1x65537, 16
  // heads of 128, bf16 forward, 13% more at 256x196, 8 heads of 64.)
  if (total > 0) fetch(total);
  for (int left = total; left > 0; left -= C) {
    if (left < C) tails(left);
    __syncthreads();   // the last chunk is read
    stage();
    __syncthreads();
    if (results > 0) flush();
    if (left > C) fetch(left - C);
    chunk(left);
  }
  if (results > 0) flush();

  if (!works || (!SUMS && (!c.s_out || seg != nseg - 1))) return;
  float* to = SUMS ? seg_states + ((long)bh * nseg + seg) * c.M * c.N : c.s_out + (long)bh * c.M * c.N;
  const int s_m = SUMS ? c.st_m : c.s_m, s_n = SUMS ? c.st_n : c.s_n;
  int m0 = 4 * g;   // (where elements lie is found again, not kept from the start)
  asm volatile("" : "+v"(m0));
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int m = 16 * mt + m0 + r, n = n_wave + col_of(nt, i0);
        if (m < c.M && n < c.N) to[(long)m * s_m + (long)n * s_n] = X[mt][nt][r];
      }
}

template <typename T, int MP, int NT, int W, int WIDTHS>
int chunk_launch(const Cores& cs, const Split& p, hipStream_t s) {
  const Core& c = cs.c[0];
  const int nb = ceil_div(c.N, 16 * NT * W);
  // all heads of a token together where there are enough units to deal out so,
  // otherwise those that share keys and values. (256x196 tokens, 8 heads of 64,
  // bf16 forward: 73 us, those that share keys alone 75, backward 139 and 142; ragged
  // sequences in 22 segments, fp16 backward: one contiguous range of blocks an XCD 35%
  // more.)
  int mates = 1;
  for (int i = 0; i < cs.n; ++i) mates = std::max({mates, cs.c[i].q.group, cs.c[i].k.group});
  // Fewer of them where that leaves fewer than 64 units, which the XCDs share about
  // evenly: all heads of one sequence over one key head would be one unit on one XCD,
  // and seven of eight blocks of the grid empty. (us, with them all on one XCD and
  // so, bf16 backward: 1x2048 tokens, 128 heads of 128 over one 1572 and 361, 1x4096,
  // 64 of 256 over one 7527 and 1341, fp16 1x300, 32 of 128 over one 121 and 65; 8
  // units in place of 64 are slower where a few more than 8 come out: bf16 2x2000, 32
  // of 64 over 8 99 and 93.)
  auto heads = [&](int segs) {
    int h = (long)c.B * segs >= 64 ? c.H : mates;
    for (int f = 2; h > 1 && (long)c.B * (c.H / h) * segs < 64;) {
      if (h % f == 0) h /= f;
      else f = f * f > h ? h : f + 1;
    }
    return h;
  };
  auto grid = [&](int segs, int passes) {
    const int h = heads(segs);
    return dim3(ceil_div((long)c.B * (c.H / h) * segs, 8) * 8 * h * nb * passes);
  };
  if (p.nseg > 1 && cs.sums) {
    hipLaunchKernelGGL((linattn_chunk_kernel<T, MP, NT, W, WIDTHS, true>), grid(p.nseg - 1, cs.sums), dim3(64 * W), 0, s,
                       cs, p, nb, heads(p.nseg - 1));
    const int r = segments_launch(cs, p, s);
    if (r) return r;
  }
  hipLaunchKernelGGL((linattn_chunk_kernel<T, MP, NT, W, WIDTHS, false>), grid(p.nseg, cs.n), dim3(64 * W), 0, s, cs, p, nb,
                     heads(p.nseg));
  return launched();
}

// A wave takes 32 columns of the state: 64 were slower (14% at 256x196 tokens, 8
// heads of 64, bf16 forward, and 21% at 1x65537, 16 heads of 128: too few waves
// beside the vector units' work on X), and 16 too (23% and 39%: every wave computes
// the scores).
template <typename T, int WIDTHS>
int widths_launch(const Cores& cs, int rows, int waves, const Split& p, hipStream_t s) {
  auto go = [&](auto r) {
    constexpr int MP = decltype(r)::value;
    if (waves == 2) return chunk_launch<T, MP, 2, 2, WIDTHS>(cs, p, s);
    // (widths below a chunk of 16 bytes are M's or N's, so that not both are large)
    if constexpr (WIDTHS < 2 || MP == 64) {
      if (waves == 4) return chunk_launch<T, MP, 2, 4, WIDTHS>(cs, p, s);
      if constexpr (MP <= 128) return chunk_launch<T, MP, 2, 8, WIDTHS>(cs, p, s);
    }
    return -1;
  };
  if (rows == 64) return go(std::integral_constant<int, 64>());
  if (rows == 128) return go(std::integral_constant<int, 128>());
  return go(std::integral_constant<int, 256>());
}

template <typename T>
int chunks_launch(const Cores& cs, const Split& p, hipStream_t s) {
  const Shape h = shape_of(prec_of<T>(), cs.c[0]);
  if (h.widths == 0) return widths_launch<T, 0>(cs, h.rows, h.waves, p, s);
  if (h.widths == 1) return widths_launch<T, 1>(cs, h.rows, h.waves, p, s);
  return widths_launch<T, 2>(cs, h.rows, h.waves, p, s);
}

}  // namespace

}  // namespace rn18

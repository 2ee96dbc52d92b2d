// The distillation loss of a student against a teacher's top logits, with the
// gradient of the student's logits:
//   P = softmax(z / T), p = softmax(z), q = softmax of the teacher's valid
//   entries t / T
//   row_loss = w (alpha T^2 sum_k q_k (log q_k - log P_{i_k}) + (1 - alpha) (-log p_label))
//   dz_j = scale w (alpha T (P_j - sum_{k: i_k = j} q_k) + (1 - alpha) (p_j - [j = label]))
//
// z is read once into registers, its maximum and sums of exponentials are
// taken there, and dz is written from there: 4 bytes of traffic and two or
// four exponentials an element in 16 bits (four with labels, for alpha = 0
// too). Bound by memory without labels (16384x32768 bf16, 64 listed, 441 us,
// 4.9 TB/s), with labels by memory and the vector units together (4096x131071
// bf16 583 us, without 472). The few classes that the list or the label name
// are written a second time with their own terms, by the lane of the first
// entry that names each. With sum q = 1 the soft term is
// alpha T (sum_k q_k (t_k - z_k) + T (log sum e^z' - log sum e^t')), t and z
// less their maxima, t' and z' over T too, so that every sum of a row is taken
// in one step. The maxima are taken out before the division by T and the sum
// over the entries is multiplied by T once: no quotient by a small T, nor T^2,
// leaves fp32's range on the way.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "kernels.h"
#include "rows.h"

namespace rn18 {

namespace {

inline int ok() { return hipGetLastError() == hipSuccess ? 0 : -4; }

// 2^x by the hardware's instruction (1 ulp; 0 below 2^-126). e^-d is taken as
// 2^(-d log2(e)) with the product rounded to 32 bits: an exponential is off by
// up to about d 2^-24 of itself, and by d e^-d 2^-24, less than half a
// rounding, of the row's largest, which the sums and the gradient are added to.
// Against 64 bits the loss and gradient of 64x1000 fp32 rows are off by 0.9e-7,
// those of library exponentials and a division by T by 1.2e-7.
__device__ inline float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// The teacher's list of a row; -1 fills its classes up to a multiple of 4.
template <int KM>
struct alignas(16) Entries {
  int32_t cls[KM];   // -1: not valid
  float e[KM];       // t, then exp((t - the largest t) / T)
  float z[KM];       // the student's logit
  int32_t named;     // the label is one of the classes
};
// Of rows whose lanes are part of a wave: lists that sixteen rows of a block
// have room for.
constexpr int kShortList = 64;

// What can be loaded of a row's entries and label before the student's logits
// there: in flight ahead of the row's own chunks, it does not wait for them
// (4096x32768 bf16 115 -> 111 us, 16777x1000 27.1 -> 25.2, 64 listed).
struct First {
  int i, label;
  float t;
};
template <bool HARD>
__device__ inline First load_first(const DistillArgs& a, long r, int l) {
  First f = {-1, -1, -INFINITY};
  // (a step checks the labels whether or not its loss has a term for them)
  if (HARD || (a.err && a.labels)) f.label = a.labels[r];
  if (l < a.K) {
    f.i = a.t_idx[r * a.K + l];
    f.t = a.t_vals[r * a.K + l];
  }
  return f;
}

// A row's label and the student's logit there; every lane holds them. (As an
// entry after the others it cost lists of 64 a second round of every loop:
// 16777x1000 bf16 40.0 us in place of 31.3.)
struct Label {
  int cls;   // -1: none
  float z;
};
// zk: the student's logits of the K entries and the label, if they have been
// gathered before, or NULL.
template <typename T, bool HARD>
__device__ inline Label load_label(const DistillArgs& a, int l, const First& f, const T* zr, const float* zk) {
  const int i = f.label;
  if (HARD && i >= 0 && i < a.C) return {i, zk ? zk[a.K] : TT<T>::to_f(zr[i])};
  if (a.err && (i < -1 || i >= a.C) && l == 0) atomicOr(a.err, (unsigned)DEVERR_LABEL);
  return {-1, 0.f};
}

// Loads a row's entries. Returns the largest t.
template <typename T, int L, int KM>
__device__ inline float load_entries(const DistillArgs& a, long r, int l, const First& f, const T* zr,
                                     const float* zk, Entries<KM>& en) {
  float tm = -INFINITY;
  bool bad = false;
  for (int k = l; k < a.K; k += L) {
    int i = k == l ? f.i : a.t_idx[r * a.K + k];
    float t = k == l ? f.t : a.t_vals[r * a.K + k];
    bad |= i < -1 || i >= a.C;
    if (i < 0 || i >= a.C || t == -INFINITY || a.alpha == 0.f) {
      i = -1;
      t = -INFINITY;
    }
    en.cls[k] = i;
    en.e[k] = t;
    en.z[k] = i < 0 ? 0.f : zk ? zk[k] : TT<T>::to_f(zr[i]);
    tm = max2(tm, t);
  }
  if (l < ((4 - (a.K & 3)) & 3)) en.cls[a.K + l] = -1;
  if (l == 0) en.named = 0;
  if (a.err && bad) atomicOr(a.err, (unsigned)DEVERR_LABEL);
  return tm;
}

// A row's sums: of exp(z') and exp(z - m) over the classes, of e and of
// e (t - z) over the entries.
enum { SUM_T, SUM_1, SUM_Q, SUM_QD, SUMS };

template <int L, int KM>
__device__ inline void entry_sums(const DistillArgs& a, int l, float tm, float m, const Label& lab,
                                  Entries<KM>& en, float* s) {
  const float ct = kLog2e / a.temperature;
  for (int k = l; k < a.K; k += L) {
    const float t = en.e[k] - tm, e = en.cls[k] < 0 ? 0.f : exp2_hw(t * ct);
    en.e[k] = e;
    s[SUM_Q] += e;
    if (en.cls[k] >= 0 && en.cls[k] == lab.cls) en.named = 1;
    if (e != 0.f) s[SUM_QD] += e * (t - (en.z[k] - m));
  }
}

// What the gradient of a row needs: dz_j = exp(z') gt + exp(z - m) g1, less
// ft q and fh at the entries and the label.
struct RowGrad {
  float m, ct, gt, g1, fq, fh;
};
template <bool HARD>
__device__ inline RowGrad row_grad(const DistillArgs& a, float w, float m, const float* s, bool labelled) {
  const bool some = s[SUM_T] != 0.f;   // false: every class of the row is masked
  const bool soft = some && s[SUM_Q] != 0.f, hard = HARD && some && labelled;
  const float f = a.scale * w * (a.ls ? a.ls->scale : 1.0f);
  const float ft = f * a.alpha * a.temperature, fh = f * (1.0f - a.alpha);
  RowGrad g;
  g.m = m;
  g.ct = kLog2e / a.temperature;
  g.gt = soft ? ft / s[SUM_T] : 0.f;
  g.fq = soft ? ft / s[SUM_Q] : 0.f;
  g.g1 = hard ? fh / s[SUM_1] : 0.f;
  g.fh = hard ? fh : 0.f;
  return g;
}
template <bool HARD>
__device__ inline float grad_at(const RowGrad& g, float z) {
  const float d = z - g.m;
  float v = exp2_hw(d * g.ct) * g.gt;
  if (HARD) v += exp2_hw(d * kLog2e) * g.g1;
  return v;
}
template <bool HARD>
__device__ inline float row_loss_of(const DistillArgs& a, float w, const float* s, float m, float zlab, bool labelled) {
  const bool some = s[SUM_T] != 0.f;
  float v = 0.f;
  if (some && s[SUM_Q] != 0.f)
    v = a.alpha * a.temperature * (s[SUM_QD] / s[SUM_Q] + a.temperature * logf(s[SUM_T] / s[SUM_Q]));
  if (HARD && some && labelled) v += (1.0f - a.alpha) * (logf(s[SUM_1]) - (zlab - m));
  return w * v;
}

// The gradients of the classes [c0, c1) and [0, head) that entries name, each
// by the lane of the first entry that names it, and of the label.
template <typename T, int L, bool HARD, int KM>
__device__ inline void write_entries(const DistillArgs& a, int l, const RowGrad& g, const Label& lab,
                                     const Entries<KM>& en, T* dr, int c0, int c1, int head) {
  auto outside = [&](int at) { return at < 0 || (at >= head && (at < c0 || at >= c1)); };
  for (int k = l; k < a.K; k += L) {
    const int at = en.cls[k];
    // entries of the same class, itself among them: most lists have none
    int same = 0;
    for (int j = 0; j < a.K; j += 4) {
      const int4 c = *(const int4*)(en.cls + j);
      same += (c.x == at ? 1 : 0) + (c.y == at ? 1 : 0) + (c.z == at ? 1 : 0) + (c.w == at ? 1 : 0);
    }
    if (outside(at)) continue;
    float q = en.e[k];
    if (same > 1) {
      bool first = true;
      q = 0.f;
      for (int j = 0; j < a.K; ++j)
        if (en.cls[j] == at) {
          first &= j >= k;
          q += en.e[j];
        }
      if (!first) continue;
    }
    float v = grad_at<HARD>(g, en.z[k]);
    if (g.fq != 0.f) v -= g.fq * q;   // (a row without a soft term: q may be anything)
    if (HARD && at == lab.cls) v -= g.fh;
    dr[at] = TT<T>::from_f(v);
  }
  if (HARD && l == L - 1 && !outside(lab.cls) && !en.named)
    dr[lab.cls] = TT<T>::from_f(grad_at<HARD>(g, lab.z) - g.fh);
}

// One row in the registers of L lanes, E chunks each; the elements before the
// first chunk and after the last are one to a lane. (Chunks at the row's own
// address, which an odd class count leaves unaligned: 10737x50001 bf16 528 us
// in place of 415.)
template <typename T, int L, int E, bool HARD>
__global__ __launch_bounds__(L > 256 ? L : 256) void distill_row_kernel(DistillArgs a) {
  constexpr int VW = TT<T>::VW, NT = L > 256 ? L : 256, G = NT / L, KM = L < 64 ? kShortList : kTopMax;
  __shared__ Entries<KM> entries[G];
  __shared__ float shm[L > 64 ? L / 64 : 1][2], shs[L > 64 ? L / 64 : 1][SUMS];
  const int grp = L < NT ? threadIdx.x / L : 0;
  Entries<KM>& en = entries[grp];
  // (L < NT: a wave or part of one has its own rows, and nothing waits for
  // another's; the lanes of a row leave the loop and skip a row together)
  for (long r = (long)blockIdx.x * G + grp; r < a.R; r += (long)gridDim.x * G) {
    int l = threadIdx.x % L;
    asm volatile("" : "+v"(l));   // offsets are computed where they are needed, not kept over the rows
    const T* zr = (const T*)a.z + r * a.ldz;
    T* dr = a.dz ? (T*)a.dz + r * a.lddz : nullptr;
    const int head = row_head(zr, a.C), nch = (a.C - head) / VW;
    const int tail = l < head ? l : nch * VW + l;
    const float w = a.weight ? a.weight[r] : 1.0f;
    if (w == 0.f) {   // the row may hold anything: not read
      if (l == 0) a.row_loss[r] = 0.f;
      if (dr) {
        for (int c = l; c < nch; c += L) store_chunk(dr + head + c * VW, make_uint4(0, 0, 0, 0));
        if (tail < a.C) dr[tail] = TT<T>::from_f(0.f);
      }
      continue;
    }
    const First first = load_first<HARD>(a, r, l);
    uint4 q[E];
    const T* zc = chunk_base(zr + head, nch);
#pragma unroll
    for (int e = 0; e < E; ++e) q[e] = load_chunk_at(zc, (e * L + l < nch ? e * L + l : 0) * 16u);
    const float zt = tail < a.C ? TT<T>::to_f(zr[tail]) : -INFINITY;
    const Label lab = load_label<T, HARD>(a, l, first, zr, nullptr);
    float mx[2] = {zt, load_entries<T, L>(a, r, l, first, zr, nullptr, en)};
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float v[VW];
      unpack<T>(q[e], v);
      if (e * L + l < nch) mx[0] = max2(mx[0], chunk_max<VW>(v));
      opaque(q[e]);
      __builtin_amdgcn_sched_barrier(0);   // one chunk's values at a time in registers
    }
    row_red<L>(mx, shm, Max());
    const float m = mx[0] == -INFINITY ? 0.f : mx[0], tm = mx[1] == -INFINITY ? 0.f : mx[1];
    const float ct = kLog2e / a.temperature;
    float s[SUMS] = {exp2_hw((zt - m) * ct), HARD ? exp2_hw((zt - m) * kLog2e) : 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float v[VW];
      unpack<T>(q[e], v);
      if (e * L + l < nch) {
#pragma unroll
        for (int j = 0; j < VW; ++j) {
          const float d = v[j] - m;
          s[SUM_T] += exp2_hw(d * ct);
          if (HARD) s[SUM_1] += exp2_hw(d * kLog2e);
        }
      }
      opaque(q[e]);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (L <= 64) row_sync<L>();
    entry_sums<L>(a, l, tm, m, lab, en, s);
    row_red<L>(s, shs, Sum());
    if (L <= 64) row_sync<L>();
    const bool labelled = lab.cls >= 0;
    if (l == 0) a.row_loss[r] = row_loss_of<HARD>(a, w, s, m, lab.z, labelled);
    if (dr) {
      const RowGrad g = row_grad<HARD>(a, w, m, s, labelled);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float v[VW];
        unpack<T>(q[e], v);
#pragma unroll
        for (int j = 0; j < VW; ++j) v[j] = grad_at<HARD>(g, v[j]);
        if (e * L + l < nch) store_chunk_at(dr + head, (e * L + l) * 16u, pack<T>(v));
        __builtin_amdgcn_sched_barrier(0);
      }
      if (tail < a.C) dr[tail] = TT<T>::from_f(grad_at<HARD>(g, zt));
      row_sync<L>();   // the named classes are written after the rest
      write_entries<T, L, HARD>(a, l, g, lab, en, dr, 0, a.C, 0);
    }
    row_sync<L>();   // before the next row's entries
  }
}

// Rows in parts, a block of 256 threads each: the first launch leaves each
// part's maximum and sums, and the student's logits of the row's entries, the
// second joins them and writes the gradient of its part.
//   ws[row]: (m, sum exp(z'), sum exp(z - m), -) of each part, then the K + 1 logits
struct Parts {
  float* ws;
  int n, chunks;   // parts of a row, chunks of a part
  __host__ __device__ long row_floats(int K) const { return 4l * n + K + 1; }
};

constexpr int kPartE = 4;   // chunks of a lane in flight

template <typename T, bool HARD>
__global__ __launch_bounds__(256) void distill_part_stats_kernel(DistillArgs a, Parts ps) {
  constexpr int VW = TT<T>::VW, L = 256;
  __shared__ Entries<kTopMax> en;
  __shared__ float shm[L / 64][1], shs[L / 64][2];
  const int l = threadIdx.x, c0 = (int)blockIdx.x * ps.chunks;
  const bool last = (int)blockIdx.x == ps.n - 1;
  const float ct = kLog2e / a.temperature;
  for (long r = blockIdx.y; r < a.R; r += gridDim.y) {
    if (a.weight && a.weight[r] == 0.f) continue;
    const T* zr = (const T*)a.z + r * a.ldz;
    const int head = row_head(zr, a.C), nch = (a.C - head) / VW, c1 = std::min(nch, c0 + ps.chunks);
    const T* zc = zr + head;
    float* wr = ps.ws + r * ps.row_floats(a.K);
    if (blockIdx.x == 0) {
      const First first = load_first<HARD>(a, r, l);
      load_entries<T, L>(a, r, l, first, zr, nullptr, en);
      for (int k = l; k < a.K; k += L) wr[4 * ps.n + k] = en.z[k];   // the lane's own entries
      const Label lab = load_label<T, HARD>(a, l, first, zr, nullptr);
      if (HARD && l == 0) wr[4 * ps.n + a.K] = lab.z;
    }
    const int tail = l < head ? l : nch * VW + l;   // (the last part has the head too)
    // a running maximum of the lane, and its sums relative to it
    float m = last && tail < a.C ? TT<T>::to_f(zr[tail]) : -INFINITY;
    float s[2] = {m == -INFINITY ? 0.f : 1.f, HARD && m != -INFINITY ? 1.f : 0.f};
    if (m != m) s[0] = s[1] = m;
    for (int b = c0 + l; b < c1; b += L * kPartE) {
      uint4 q[kPartE];
      float v[kPartE][VW], top = m;
#pragma unroll
      for (int e = 0; e < kPartE; ++e) q[e] = load_chunk(zc + (long)std::min(b + e * L, c1 - 1) * VW);
#pragma unroll
      for (int e = 0; e < kPartE; ++e) {
        unpack<T>(q[e], v[e]);
        top = max2(top, chunk_max<VW>(v[e]));   // (a chunk past the part is one of the part)
      }
      if (top == -INFINITY) continue;
      if (top != m) {
        s[0] *= exp2_hw((m - top) * ct);
        s[1] *= exp2_hw((m - top) * kLog2e);
        m = top;
      }
#pragma unroll
      for (int e = 0; e < kPartE; ++e)
        if (b + e * L < c1)
#pragma unroll
          for (int j = 0; j < VW; ++j) {
            s[0] += exp2_hw((v[e][j] - m) * ct);
            if (HARD) s[1] += exp2_hw((v[e][j] - m) * kLog2e);
          }
    }
    float mx[1] = {m};
    row_red<L>(mx, shm, Max());
    const float all = mx[0] == -INFINITY ? 0.f : mx[0];
    if (m == -INFINITY) m = all;   // sums of zero
    s[0] *= exp2_hw((m - all) * ct);
    s[1] *= exp2_hw((m - all) * kLog2e);
    row_red<L>(s, shs, Sum());
    if (l == 0) {
      float* o = wr + 4 * blockIdx.x;
      o[0] = mx[0];
      o[1] = s[0];
      o[2] = s[1];
    }
    __syncthreads();   // before the next row's entries and reductions
  }
}

template <typename T, bool HARD>
__global__ __launch_bounds__(256) void distill_part_grad_kernel(DistillArgs a, Parts ps) {
  constexpr int VW = TT<T>::VW, L = 256;
  __shared__ Entries<kTopMax> en;
  __shared__ float shm[L / 64][2], shs[L / 64][SUMS];
  const int l = threadIdx.x, c0 = (int)blockIdx.x * ps.chunks;
  const bool last = (int)blockIdx.x == ps.n - 1;
  const float ct = kLog2e / a.temperature;
  for (long r = blockIdx.y; r < a.R; r += gridDim.y) {
    const T* zr = (const T*)a.z + r * a.ldz;
    T* dr = a.dz ? (T*)a.dz + r * a.lddz : nullptr;
    const int head = row_head(zr, a.C), nch = (a.C - head) / VW, c1 = std::min(nch, c0 + ps.chunks);
    const float w = a.weight ? a.weight[r] : 1.0f;
    const int mine = l < head ? l : nch * VW + l, tail = last && mine < a.C ? mine : -1;
    if (w == 0.f) {
      if (blockIdx.x == 0 && l == 0) a.row_loss[r] = 0.f;
      if (dr) {
        for (int c = c0 + l; c < c1; c += L) store_chunk(dr + head + (long)c * VW, make_uint4(0, 0, 0, 0));
        if (tail >= 0) dr[tail] = TT<T>::from_f(0.f);
      }
      continue;
    }
    const float* wr = ps.ws + r * ps.row_floats(a.K);
    const First first = load_first<HARD>(a, r, l);
    const Label lab = load_label<T, HARD>(a, l, first, zr, wr + 4 * ps.n);
    float mx[2] = {-INFINITY, load_entries<T, L>(a, r, l, first, zr, wr + 4 * ps.n, en)};
    for (int p = l; p < ps.n; p += L) mx[0] = max2(mx[0], wr[4 * p]);
    row_red<L>(mx, shm, Max());
    const float m = mx[0] == -INFINITY ? 0.f : mx[0], tm = mx[1] == -INFINITY ? 0.f : mx[1];
    float s[SUMS] = {};
    for (int p = l; p < ps.n; p += L) {
      const float mp = wr[4 * p];
      if (mp == -INFINITY) continue;
      s[SUM_T] += wr[4 * p + 1] * exp2_hw((mp - m) * ct);
      if (HARD) s[SUM_1] += wr[4 * p + 2] * exp2_hw((mp - m) * kLog2e);
    }
    entry_sums<L>(a, l, tm, m, lab, en, s);
    row_red<L>(s, shs, Sum());
    const bool labelled = lab.cls >= 0;
    if (blockIdx.x == 0 && l == 0) a.row_loss[r] = row_loss_of<HARD>(a, w, s, m, lab.z, labelled);
    if (dr) {
      const RowGrad g = row_grad<HARD>(a, w, m, s, labelled);
      for (int b = c0 + l; b < c1; b += L * kPartE) {
        uint4 q[kPartE];
#pragma unroll
        for (int e = 0; e < kPartE; ++e)
          if (b + e * L < c1) q[e] = load_chunk(zr + head + (long)(b + e * L) * VW);
#pragma unroll
        for (int e = 0; e < kPartE; ++e)
          if (b + e * L < c1) {
            float v[VW];
            unpack<T>(q[e], v);
#pragma unroll
            for (int j = 0; j < VW; ++j) v[j] = grad_at<HARD>(g, v[j]);
            store_chunk(dr + head + (long)(b + e * L) * VW, pack<T>(v));
          }
      }
      if (tail >= 0) dr[tail] = TT<T>::from_f(grad_at<HARD>(g, TT<T>::to_f(zr[tail])));
      __syncthreads();   // the named classes are written after the rest
      write_entries<T, L, HARD>(a, l, g, lab, en, dr, head + c0 * VW, last ? a.C : head + c1 * VW, last ? head : 0);
    }
    __syncthreads();
  }
}

// loss = scale * sum of the row losses, added in 64 bits in a fixed order.
__global__ __launch_bounds__(1024) void distill_loss_kernel(const float* __restrict__ row_loss, long R, float scale,
                                                            float* __restrict__ loss, unsigned* err) {
  __shared__ double sh[16];
  double v = 0.0;
#pragma unroll 4
  for (long i = threadIdx.x; i < R / 4; i += 1024) {
    float x[4];
    __builtin_memcpy(x, row_loss + 4 * i, 16);
    v += ((double)x[0] + (double)x[1]) + ((double)x[2] + (double)x[3]);
  }
  if ((long)threadIdx.x < R % 4) v += (double)row_loss[R / 4 * 4 + threadIdx.x];
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 16; ++i) v += sh[i];
    const float f = (float)(v * (double)scale);
    loss[0] = f;
    if (err && !isfinite(f)) atomicOr(err, (unsigned)DEVERR_NONFINITE);
  }
}

// ------------------------------------------------------------------ choice of kernel
// Parts of a row (1: none): for rows beyond a block's registers, and for up
// to a row for every fourth compute unit, of more than 4096 chunks, which
// alone take longer than the launch that joins parts (one row of 131072 bf16
// logits: 12.9 us in parts, 19.4 whole, 64 of them 18.2 and 25.9; of 32768:
// 12.5 and 10.7; 128 rows of 65536: 20.6 and 19.9).
Parts distill_parts(int prec, long R, int C, float* ws) {
  const int nch = C / prec_vw(prec), cus = plan_cus();
  int n = 1;
  if (nch > 16384) n = ceil_div(nch, 8192);
  if (nch > 4096 && R * 4 <= cus) n = std::max(n, std::min(nch / 512, ceil_div(2l * cus, std::max(R, 1l))));
  n = std::min(n, 4096);
  const int chunks = ceil_div(std::max(nch, 1), n);
  return {ws, ceil_div(std::max(nch, 1), chunks), chunks};
}

template <typename T, bool HARD>
int distill_go(const DistillArgs& a, const Parts& ps, hipStream_t s) {
  if (ps.n > 1) {
    const dim3 grid(ps.n, (unsigned)std::min(a.R, 65535l));
    hipLaunchKernelGGL((distill_part_stats_kernel<T, HARD>), grid, dim3(256), 0, s, a, ps);
    hipLaunchKernelGGL((distill_part_grad_kernel<T, HARD>), grid, dim3(256), 0, s, a, ps);
    return ok();
  }
  const int nch = a.C / TT<T>::VW;
  auto go = [&](auto l, auto e) {
    constexpr int L = decltype(l)::value, NT = L > 256 ? L : 256, G = NT / L;
    hipLaunchKernelGGL((distill_row_kernel<T, L, decltype(e)::value, HARD>),
                       dim3((unsigned)std::min((a.R + G - 1) / G, 1l << 22)), dim3(NT), 0, s, a);
    return ok();
  };
#define GO(L, E) return go(std::integral_constant<int, L>{}, std::integral_constant<int, E>{})
  // Many short rows: sixteen lanes a row, so that four rows share what a wave
  // spends on sums and entries, unless entries are most of the work
  // (167772x100 bf16, 20 listed: 49 us, with a wave a row 119; 64 listed: 88
  // and 140; 55924x300: 46 and 53; 33554x500, 20 listed: 26 and 31, 64: 45
  // and 36).
  if (nch <= 64 && a.K <= kShortList && nch * a.K <= 2400 && a.R >= 8l * plan_cus()) {
    if (nch <= 16) GO(16, 1);
    if (nch <= 32) GO(16, 2);
    GO(16, 4);
  }
  if (nch <= 512 && a.R >= 4l * plan_cus()) {
    if (nch <= 64) GO(64, 1);
    if (nch <= 128) GO(64, 2);
    if (nch <= 256) GO(64, 4);
    GO(64, 8);
  }
  if (nch <= 256) GO(256, 1);
  if (nch <= 512) GO(256, 2);
  if (nch <= 1024) GO(256, 4);
  if (nch <= 2048) GO(256, 8);
  if (nch <= 4096) GO(512, 8);
  if (nch <= 8192) GO(512, 16);
  GO(1024, 16);
#undef GO
}

}  // namespace

size_t distill_workspace(int prec, long R, int C, int K) {
  const Parts ps = distill_parts(prec, R, C, nullptr);
  return ps.n > 1 && R > 0 ? (size_t)R * ps.row_floats(K) * 4 : 0;
}

int distill_launch(int prec, const DistillArgs& a, float* loss, void* ws, hipStream_t s) {
  if (a.R > 0) {
    const Parts ps = distill_parts(prec, a.R, a.C, (float*)ws);
    const int r = with_prec(prec, [&](auto tag) {
      using T = decltype(tag);
      return a.labels && a.alpha != 1.0f ? distill_go<T, true>(a, ps, s) : distill_go<T, false>(a, ps, s);
    });
    if (r) return r;
  }
  if (loss) {
    hipLaunchKernelGGL(distill_loss_kernel, dim3(1), dim3(1024), 0, s, a.row_loss, a.R, a.scale, loss, a.err);
    return ok();
  }
  return 0;
}

}  // namespace rn18

// The K largest logits of a row with their classes, in descending order, ties
// in the order of the classes.
//
// A row is read once, into the registers of L lanes. The K-th largest of the
// lanes' own maxima is a bound that at least K logits reach and few more do
// (about K^2 / 2L of a random row), so one compare against it leaves a short
// list, and counting for each entry of the list how many others precede it
// gives its place. The work beyond the one pass over the row is small, and
// the pass is bound by memory. Where more logits reach the bound than the list holds
// (equal logits: masked rows; rows whose large logits crowd in few lanes), a
// bisection over the order of the values, counted over the row, finds a bound
// that fits or the value that all the surplus shares, of which the first
// classes are taken.
#include <math.h>

#include <algorithm>

#include "kernels.h"
#include "rows.h"

namespace rn18 {

namespace {

inline int ok() { return hipGetLastError() == hipSuccess ? 0 : -4; }

// Order-preserving unsigned key of a float: larger value, larger key; the
// two zeros share a key and every NaN has the largest one. 0 is no value's.
__device__ inline uint32_t order_key(float v) {
  if (v != v) return 0xfffffffeu;
  const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.0f);   // -0 + 0 = +0
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
// The value of a key whose bits below the type's are cut to zero.
template <typename T>
__device__ inline float key_value(uint32_t k) {
  constexpr uint32_t low = prec_of<T>() == PREC_BF16 ? 0xffffu : prec_of<T>() == PREC_F16 ? 0x1fffu : 0u;
  return __builtin_bit_cast(float, k & 0x80000000u ? k & 0x7fffffffu : ~(k | low));
}
template <typename T>
__device__ constexpr int key_bits() {   // leading bits of a key that tell values of the type apart
  return prec_of<T>() == PREC_BF16 ? 16 : prec_of<T>() == PREC_F16 ? 19 : 32;
}

// max(a, b, c) in one instruction. A NaN may drop out with what it meets:
// the result is a number of the row or a NaN.
__device__ inline float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// The K-th largest of the 64 * PER keys that a wave holds, cut to `bits`
// leading bits; 0 if there are fewer.
template <int PER>
__device__ inline uint32_t kth_key(const uint32_t (&k)[PER], int K, int bits) {
  uint32_t t = 0;
  for (int b = 31; b >= 32 - bits; --b) {
    const uint32_t c = t | 1u << b;
    int n = 0;
#pragma unroll
    for (int p = 0; p < PER; ++p) n += __popcll(__ballot(k[p] >= c));
    if (n >= K) t = c;
  }
  return t;
}

template <int L>
struct TopShared {
  static constexpr int M = L > 64 ? 2048 : 256;   // entries of the list
  uint64_t list[M];
  uint32_t keys[L];
  uint32_t count, bound;
  int part[16];
};

// Between writes and reads of the row's shared memory.
template <int L>
__device__ inline void row_sync() {
  if (L > 64) {
    __syncthreads();
  } else {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// Sum over the row's lanes, and the sum over the lanes before this one.
template <int L>
__device__ inline int row_count(int n, int* before, TopShared<L>& sh) {
  const int lane = threadIdx.x & 63;
  int inc = n;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(inc, o);
    if (lane >= o) inc += up;
  }
  int base = 0, total = __shfl(inc, 63);
  if (L > 64) {
    const int w = threadIdx.x >> 6;
    __syncthreads();   // earlier readers of part are done
    if (lane == 63) sh.part[w] = inc;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int i = 0; i < L / 64; ++i) {
      if (i < w) base += sh.part[i];
      total += sh.part[i];
    }
  }
  *before = base + inc - n;
  return total;
}

// REG: a row is E chunks a lane and its tail, kept in registers; otherwise it
// is read again from memory in every phase.
template <typename T, int L, int E, bool REG>
__global__ __launch_bounds__(L > 256 ? L : 256) void topk_kernel(const T* __restrict__ z, float* __restrict__ vals,
                                                                 int32_t* __restrict__ idx, long R, int C, long ldz,
                                                                 int K) {
  constexpr int VW = TT<T>::VW, NT = L > 256 ? L : 256, G = NT / L;
  constexpr int M = TopShared<L>::M;
  __shared__ TopShared<L> shared[G];
  TopShared<L>& sh = shared[L < NT ? threadIdx.x / L : 0];
  const int nch = C / VW, steps = (nch + L - 1) / L;
  for (long b = (long)blockIdx.x * G; b < R; b += (long)gridDim.x * G) {
    int l = threadIdx.x % L;
    asm volatile("" : "+v"(l));   // classes are computed where they are needed, not kept over the rows
    const int tail = nch * VW + l;
    const long r = b + (L < NT ? threadIdx.x / L : 0);
    if (L < NT && r >= R) return;   // whole waves, which nothing waits for
    const T* zr = z + r * ldz;
    uint4 q[REG ? E : 1];
    T qt{};
    if (REG) {
#pragma unroll
      for (int e = 0; e < E; ++e) q[e] = load_chunk(zr + (e * L + l < nch ? (e * L + l) * VW : 0));
    }
    if (tail < C) qt = zr[tail];
    // f(values, first class) over the lane's chunks: from memory, and from the
    // registers if they are there
    auto chunks_again = [&](auto f) {
      float v[VW];
#pragma unroll 1
      for (int c = l; c < nch; c += L) {
        unpack<T>(load_chunk(zr + (long)c * VW), v);
        f(v, c * VW);
      }
    };
    auto chunks = [&](auto f) {
      if constexpr (REG) {
        float v[VW];
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (e * L + l < nch) {
            unpack<T>(q[e], v);
            f(v, (e * L + l) * VW);
            opaque(q[e]);
            __builtin_amdgcn_sched_barrier(0);   // one chunk's values at a time in registers
          }
      } else {
        chunks_again(f);
      }
    };
    float top = tail < C ? TT<T>::to_f(qt) : -INFINITY;
    chunks([&](const float* v, int) {
#pragma unroll
      for (int j = 0; j < VW; j += 2) top = max3(top, v[j], v[j + 1]);
    });
    if (!(top == top)) top = -INFINITY;   // any number that no logit of the lane is below is a bound

    // the bound: the K-th largest of the lanes' maxima, or of those of fours
    // of lanes where these are enough
    const int bits = key_bits<T>();
    float bound;
    if constexpr (L == 64) {
      const uint32_t k[1] = {order_key(top)};
      bound = key_value<T>(kth_key<1>(k, K, bits));
    } else {
      const bool fours = K * 16 <= L;
      if (fours) top = group_max<4>(top);
      if (!fours || (l & 3) == 0) sh.keys[fours ? l >> 2 : l] = order_key(top);
      if (l == 0) sh.count = 0;
      __syncthreads();
      if (threadIdx.x < 64) {
        uint32_t t;
        if (fours) {
          uint32_t k[L / 256];
#pragma unroll
          for (int p = 0; p < L / 256; ++p) k[p] = sh.keys[p * 64 + l];
          t = kth_key<L / 256>(k, K, bits);
        } else {
          uint32_t k[L / 64];
#pragma unroll
          for (int p = 0; p < L / 64; ++p) k[p] = sh.keys[p * 64 + l];
          t = kth_key<L / 64>(k, K, bits);
        }
        if (l == 0) sh.bound = t;
      }
      __syncthreads();
      bound = key_value<T>(sh.bound);
    }
    if (L == 64) {
      if (l == 0) sh.count = 0;
      row_sync<L>();
    }
    if (!(bound == bound)) bound = -INFINITY;   // no key: fewer lanes than K

    auto take = [&](float v, int c) {
      const uint32_t at = atomicAdd(&sh.count, 1u);
      if (at < M) sh.list[at] = (uint64_t)order_key(v) << 32 | (uint32_t)~c;
    };
    chunks([&](const float* v, int c) {
      bool some = false;
#pragma unroll
      for (int j = 0; j < VW; ++j) some |= !(v[j] < bound);
      if (some) {
#pragma unroll
        for (int j = 0; j < VW; ++j)
          if (!(v[j] < bound)) take(v[j], c + j);
      }
    });
    if (tail < C && !(TT<T>::to_f(qt) < bound)) take(TT<T>::to_f(qt), tail);
    row_sync<L>();
    int n = (int)sh.count;
    if (n > M) {
      // count of logits above a key
      auto above = [&](uint32_t k) {
        int s = tail < C && order_key(TT<T>::to_f(qt)) > k ? 1 : 0, before;
        chunks_again([&](const float* v, int) {
#pragma unroll
          for (int j = 0; j < VW; ++j) s += order_key(v[j]) > k ? 1 : 0;
        });
        return row_count<L>(s, &before, sh);
      };
      // above(lo) > M, above(hi) < K; the bound's own key is the likely answer
      uint32_t lo = order_key(bound) - 1, hi = 0xffffffffu, at = lo + 1;
      int have = 0;
      while (hi - lo > 1) {
        have = above(at);
        if (have > M) lo = at;
        else if (have < K) hi = at;
        else break;
        at = lo + (hi - lo) / 2;
      }
      if (hi - lo <= 1) {   // all above hi, and the first classes at hi
        at = hi;
        have = above(at);
      }
      row_sync<L>();
      if (l == 0) sh.count = 0;
      row_sync<L>();
      auto take_above = [&](float v, int c) {
        if (order_key(v) > at) take(v, c);
      };
      chunks_again([&](const float* v, int c) {
#pragma unroll
        for (int j = 0; j < VW; ++j) take_above(v[j], c + j);
      });
      if (tail < C) take_above(TT<T>::to_f(qt), tail);
      n = have;
      for (int e = 0; e <= steps && n < K; ++e) {   // e = steps: the tail
        float v[VW];
        const int c = e * L + l;
        int first = c * VW, count = c < nch ? VW : 0;
        if (e == steps) {
          first = tail;
          count = tail < C ? 1 : 0;
          v[0] = TT<T>::to_f(qt);
        } else if (count) {
          unpack<T>(load_chunk(zr + first), v);
        }
        int same = 0, before;
#pragma unroll
        for (int j = 0; j < VW; ++j) same += j < count && order_key(v[j]) == at ? 1 : 0;
        const int total = row_count<L>(same, &before, sh);
        before += n;
#pragma unroll
        for (int j = 0; j < VW; ++j)
          if (j < count && order_key(v[j]) == at) {
            if (before < K) sh.list[before] = (uint64_t)at << 32 | (uint32_t)~(first + j);
            ++before;
          }
        n = std::min(K, n + total);
      }
      row_sync<L>();
    }
    // places: `per` lanes (a power of two) count for each entry
    int per = 1;
    while (per < 16 && n * per * 2 <= L) per *= 2;
    const int sub = l & (per - 1);
    for (int i0 = 0; i0 < n; i0 += L / per) {
      const int i = i0 + l / per;
      const uint64_t mine = i < n ? sh.list[i] : ~0ull;
      int place = 0;
      for (int j = sub; j < n; j += per) place += sh.list[j] > mine ? 1 : 0;
      for (int o = 1; o < per; o <<= 1) place += __shfl_xor(place, o);
      if (i < n && sub == 0 && place < K) {
        const int c = (int)~(uint32_t)mine;
        vals[r * K + place] = TT<T>::to_f(zr[c]);
        idx[r * K + place] = c;
      }
    }
    row_sync<L>();   // before the next row's list
  }
}

template <typename T, int L, int E, bool REG = true, typename... A>
int topk_go(long R, hipStream_t s, A... a) {
  constexpr int NT = L > 256 ? L : 256, G = NT / L;
  const long units = (R + G - 1) / G;
  hipLaunchKernelGGL((topk_kernel<T, L, E, REG>), dim3((unsigned)std::min(units, 1l << 20)), dim3(NT), 0, s, a...);
  return ok();
}

}  // namespace

size_t topk_workspace(int prec, long R, int C, int K) {
  (void)prec; (void)R; (void)C; (void)K;
  return 0;
}

int topk_launch(int prec, const void* z, float* vals, int32_t* idx, long R, int C, long ldz, int K, void* ws,
                hipStream_t s) {
  (void)ws;
  if (R <= 0) return 0;
  return with_prec(prec, [&](auto tag) {
    using T = decltype(tag);
    const T* zt = (const T*)z;
    const int nch = C / TT<T>::VW;
    if (K <= 16 && nch <= 256) {
      if (nch <= 64) return topk_go<T, 64, 1>(R, s, zt, vals, idx, R, C, ldz, K);
      if (nch <= 128) return topk_go<T, 64, 2>(R, s, zt, vals, idx, R, C, ldz, K);
      return topk_go<T, 64, 4>(R, s, zt, vals, idx, R, C, ldz, K);
    }
    if (nch <= 256) return topk_go<T, 256, 1>(R, s, zt, vals, idx, R, C, ldz, K);
    if (nch <= 512) return topk_go<T, 256, 2>(R, s, zt, vals, idx, R, C, ldz, K);
    if (nch <= 1024) return topk_go<T, 256, 4>(R, s, zt, vals, idx, R, C, ldz, K);
    if (nch <= 2048) return topk_go<T, 256, 8>(R, s, zt, vals, idx, R, C, ldz, K);
    if (nch <= 4096) return topk_go<T, 512, 8>(R, s, zt, vals, idx, R, C, ldz, K);
    if (nch <= 8192) return topk_go<T, 1024, 8>(R, s, zt, vals, idx, R, C, ldz, K);
    if (nch <= 16384) return topk_go<T, 1024, 16>(R, s, zt, vals, idx, R, C, ldz, K);
    return topk_go<T, 1024, 1, false>(R, s, zt, vals, idx, R, C, ldz, K);
  });
}

}  // namespace rn18

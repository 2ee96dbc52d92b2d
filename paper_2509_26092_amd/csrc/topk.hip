// The K largest logits of a row with their classes, in descending order, ties
// in the order of the classes.
//
// A row is read once, into the registers of L lanes. The K-th largest of the
// lanes' own maxima is a bound that at least K logits reach and few more do
// (about K^2 / 2L of a random row), so one compare against it leaves a short
// list, and counting for each entry of the list how many others precede it
// gives its place. The work beyond the one pass over the row is small, and
// the pass is bound by memory: 16384x32768 bf16, 20 kept, 175 us (6.1 TB/s,
// what reads alone reach), 64 kept 193 us; 4096x32768, 64 kept, 54 us. Where
// more logits reach the bound than the list holds (equal logits: masked rows;
// rows whose large logits crowd in few lanes), a bisection over the order of
// the values, counted over the row, finds a bound that fits or the value that
// all the surplus shares, of which the first classes are taken. Lists of about
// as many entries as the row has chunks get there too, which takes several
// times the pass (5592x1500 bf16: 64 kept 17 us, 256 kept 446).
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "kernels.h"
#include "rows.h"

namespace rn18 {

namespace {

inline int ok() { return hipGetLastError() == hipSuccess ? 0 : -4; }

// Order-preserving unsigned key of a float: larger value, larger key; the
// two zeros share a key and every NaN has the largest one. 0 is no value's.
constexpr uint32_t kNanKey = 0xfffffffeu;
__device__ inline uint32_t order_key(float v) {
  if (v != v) return kNanKey;
  const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.0f);   // -0 + 0 = +0
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
// The smallest value whose key has these leading bits (the others of k are 0).
__device__ inline float key_value(uint32_t k) {
  return __builtin_bit_cast(float, k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// A value such that the numbers above it are those with keys above k, for k
// from -inf's key on: -0's own pattern is no number's key, and above +inf
// there are only NaNs.
__device__ inline float above_value(uint32_t k) {
  if (k == 0x7fffffffu) --k;
  return k >= 0xff800000u ? INFINITY : key_value(k);
}
// The key of a maximum that a bound may rest on: 0 for a NaN's.
__device__ inline uint32_t max_key(float m) { return m == m ? order_key(m) : 0; }

// A bound for the K-th largest of the 64 * PER keys that a wave holds: its
// leading kBoundBits bits (sign, exponent and 5 bits of the mantissa: it is
// less than 1/32 below, which adds a few entries to the list and takes a
// third of the steps of 32 bits off); 0 if there are fewer than K keys.
constexpr int kBoundBits = 14;
template <int PER, typename F>
__device__ inline uint32_t kth_key(F key, int K) {   // key(p): the lane's p-th
  auto enough = [&](uint32_t c) {
    int n = 0;
#pragma unroll
    for (int p = 0; p < PER; ++p) n += __popcll(__ballot(key(p) >= c));
    return n >= K;
  };
  // from 2 to 2^33, with the sign: where the K-th logit of most rows lies
  uint32_t t = 0xc0000000u;
  int b = 28;
  if (!enough(t) || enough(0xd0000000u)) {
    t = 0;
    b = 31;
  }
#pragma unroll 1
  for (; b >= 32 - kBoundBits; --b) {
    const uint32_t c = t | 1u << b;
    if (enough(c)) t = c;
  }
  return t;
}

template <int L>
struct TopShared {
  static constexpr int M = L > 512 ? 2048 : L > 64 ? 1024 : 256;   // entries of the list
  uint64_t list[M];
  uint32_t chunk[M];
  uint32_t keys[L > 64 ? L : 1];
  uint32_t count, chunks, bound;
  int part[16];
};

// Sum over the row's waves of a count that each holds, and the sum over the
// waves before this one.
template <int L>
__device__ inline int row_count(int n, int* before, TopShared<L>& sh) {
  *before = 0;
  if (L == 64) return n;
  const int w = threadIdx.x >> 6;
  __syncthreads();   // earlier readers of part are done
  if ((threadIdx.x & 63) == 0) sh.part[w] = n;
  __syncthreads();
  int total = 0;
  for (int i = 0; i < L / 64; ++i) {
    if (i < w) *before += sh.part[i];
    total += sh.part[i];
  }
  return total;
}

// REG: a lane has E chunks, whose maxima it keeps; otherwise any number, and
// it reads them again to find those that reach the bound. A row may be cut into gridDim.y
// parts of `len` logits, whose entries (key, ~class) go to
// part[row][part][K]. (Eight waves a SIMD for blocks of 256: 65536x8192
// bf16, 20 kept, 223 us in place of 244; for blocks of 512 16384x32768 would
// take 188 us in place of 175.)
template <typename T, int L, int E, bool REG>
__global__ __launch_bounds__(L > 256 ? L : 256, L == 256 ? 8 : 1) void topk_kernel(
    const T* __restrict__ z, float* __restrict__ vals, int32_t* __restrict__ idx, uint64_t* __restrict__ part, long R,
    int Call, int len, long ldz, int K) {
  constexpr int VW = TT<T>::VW, NT = L > 256 ? L : 256, G = NT / L;
  constexpr int M = TopShared<L>::M;
  __shared__ TopShared<L> shared[G];
  const int grp = L < NT ? threadIdx.x / L : 0;
  TopShared<L>& sh = shared[grp];
  const int first = (int)blockIdx.y * len;
  const int C = std::min(len, Call - first);
  // (L < NT: each wave has its own rows, and nothing waits for another's)
  for (long r = (long)blockIdx.x * G + grp; r < R; r += (long)gridDim.x * G) {
    int l = threadIdx.x % L;
    asm volatile("" : "+v"(l));   // classes are computed where they are needed, not kept over the rows
    const T* zr = z + r * ldz + first;
    // (chunks at odd addresses: a row of 131071 fp16 logits 12.3 us in place of 8.1)
    const int head = row_head(zr, C);
    const int nch = (C - head) / VW;
    const T* zc = zr + head;
    const int tail = l < head ? l : nch * VW + l;
    const float vt = TT<T>::to_f(zr[tail < C ? tail : 0]);

    // the bound: the K-th largest of the maxima of chunks (of a wave's row),
    // lanes, or fours of lanes where these are enough
    uint32_t kth;
    float tops[REG ? E : 1];   // the largest of each of the lane's chunks
    if (l == 0) sh.count = sh.chunks = 0;
    if constexpr (REG) {
      constexpr int B = E < 8 ? E : 8;   // chunks in flight
#pragma unroll
      for (int e0 = 0; e0 < E; e0 += B) {
        uint4 q[B];
#pragma unroll
        for (int e = 0; e < B; ++e) {
          const int c = (e0 + e) * L + l;
          q[e] = load_chunk_at(chunk_base(zc, nch), (c < nch ? c : 0) * 16u);
        }
#pragma unroll
        for (int e = 0; e < B; ++e) {
          float v[VW];
          unpack<T>(q[e], v);
          tops[e0 + e] = (e0 + e) * L + l < nch ? chunk_max<VW>(v) : -INFINITY;
        }
        // registers for B chunks, so that two blocks fit a compute unit
        if (e0 + B < E) __builtin_amdgcn_sched_barrier(0);
      }
    }
    if constexpr (L == 64) {
      uint32_t k[E];
#pragma unroll
      for (int e = 0; e < E; ++e) k[e] = max_key(tops[e]);
      kth = kth_key<E>([&](int p) { return k[p]; }, K);
    } else {
      float top = tail < C ? vt : -INFINITY;
      if constexpr (REG) {
#pragma unroll
        for (int e = 0; e < E; ++e) top = max2(top, tops[e]);
      } else {
        float v[VW];
        for (int c = l; c < nch; c += L) {
          unpack<T>(load_chunk(zc + (long)c * VW), v);
          top = max2(top, chunk_max<VW>(v));
        }
      }
      const bool fours = K * 8 <= L;
      if (!(top == top)) top = -INFINITY;
      if (fours) top = group_max<4>(top);
      if (!fours || (l & 3) == 0) sh.keys[fours ? l >> 2 : l] = max_key(top);
      __syncthreads();
      if (threadIdx.x < 64) {
        uint32_t t;
        if (fours) {
          uint32_t k[L / 256];
#pragma unroll
          for (int p = 0; p < L / 256; ++p) k[p] = sh.keys[p * 64 + l];
          t = kth_key<L / 256>([&](int p) { return k[p]; }, K);
        } else {
          // (registers for four keys, no more: a block's other waves need none)
          uint32_t k[4];
#pragma unroll
          for (int p = 0; p < 4; ++p) k[p] = sh.keys[p * 64 + l];
          t = kth_key<L / 64>([&](int p) { return p < 4 ? k[p] : sh.keys[p * 64 + l]; }, K);
        }
        if (l == 0) sh.bound = t;
      }
      __syncthreads();
      kth = sh.bound;
    }
    float bound = key_value(kth);
    if (!(bound == bound)) bound = -INFINITY;   // fewer maxima than K, or cut to below the key of -inf

    // The chunks whose maximum reaches the bound (a NaN does), then, a lane for
    // each of their logits, the list of those that do, in any order. (Few
    // lanes of a wave have such a chunk, so the lanes would idle if each went
    // through its own.)
    if (L == 64) row_sync<L>();   // (the counts are zero)
    if constexpr (REG) {
      uint32_t hit = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) hit |= !(tops[e] < bound) && e * L + l < nch ? 1u << e : 0u;
      if (hit) {
        uint32_t at = atomicAdd(&sh.chunks, (uint32_t)__popc(hit));
#pragma unroll 1
        for (; hit; hit &= hit - 1, ++at)
          if (at < M) sh.chunk[at] = (uint32_t)((__ffs(hit) - 1) * L + l);
      }
    } else {
      for (int c = l; c < nch; c += L) {
        float v[VW];
        unpack<T>(load_chunk(zc + (long)c * VW), v);
        if (!(chunk_max<VW>(v) < bound)) {
          const uint32_t at = atomicAdd(&sh.chunks, 1u);
          if (at < M) sh.chunk[at] = (uint32_t)c;
        }
      }
    }
    auto take = [&](float v, int c) {
      const uint32_t at = atomicAdd(&sh.count, 1u);
      if (at < M) sh.list[at] = (uint64_t)order_key(v) << 32 | (uint32_t)~c;
    };
    if (tail < C && !(vt < bound)) take(vt, tail);
    row_sync<L>();
    const int hits = (int)sh.chunks;
    if (hits <= M)
#pragma unroll 1
      for (int i = l; i < hits * VW; i += L) {
        const int c = head + (int)sh.chunk[i / VW] * VW + i % VW;
        const float v = TT<T>::to_f(zr[c]);
        if (!(v < bound)) take(v, c);
      }
    row_sync<L>();
    int n = hits <= M ? (int)sh.count : M + 1;
    if (n > M) {
      // the list of the logits above a key, and their count
      auto above = [&](uint32_t k) {
        row_sync<L>();
        if (l == 0) sh.count = 0;
        row_sync<L>();
        const float v0 = above_value(k);   // above k: not at or below v0
        if (k < kNanKey) {
#pragma unroll 1
          for (int c = l; c < nch; c += L) {
            float v[VW];
            unpack<T>(load_chunk(zc + (long)c * VW), v);
            if (chunk_max<VW>(v) <= v0) continue;
            uint32_t hit = 0;
#pragma unroll
            for (int j = 0; j < VW; ++j) hit |= !(v[j] <= v0) ? 1u << j : 0u;
            uint32_t at = atomicAdd(&sh.count, (uint32_t)__popc(hit));
#pragma unroll 1
            for (; hit; hit &= hit - 1, ++at) {
              const int i = head + c * VW + __ffs(hit) - 1;
              if (at < M) sh.list[at] = (uint64_t)order_key(TT<T>::to_f(zr[i])) << 32 | (uint32_t)~i;
            }
          }
          if (tail < C && !(vt <= v0)) take(vt, tail);
        }
        row_sync<L>();
        return (int)sh.count;
      };
      // above(lo) > M, above(hi) < K; the bound's own key is the likely answer
      uint32_t lo = order_key(bound) - 1, hi = 0xffffffffu, at = lo + 1;
      int have = 0;
#pragma unroll 1
      while (true) {
        have = above(at);
        if (have > M) lo = at;
        else if (have < K) hi = at;
        else break;
        if (hi - lo <= 1) break;
        at = lo + (hi - lo) / 2;
      }
      if (have > M) {   // all above hi, and the first classes at hi
        at = hi;
        have = above(at);
      }
      n = have;
#pragma unroll 1
      for (int c0 = 0; c0 < C && n < K; c0 += L) {
        const int c = c0 + l;
        const bool same = c < C && order_key(TT<T>::to_f(zr[c < C ? c : 0])) == at;
        const uint64_t who = __ballot(same);
        int before;
        const int total = row_count<L>(__popcll(who), &before, sh);
        before += n + __popcll(who & ((1ull << (threadIdx.x & 63)) - 1));
        if (same && before < K) sh.list[before] = (uint64_t)at << 32 | (uint32_t)~c;
        n = std::min(K, n + total);
      }
      row_sync<L>();
    }
    // places: `per` lanes (a power of two) count for each entry
    int per = 1;
    while (per < 16 && n * per * 2 <= L) per *= 2;
    const int sub = l & (per - 1);
#pragma unroll 1
    for (int i0 = 0; i0 < n; i0 += L / per) {
      const int i = i0 + l / per;
      const uint64_t mine = i < n ? sh.list[i] : ~0ull;
      int place = 0;
#pragma unroll 4
      for (int j = sub; j < n; j += per) place += sh.list[j] > mine ? 1 : 0;
      for (int o = 1; o < per; o <<= 1) place += __shfl_xor(place, o);
      if (i < n && sub == 0 && place < K) {
        const int c = (int)~(uint32_t)mine;
        if (gridDim.y > 1) {
          part[(r * gridDim.y + blockIdx.y) * K + place] = mine - first;   // ~(c + first)
        } else {
          vals[r * K + place] = TT<T>::to_f(zr[c]);
          idx[r * K + place] = c;
        }
      }
    }
    row_sync<L>();   // before the next row's list
  }
}

// Short rows, a wave each: P logits a lane, the K-th largest of all of them
// as the bound, and each lane counts the entries before its own.
template <typename T, int P>
__global__ __launch_bounds__(256) void topk_short_kernel(const T* __restrict__ z, float* __restrict__ vals,
                                                         int32_t* __restrict__ idx, long R, int C, long ldz, int K) {
  __shared__ uint64_t lists[4][64 * P];
  const int l = threadIdx.x & 63;
  uint64_t* list = lists[threadIdx.x >> 6];
  for (long r = (long)blockIdx.x * 4 + (threadIdx.x >> 6); r < R; r += (long)gridDim.x * 4) {
    const T* zr = z + r * ldz;
    float v[P];
    uint32_t k[P];
#pragma unroll
    for (int p = 0; p < P; ++p) v[p] = TT<T>::to_f(zr[p * 64 + l < C ? p * 64 + l : 0]);
#pragma unroll
    for (int p = 0; p < P; ++p) k[p] = p * 64 + l < C ? order_key(v[p]) : 0;
    // (not 0: there are K keys, and the smallest, of -inf, has bits among the bound's)
    const uint32_t bound = kth_key<P>([&](int p) { return k[p]; }, K);
    int n = 0;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const bool hit = k[p] >= bound;
      const uint64_t who = __ballot(hit);
      if (hit) list[n + __popcll(who & ((1ull << l) - 1))] = (uint64_t)k[p] << 32 | (uint32_t)~(p * 64 + l);
      n += __popcll(who);
    }
    row_sync<64>();
    int place[P] = {};
#pragma unroll 4
    for (int j = 0; j < n; ++j) {
      const uint64_t e = list[j];
#pragma unroll
      for (int p = 0; p < P; ++p) place[p] += e > ((uint64_t)k[p] << 32 | (uint32_t)~(p * 64 + l)) ? 1 : 0;
    }
#pragma unroll
    for (int p = 0; p < P; ++p)
      if (k[p] >= bound && place[p] < K) {
        vals[r * K + place[p]] = v[p];
        idx[r * K + place[p]] = p * 64 + l;
      }
    row_sync<64>();   // before the next row's list
  }
}

// The places of a row's n entries from all its parts: 8 lanes count for each.
constexpr int kMergeMax = 2048;
template <typename T>
__global__ __launch_bounds__(1024) void topk_merge_kernel(const T* __restrict__ z, float* __restrict__ vals,
                                                          int32_t* __restrict__ idx, const uint64_t* __restrict__ part,
                                                          long R, long ldz, int K, int n) {
  __shared__ uint64_t list[kMergeMax];
  const int sub = threadIdx.x & 7;
  for (long r = blockIdx.x; r < R; r += gridDim.x) {
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += 1024) list[i] = part[r * n + i];
    __syncthreads();
    for (int i0 = 0; i0 < n; i0 += 128) {
      const int i = i0 + (int)(threadIdx.x >> 3);
      const uint64_t mine = i < n ? list[i] : ~0ull;
      int place = 0;
#pragma unroll 8
      for (int j = sub; j < n; j += 8) place += list[j] > mine ? 1 : 0;
      for (int o = 1; o < 8; o <<= 1) place += __shfl_xor(place, o);
      if (i < n && sub == 0 && place < K) {
        const int c = (int)~(uint32_t)mine;
        vals[r * K + place] = TT<T>::to_f(z[r * ldz + c]);
        idx[r * K + place] = c;
      }
    }
  }
}

struct TopPlan {
  int parts, len;
};
// Rows of more than 2^14 chunks, more than a block keeps the maxima of, are
// cut into parts of up to 2^13 (512 rows of 131071 fp32 logits: 45 us, 2048
// rows 191; in parts of 2^14, of which a compute unit holds one at a time, 58
// and 225; fewer rows or shorter ones gain nothing from parts: the launch that
// joins them costs what they save).
TopPlan topk_plan(int prec, int C, int K) {
  const int vw = prec_vw(prec);
  if (C / vw <= 16384) return {1, C};
  const int most = 8192 * vw;
  const int parts = ceil_div(C, most);
  const int len = (ceil_div(C, parts) + vw - 1) / vw * vw;
  // (the last part is the shortest and still holds K)
  if ((long)parts * K > kMergeMax || (long)(parts - 1) * len + K > C) return {1, C};
  return {parts, len};
}

template <typename T, int L, int E, bool REG = true, typename... A>
int topk_go(long R, int parts, hipStream_t s, A... a) {
  constexpr int NT = L > 256 ? L : 256, G = NT / L;
  const long units = std::min((R + G - 1) / G, 1l << 22);
  hipLaunchKernelGGL((topk_kernel<T, L, E, REG>), dim3((unsigned)units, parts), dim3(NT), 0, s, a...);
  return ok();
}

}  // namespace

size_t topk_workspace(int prec, long R, int C, int K) {
  const TopPlan pl = topk_plan(prec, C, K);
  return pl.parts > 1 && R > 0 ? (size_t)R * pl.parts * K * 8 : 0;
}

int topk_launch(int prec, const void* z, float* vals, int32_t* idx, long R, int C, long ldz, int K, void* ws,
                hipStream_t s) {
  if (R <= 0) return 0;
  const TopPlan pl = topk_plan(prec, C, K);
  return with_prec(prec, [&](auto tag) {
    using T = decltype(tag);
    const T* zt = (const T*)z;
    uint64_t* part = (uint64_t*)ws;
    const int nch = pl.len / TT<T>::VW;
    auto go = [&](auto l, auto e, auto reg) {
      return topk_go<T, decltype(l)::value, decltype(e)::value, decltype(reg)::value>(R, pl.parts, s, zt, vals, idx,
                                                                                     part, R, C, pl.len, ldz, K);
    };
    auto pick = [&]() {
#define SHORT(P)                                                                                                  \
  {                                                                                                               \
    const dim3 grid((unsigned)std::min((R + 3) / 4, 1l << 22));                                                   \
    hipLaunchKernelGGL((topk_short_kernel<T, P>), grid, dim3(256), 0, s, zt, vals, idx, R, C, ldz, K);            \
    return ok();                                                                                                  \
  }
      // Every logit's key takes part in the bound: rows to 256 logits (335544x100
      // bf16, 10 kept: 107 us, with maxima of chunks 176; 64 kept: 207 and 501),
      // longer ones whose chunks are too few for a bound (16384x512 bf16, 100
      // kept: 60 and 444, 52 kept: 37 and 54; 8192x1024, 256 kept: 136 and 874;
      // but 40 kept of 512, from 64 chunks: 33 and 23). At the rule's edge the
      // two cross within a tenth: 8192x1024, 100 kept: 66 and 63, 8388x1000 71
      // and 64.
      const int chunks = C / TT<T>::VW;
      if (C <= 64) SHORT(1);
      if (C <= 128) SHORT(2);
      if (C <= 256) SHORT(4);
      if (C <= 512 && chunks * 3 < K * 4) SHORT(8);
      if (C <= 1024 && chunks * 3 < K * 4) SHORT(16);
#undef SHORT
#define GO(L, E) return go(std::integral_constant<int, L>{}, std::integral_constant<int, E>{}, std::true_type{})
      // a wave per row where its chunks are more than K
      if (K <= 64 && nch <= 512 && nch * 2 >= K * 3) {
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
      if (nch <= 16384) GO(1024, 16);
#undef GO
      return go(std::integral_constant<int, 1024>{}, std::integral_constant<int, 1>{}, std::false_type{});
    };
    int r = pick();
    if (r || pl.parts == 1) return r;
    hipLaunchKernelGGL(topk_merge_kernel<T>, dim3((unsigned)std::min(R, 1l << 22)), dim3(1024), 0, s, zt, vals, idx,
                       (const uint64_t*)part, R, ldz, K, pl.parts * K);
    return ok();
  });
}

}  // namespace rn18

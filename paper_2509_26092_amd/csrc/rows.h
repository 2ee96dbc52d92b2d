// Device helpers of the row operators (layer norm, top logits, distillation):
// 16-byte chunks of rows that may start at any element, and reductions over
// groups of lanes.
#pragma once
#include "common.h"

namespace rn18 {

// A 16-byte chunk at any element. Global memory takes 16-byte accesses at any
// byte address here, so rows need no alignment beyond their element's.
template <typename T>
__device__ inline uint4 load_chunk(const T* p) {
  uint4 q;
  __builtin_memcpy(&q, p, 16);
  return q;
}
// The same at a byte offset below 2^32, which leaves a row's address, where it
// is the same for the whole wave, out of the lanes' registers.
template <typename T>
__device__ inline uint4 load_chunk_at(const T* row, uint32_t bytes) {
  uint4 q;
  __builtin_memcpy(&q, (const T*)((const char*)row + bytes), 16);
  return q;
}
template <typename T>
__device__ inline void store_chunk(T* p, const uint4& q) {
  __builtin_memcpy(p, &q, 16);
}
template <typename T>
__device__ inline void store_chunk_at(T* row, uint32_t bytes, const uint4& q) {
  __builtin_memcpy((T*)((char*)row + bytes), &q, 16);
}

// A row of W elements is W / VW whole chunks and up to VW - 1 further
// elements, its tail, one to a lane. Where loads at odd addresses cost time,
// the chunks start at the row's first 16-byte boundary, after row_head
// elements; these are one to a lane as well.
template <typename T>
__device__ inline int row_head(const T* row, int width) {
  const int head = (int)((0 - (uintptr_t)row) & 15) / (int)sizeof(T);
  return head < width ? head : width;
}

// Where a lane without a chunk of a row loads from: the row's first chunk, or
// 16 bytes of zeros where the row has none (a branch around the loads would
// wait for each of them). Not const: global memory like the rows, so that the
// loads are global ones.
static __device__ uint4 kNoChunk = {0, 0, 0, 0};
template <typename T>
__device__ inline const T* chunk_base(const T* row, int nch) {
  return nch > 0 ? row : (const T*)&kNoChunk;
}

// Hides where a chunk came from, so that values unpacked from it before are
// not kept in registers until they are needed again.
__device__ inline void opaque(uint4& q) { asm volatile("" : "+v"(q.x), "+v"(q.y), "+v"(q.z), "+v"(q.w)); }

// f over the values of L lanes of a wave (L a power of two up to 64, groups
// aligned); every lane of the group gets the same bits. Lanes are exchanged
// at distances 1, 2 (quad permutes), 4, 8 (mirrors of half rows and rows,
// whose halves hold equal values by then), 16 and 32 (row and half-wave
// swaps). Every lane of the wave takes part.
template <int CTRL>
__device__ inline uint32_t dpp_mov(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
template <int L, typename F>
__device__ inline float group_red(float v, F f) {
  auto bits = [](float x) { return __builtin_bit_cast(uint32_t, x); };
  auto flt = [](uint32_t x) { return __builtin_bit_cast(float, x); };
  if (L >= 2) v = f(v, flt(dpp_mov<0xB1>(bits(v))));
  if (L >= 4) v = f(v, flt(dpp_mov<0x4E>(bits(v))));
  if (L >= 8) v = f(v, flt(dpp_mov<0x141>(bits(v))));
  if (L >= 16) v = f(v, flt(dpp_mov<0x140>(bits(v))));
  if (L >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(bits(v), bits(v), false, false);
    v = f(flt(r[0]), flt(r[1]));
  }
  if (L >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(bits(v), bits(v), false, false);
    v = f(flt(r[0]), flt(r[1]));
  }
  return v;
}
struct Sum {
  __device__ float operator()(float a, float b) const { return a + b; }
};
struct Max {
  __device__ float operator()(float a, float b) const { return __builtin_elementwise_maximum(a, b); }
};
template <int L>
__device__ inline float group_sum(float v) {
  return group_red<L>(v, Sum());
}
template <int L>
__device__ inline float group_max(float v) {
  return group_red<L>(v, Max());
}

// The same over the L lanes of a row, N values at a time. Lanes of more than
// one wave meet in `sh`, a buffer of the caller that no lane may still read
// from: callers alternate between two.
template <int L, int N, typename F>
__device__ inline void row_red(float (&v)[N], float (*sh)[N], F f) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = group_red<(L < 64 ? L : 64)>(v[i], f);
  if (L > 64) {
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) sh[w][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = group_red<(L > 64 ? L / 64 : 1)>(sh[threadIdx.x & (L / 64 - 1)][i], f);
  }
}
template <int L, int N>
__device__ inline void row_sums(float (&v)[N], float (*sh)[N]) {
  row_red<L>(v, sh, Sum());
}

// The largest of two and of three, or a NaN if one of them is (one
// instruction).
__device__ inline float max2(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ inline float max3(float a, float b, float c) {
  return max2(max2(a, b), c);
}
template <int VW>
__device__ inline float chunk_max(const float* v) {
  float m = max3(v[0], v[1], v[2]);
#pragma unroll
  for (int j = 3; j + 1 < VW; j += 2) m = max3(m, v[j], v[j + 1]);
  return max2(m, v[VW - 1]);
}
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

}  // namespace rn18

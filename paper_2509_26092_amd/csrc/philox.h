// Random words of a counter, for dropout masks that are never stored.
#pragma once
#include "common.h"

namespace rn18 {

// Philox4x32-10 (Salmon et al., SC'11): ten rounds of two 32x32 -> 64-bit
// products mixed with the other counter words and the key, the key bumped by
// the Weyl constants between rounds.
__device__ inline void philox4x32_10(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    if (r) {
      k0 += 0x9E3779B9u;
      k1 += 0xBB67AE85u;
    }
    const uint64_t p0 = (uint64_t)0xD2511F53u * c[0], p1 = (uint64_t)0xCD9E8D57u * c[2];
    const uint32_t n0 = (uint32_t)(p1 >> 32) ^ c[1] ^ k0, n2 = (uint32_t)(p0 >> 32) ^ c[3] ^ k1;
    c[0] = n0;
    c[1] = (uint32_t)p1;
    c[2] = n2;
    c[3] = (uint32_t)p0;
  }
}

// Dropout of the rows of a matrix of D columns, p > 0: element j of row r is
// kept iff the top 24 bits of word j mod 4 of the counter (r ceil(D/4) + j
// div 4, step) are >= thresh, and kept elements are multiplied by `scale`.
// `step_add` (may be NULL) is read when the kernel runs: a replayed graph
// takes the step that stands there then.
struct Dropout {
  uint32_t k0, k1, thresh;
  float scale;
  uint64_t step;
  const uint64_t* step_add;
};
// What a kernel holds of it.
struct DropKey {
  uint32_t k0, k1, s0, s1, thresh;
  float scale;
  long quads;   // words of a row, by fours
  __device__ DropKey(const Dropout& d, int D) : k0(d.k0), k1(d.k1), thresh(d.thresh), scale(d.scale) {
    const uint64_t t = d.step + (d.step_add ? *d.step_add : 0);
    s0 = (uint32_t)t;
    s1 = (uint32_t)(t >> 32);
    quads = (D + 3l) / 4;
  }
  // v[0..3], columns 4 * quad .. + 3 of row r, dropped or scaled.
  __device__ inline void apply4(float* v, long r, int quad) const {
    const uint64_t q = (uint64_t)(r * quads + quad);
    uint32_t c[4] = {(uint32_t)q, (uint32_t)(q >> 32), s0, s1};
    philox4x32_10(c, k0, k1);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (c[i] >> 8) >= thresh ? v[i] * scale : 0.f;
  }
  template <int VW>
  __device__ inline void apply(float* v, long r, int start) const {
#pragma unroll
    for (int h = 0; h < VW / 4; ++h) apply4(v + 4 * h, r, start / 4 + h);
  }
  // One element.
  __device__ inline float one(float v, long r, int col) const {
    const uint64_t q = (uint64_t)(r * quads + col / 4);
    uint32_t c[4] = {(uint32_t)q, (uint32_t)(q >> 32), s0, s1};
    philox4x32_10(c, k0, k1);
    const uint32_t lo = col & 1 ? c[1] : c[0], hi = col & 1 ? c[3] : c[2];
    return ((col & 2 ? hi : lo) >> 8) >= thresh ? v * scale : 0.f;
  }
};

}  // namespace rn18

// Dropout masks from the library's Philox4x32-10 stream: 16 bits per element, eight elements per call, never stored.
#pragma once

#include <math.h>

#include "hdqt_types.cuh"

namespace hdqt {

struct DropParams {
  PhiloxKeys keys;
  const uint32_t* offset;   // device word, fourth counter word (null = 0)
  uint32_t tag;
  uint32_t limit;           // (T << 16) - 1: an element is kept if its 16 bits, in the upper half of a word, are above it
  int32_t on;               // T > 0
  float scale;
};

inline bool valid_probability(double p) { return p >= 0.0 && p <= 1.0; }

inline DropParams make_drop(double p, uint64_t seed, uint32_t tag, const uint32_t* offset) {
  DropParams d{};
  const uint32_t t = (uint32_t)rint(p * 65536.0);
  d.keys = make_philox_keys(seed);
  d.offset = offset;
  d.tag = tag;
  d.on = t > 0;
  d.limit = (uint32_t)(((uint64_t)t << 16) - 1);
  d.scale = t < 65536 ? (float)(65536.0 / (65536 - t)) : 0.0f;
  return d;
}

__device__ __forceinline__ uint32_t drop_offset(const DropParams& d) { return d.offset ? *d.offset : 0u; }

// random words of the elements 8 g .. 8 g + 7
__device__ __forceinline__ Philox4 drop_words(const DropParams& d, uint32_t offset, uint64_t g) {
  return philox4x32_10((uint32_t)g, (uint32_t)(g >> 32), d.tag, offset, d.keys);
}
// those of several groups at once, so that a round's keys are fetched once for all
template <int N>
__device__ __forceinline__ void drop_words(const DropParams& d, uint32_t offset, const uint64_t (&g)[N], Philox4 (&w)[N]) {
  constexpr uint32_t M0 = 0xD2511F53u, M1 = 0xCD9E8D57u;
#pragma unroll
  for (int u = 0; u < N; ++u) {
    w[u].w[0] = (uint32_t)g[u];
    w[u].w[1] = (uint32_t)(g[u] >> 32);
    w[u].w[2] = d.tag;
    w[u].w[3] = offset;
  }
#pragma unroll
  for (int r = 0; r < 10; ++r) {
#pragma unroll
    for (int u = 0; u < N; ++u) {
      uint32_t(&c)[4] = w[u].w;
      const uint32_t hi0 = __umulhi(M0, c[0]), lo0 = M0 * c[0], hi1 = __umulhi(M1, c[2]), lo1 = M1 * c[2];
      c[0] = hi1 ^ c[1] ^ d.keys.k[r][0];
      c[1] = lo1;
      c[2] = hi0 ^ c[3] ^ d.keys.k[r][1];
      c[3] = lo0;
    }
  }
}
__device__ __forceinline__ bool drop_keeps(const Philox4& r, int j, uint32_t limit) {
  return (j & 1 ? r.w[j >> 1] : r.w[j >> 1] << 16) > limit;
}
// the eight decisions as bits
__device__ __forceinline__ uint32_t drop_bits(const DropParams& d, uint32_t offset, uint64_t g) {
  const Philox4 r = drop_words(d, offset, g);
  uint32_t bits = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) bits |= drop_keeps(r, j, d.limit) ? 1u << j : 0u;
  return bits;
}

}  // namespace hdqt

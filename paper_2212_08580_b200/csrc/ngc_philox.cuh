// Dropout decisions from a counter-based generator: Philox4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers:
// as easy as 1, 2, 3", 2011).  Element (row, column) takes 16 of the 128 bits that the counter
// (column / 8, row's low word, row's high word, step) gives under the key `seed`; it is dropped where they are below
// round(65536 p).  So the decision depends on nothing but seed, step and position: not on the type, the strides, the launch, or
// which worker holds the row.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

namespace ngc {

// (The keys of the ten rounds are worked out on the host and read from the kernel's parameters: as adds in every thread they were a third
// of the generator's instructions.)
struct DropoutKey {
  uint64_t first_row;
  uint32_t step;
  uint32_t threshold;  // 0: nothing is dropped, 65536: everything
  uint32_t round[10][2];
};

inline uint32_t dropout_threshold(double p) { return (uint32_t)(p * 65536.0 + 0.5); }
inline DropoutKey dropout_key(double p, uint64_t seed, uint64_t first_row, uint32_t step) {
  DropoutKey d;
  d.first_row = first_row;
  d.step = step;
  d.threshold = dropout_threshold(p);
  for (uint32_t r = 0; r < 10; ++r) {
    d.round[r][0] = (uint32_t)seed + r * 0x9E3779B9u;
    d.round[r][1] = (uint32_t)(seed >> 32) + r * 0xBB67AE85u;
  }
  return d;
}

__device__ __forceinline__ uint4 philox4x32(uint4 c, const uint32_t (&key)[10][2]) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p0 = (uint64_t)c.x * 0xD2511F53u, p1 = (uint64_t)c.z * 0xCD9E8D57u;
    c = make_uint4((uint32_t)(p1 >> 32) ^ c.y ^ key[r][0], (uint32_t)p1, (uint32_t)(p0 >> 32) ^ c.w ^ key[r][1], (uint32_t)p0);
  }
  return c;
}

// Which of the elements 8 block .. 8 block + 7 of a row are kept.
struct Keep8 {
  uint32_t w[4];
  uint32_t limit;  // an element is kept where its 16 bits, as the upper half of a word, are above this
  __device__ __forceinline__ bool operator[](int j) const { return (j & 1 ? w[j >> 1] : w[j >> 1] << 16) > limit; }
  // The same as a mask of the 16-bit elements 2 i and 2 i + 1.
  __device__ __forceinline__ uint32_t halves(int i) const {
    return ((*this)[2 * i] ? 0xffffu : 0u) | ((*this)[2 * i + 1] ? 0xffff0000u : 0u);
  }
};
// (The upper half of a word is at least t > 0 where the word is above t 2^16 - 1, whatever its lower half is; t = 65536 keeps
// nothing.)
__device__ __forceinline__ Keep8 dropout_keep8(const DropoutKey &d, uint64_t row, uint32_t block) {
  if (d.threshold == 0) return {{~0u, ~0u, ~0u, ~0u}, 0u};
  row += d.first_row;
  const uint4 b = philox4x32(make_uint4(block, (uint32_t)row, (uint32_t)(row >> 32), d.step), d.round);
  return {{b.x, b.y, b.z, b.w}, (d.threshold << 16) - 1u};
}

}  // namespace ngc

// Blocks of 8 elements (fp32 or bf16, as 32-bit words) at addresses that need not be multiples of 16 bytes.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace ngc {

template <typename T>
struct Words;  // of 8 elements
template <>
struct Words<float> {
  static constexpr int n = 8;
};
template <>
struct Words<__nv_bfloat16> {
  static constexpr int n = 4;
};

// Elements [0, n) one by one, as words.
__device__ __forceinline__ void load_some(const float *p, int n, uint32_t (&w)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = i < n ? __float_as_uint(p[i]) : 0u;
}
__device__ __forceinline__ void load_some(const __nv_bfloat16 *p, int n, uint32_t (&w)[4]) {
  const uint16_t *s = reinterpret_cast<const uint16_t *>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = 2 * i < n ? s[2 * i] : 0, hi = 2 * i + 1 < n ? s[2 * i + 1] : 0;
    w[i] = lo | hi << 16;
  }
}
// Elements [from, to) one by one, zero beside them.
__device__ __forceinline__ void load_between(const float *p, int from, int to, uint32_t (&w)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = i >= from && i < to ? __float_as_uint(p[i]) : 0u;
}
__device__ __forceinline__ void load_between(const __nv_bfloat16 *p, int from, int to, uint32_t (&w)[4]) {
  const uint16_t *s = reinterpret_cast<const uint16_t *>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = 2 * i >= from && 2 * i < to ? s[2 * i] : 0, hi = 2 * i + 1 >= from && 2 * i + 1 < to ? s[2 * i + 1] : 0;
    w[i] = lo | hi << 16;
  }
}
// Elements [from, to) one by one.
__device__ __forceinline__ void store_some(float *p, int from, int to, const uint32_t (&w)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i >= from && i < to) p[i] = __uint_as_float(w[i]);
}
__device__ __forceinline__ void store_some(__nv_bfloat16 *p, int from, int to, const uint32_t (&w)[4]) {
  uint16_t *d = reinterpret_cast<uint16_t *>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i >= from && i < to) d[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
}

template <int N>
__device__ __forceinline__ void load_whole(const void *p, uint32_t (&w)[N]) {
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const uint4 q = static_cast<const uint4 *>(p)[i];
    w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
  }
}
template <int N>
__device__ __forceinline__ void store_whole(void *p, const uint32_t (&w)[N]) {
#pragma unroll
  for (int i = 0; i < N / 4; ++i)
    static_cast<uint4 *>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
}

// N words that begin `bytes` (even, at most 16) into `w`, to its front.
template <int N>
__device__ __forceinline__ void shift_words(uint32_t (&w)[N + 4], int bytes, uint32_t (&out)[N]) {
#pragma unroll
  for (int s = 4; s > 0; s >>= 1)
    if (bytes & (4 * s)) {
#pragma unroll
      for (int i = 0; i + s < N + 4; ++i) w[i] = w[i + s];
    }
#pragma unroll
  for (int i = 0; i < N; ++i) out[i] = bytes & 2 ? __funnelshift_r(w[i], w[i + 1], 16) : w[i];
}

// 8 elements anywhere, from the whole 16-byte vectors that they lie in; these belong to the matrix [first, last).
template <typename T>
__device__ __forceinline__ void load_anywhere(const T *p, int n, const void *first, const void *last, uint32_t (&w)[Words<T>::n]) {
  constexpr int N = Words<T>::n;
  const uintptr_t at = reinterpret_cast<uintptr_t>(p), base = at & ~(uintptr_t)15;
  if (n >= 8 && at == base) {
    load_whole(p, w);
    return;
  }
  if (n < 8 || base < reinterpret_cast<uintptr_t>(first) || base + 4 * N + 16 > reinterpret_cast<uintptr_t>(last)) {
    load_some(p, n, w);
    return;
  }
  uint32_t whole[N + 4];
  load_whole(reinterpret_cast<const void *>(base), whole);
  shift_words<N>(whole, (int)(at & 15), w);
}

}  // namespace ngc

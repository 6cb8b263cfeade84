// ngc_dropout: dropout whose mask is worked out again wherever it is needed, from seed, step, row and column.
//
// A thread takes blocks of 8 elements of a row, which share one call of the generator (ten rounds of two 32 x 32 -> 64-bit
// products for eight 16-bit numbers).  One read (two with a residual), one write.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>
#include <utility>

#include "ngc.h"
#include "ngc_device.h"
#include "ngc_pdl.cuh"
#include "ngc_philox.cuh"
#include "ngc_spans.h"
#include "ngc_words.cuh"

namespace ngc {

namespace {

struct DropoutArgs {
  const void *x, *residual;
  void *out;
  long long ld_x, ld_residual, ld_out;
  long long rows, items;  // items: blocks of 8 columns, or segments of 32 blocks, of all rows
  int columns, per_row;   // items of a row
  long long row_step;     // what a thread's (a warp's) next item is further on
  int item_step;
  float stretch;
  DropoutKey key;
};

// Rows that all begin at 16-byte boundaries: a thread per block.  The next item's row and block follow from the last one's
// without a division.
constexpr int kThreads = 256;

__device__ __forceinline__ void unpack(const uint32_t (&w)[8], float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
}
__device__ __forceinline__ void unpack(const uint32_t (&w)[4], float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void pack(const float (&v)[8], uint32_t (&w)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[i]);
}
__device__ __forceinline__ void pack(const float (&v)[8], uint32_t (&w)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t *>(&h);
  }
}

template <typename T>
__device__ __forceinline__ void drop(const DropoutArgs &a, long long row, int block, const uint32_t (&x)[Words<T>::n],
                                     const uint32_t (&residual)[Words<T>::n], uint32_t (&out)[Words<T>::n]) {
  float v[8], r[8];
  unpack(x, v);
  if (a.key.threshold) {
    const Keep8 keep = dropout_keep8(a.key, (uint64_t)row, (uint32_t)block);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = keep[j] ? v[j] * a.stretch : 0.f;
  }
  if (a.residual) {
    unpack(residual, r);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += r[j];
  }
  pack(v, out);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) dropout_kernel(const DropoutArgs a) {
  pdl_sync();
  constexpr int N = Words<T>::n;
  long long i = (long long)blockIdx.x * kThreads + threadIdx.x;
  long long row = i / a.per_row;
  int block = (int)(i - row * a.per_row);
  const long long step = (long long)gridDim.x * kThreads;
  for (; i < a.items; i += step) {
    const int n = a.columns - block * 8;
    const T *x = static_cast<const T *>(a.x) + row * a.ld_x + block * 8;
    const T *residual = static_cast<const T *>(a.residual) + row * a.ld_residual + block * 8;
    T *dst = static_cast<T *>(a.out) + row * a.ld_out + block * 8;
    uint32_t w[N], r[N] = {}, out[N];
    if (n >= 8) {
      load_whole(x, w);
      if (a.residual) load_whole(residual, r);
    } else {
      load_some(x, n, w);
      if (a.residual) load_some(residual, n, r);
    }
    drop<T>(a, row, block, w, r, out);
    if (n >= 8) store_whole(dst, out);
    else store_some(dst, 0, n, out);
    row += a.row_step;
    block += a.item_step;
    if (block >= a.per_row) {
      block -= a.per_row;
      ++row;
    }
  }
}

// Rows that begin anywhere: a warp per 32 blocks.  Lanes read the whole vectors that their elements lie in, and write whole
// vectors of the output, whose first elements come from the lane before; what is left at either end goes element by
// element (bf16 [1999][5003] in rows of 5009: 8 loads and 8 stores of 2 bytes per lane took 28 us).
template <typename T>
__global__ void __launch_bounds__(kThreads) dropout_anywhere_kernel(const DropoutArgs a) {
  pdl_sync();
  constexpr int N = Words<T>::n, E = 4 * N / 8;  // E: bytes of an element
  const int lane = threadIdx.x & 31;
  long long i = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  long long row = i / a.per_row;
  int segment = (int)(i - row * a.per_row);
  const long long step = (long long)gridDim.x * (kThreads / 32);
  const T *x_end = static_cast<const T *>(a.x) + (a.rows - 1) * a.ld_x + a.columns;
  const T *residual_end = static_cast<const T *>(a.residual) + (a.rows - 1) * a.ld_residual + a.columns;
  for (; i < a.items; i += step) {
    const int block = segment * 32 + lane, n = a.columns - block * 8;
    uint32_t w[N] = {}, r[N] = {}, out[N];
    if (n > 0) {
      load_anywhere(static_cast<const T *>(a.x) + row * a.ld_x + block * 8, n, a.x, x_end, w);
      if (a.residual)
        load_anywhere(static_cast<const T *>(a.residual) + row * a.ld_residual + block * 8, n, a.residual, residual_end, r);
    }
    drop<T>(a, row, block, w, r, out);
    T *dst = static_cast<T *>(a.out) + row * a.ld_out + block * 8;
    const int off = (int)(reinterpret_cast<uintptr_t>(dst) & 15);  // the same in all lanes, as a block is whole vectors
    uint32_t whole[N + 4], shifted[N];
#pragma unroll
    for (int j = 0; j < 4; ++j) whole[j] = __shfl_up_sync(0xffffffffu, out[N - 4 + j], 1);
#pragma unroll
    for (int j = 0; j < N; ++j) whole[4 + j] = out[j];
    shift_words<N>(whole, 16 - off, shifted);
    // (lanes are whole up to some lane of the row)
    const bool full = n >= 8, joined = full && lane > 0, next = n >= 16 && lane < 31;
    unsigned char *base = reinterpret_cast<unsigned char *>(dst) - off;
    if (joined || (full && off == 0)) {
      store_whole(base, shifted);
    } else if (full) {  // the first vector also holds another warp's, or row's, elements
#pragma unroll
      for (int k = 1; k < N / 4; ++k)
        reinterpret_cast<uint4 *>(base)[k] = make_uint4(shifted[4 * k], shifted[4 * k + 1], shifted[4 * k + 2], shifted[4 * k + 3]);
      store_some(dst, 0, (16 - off) / E, out);
    }
    if (full && !next && off) store_some(dst, 8 - off / E, 8, out);
    if (!full && n > 0) store_some(dst, 0, n, out);
    row += a.row_step;
    segment += a.item_step;
    if (segment >= a.per_row) {
      segment -= a.per_row;
      ++row;
    }
  }
}

template <typename T>
cudaError_t launch_dropout(DropoutArgs a, bool vectors, int sms, cudaStream_t stream) {
  const int blocks = (int)(((long long)a.columns + 7) / 8), each = vectors ? kThreads : kThreads / 32;
  a.per_row = vectors ? blocks : (blocks + 31) / 32;
  a.items = a.rows * a.per_row;
  const long long work = (a.items + each - 1) / each, most = (long long)sms * 8;
  const unsigned grid = (unsigned)(work < most ? work : most);
  const long long step = (long long)grid * each;
  a.row_step = step / a.per_row;
  a.item_step = (int)(step % a.per_row);
  return vectors ? launch_k(dropout_kernel<T>, grid, kThreads, 0, stream, a)
                 : launch_k(dropout_anywhere_kernel<T>, grid, kThreads, 0, stream, a);
}

}  // namespace
}  // namespace ngc

extern "C" {

int ngc_dropout(const ngc_dropout_t *cfg, const void *x, int64_t ld_x, const void *residual, int64_t ld_residual, void *out,
                int64_t ld_out, void *cuda_stream) {
  using namespace ngc;
  if (!cfg || cfg->rows < 0 || cfg->rows >= 1ll << 44 || cfg->columns < 1 || (cfg->dtype != NGC_F32 && cfg->dtype != NGC_BF16) ||
      !(cfg->p >= 0.0 && cfg->p <= 1.0))
    return NGC_ERR_INVALID;
  if (cfg->rows == 0) return NGC_OK;
  const size_t e = cfg->dtype == NGC_F32 ? 4 : 2;
  const long long far = (1ll << 44) / (cfg->rows + 1);
  if (!x || !out || !aligned(x, e) || !aligned(out, e) || !aligned(residual, e) || ld_x < cfg->columns || ld_x > far ||
      ld_out < cfg->columns || ld_out > far || (residual && (ld_residual < cfg->columns || ld_residual > far)))
    return NGC_ERR_INVALID;
  const Span o = matrix_span(out, cfg->rows, cfg->columns, ld_out, e);
  if ((out != x || (ld_out != ld_x && cfg->rows > 1)) && !apart(o, matrix_span(x, cfg->rows, cfg->columns, ld_x, e)))
    return NGC_ERR_INVALID;
  if (residual && (out != residual || (ld_out != ld_residual && cfg->rows > 1)) &&
      !apart(o, matrix_span(residual, cfg->rows, cfg->columns, ld_residual, e)))
    return NGC_ERR_INVALID;
  const int sms = device_sm_count();
  if (sms <= 0) return NGC_ERR_CUDA;
  DropoutArgs a = {};
  a.x = x; a.residual = residual; a.out = out;
  a.ld_x = ld_x; a.ld_residual = ld_residual; a.ld_out = ld_out;
  a.rows = cfg->rows; a.columns = cfg->columns;
  const uint32_t t = dropout_threshold(cfg->p);
  a.stretch = t < 65536 ? (float)(65536.0 / (65536 - t)) : 0.f;
  a.key = {cfg->seed, cfg->first_row, cfg->step, t};
  bool vectors = true;
  for (auto [p, ld] : {std::make_pair(x, ld_x), std::make_pair(residual, ld_residual), std::make_pair((const void *)out, ld_out)})
    vectors = vectors && (!p || (aligned(p, 16) && (cfg->rows == 1 || (size_t)ld * e % 16 == 0)));
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t rc = cfg->dtype == NGC_F32 ? launch_dropout<float>(a, vectors, sms, stream)
                                               : launch_dropout<__nv_bfloat16>(a, vectors, sms, stream);
  return rc == cudaSuccess ? NGC_OK : NGC_ERR_CUDA;
}

}  // extern "C"

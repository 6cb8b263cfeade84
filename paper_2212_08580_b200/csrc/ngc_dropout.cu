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
  long long rows, items;  // items: 32 bytes of a row, or segments of 32 blocks of 8 columns, of all rows
  int columns, per_row;   // items of a row
  long long row_step;     // what a thread's (a warp's) next item is further on
  int item_step;
  float stretch;
  DropoutKey key;
};

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
__device__ __forceinline__ void drop(const DropoutArgs &a, const Keep8 &keep, const uint32_t (&x)[Words<T>::n],
                                     const uint32_t (&residual)[Words<T>::n], uint32_t (&out)[Words<T>::n]) {
  float v[8], r[8];
  unpack(x, v);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = keep[j] ? v[j] * a.stretch : 0.f;
  if (a.residual) {
    unpack(residual, r);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += r[j];
  }
  pack(v, out);
}

// 32 bytes at a multiple of 32.
__device__ __forceinline__ void load32(const void *p, uint32_t (&w)[8]) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
               : "l"(p)
               : "memory");
}
__device__ __forceinline__ void store32(void *p, const uint32_t (&w)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]),
               "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}

// Rows that all begin at multiples of 32 bytes: a thread per 32 bytes (one block of 8 fp32, two of bf16).  The next item's row and
// place follow from the last one's without a division.  Five blocks on an SM: the registers of more would spill (8192 x 4096 bf16 with
// residual and back: four 63, five 60, six 68 us).
constexpr int kResident = 5;
template <typename T>
__global__ void __launch_bounds__(kThreads, kResident) dropout_kernel(const DropoutArgs a) {
  pdl_sync();
  constexpr int N = Words<T>::n, kBlocks = 8 / N;
  long long i = (long long)blockIdx.x * kThreads + threadIdx.x;
  long long row = i / a.per_row;
  int item = (int)(i - row * a.per_row);
  const long long step = (long long)gridDim.x * kThreads;
  const T *x = static_cast<const T *>(a.x) + row * a.ld_x + item * 8 * kBlocks;
  const T *residual = static_cast<const T *>(a.residual) + row * a.ld_residual + item * 8 * kBlocks;
  T *dst = static_cast<T *>(a.out) + row * a.ld_out + item * 8 * kBlocks;
  for (; i < a.items; i += step) {
    const int n = a.columns - item * 8 * kBlocks;
    uint32_t w[8], r[8] = {}, out[8];
    if (n >= 8 * kBlocks) {
      load32(x, w);
      if (a.residual) load32(residual, r);
    } else {
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        load_some(x + 8 * b, n - 8 * b, *reinterpret_cast<uint32_t(*)[N]>(&w[b * N]));
        if (a.residual) load_some(residual + 8 * b, n - 8 * b, *reinterpret_cast<uint32_t(*)[N]>(&r[b * N]));
      }
    }
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
      drop<T>(a, dropout_keep8(a.key, (uint64_t)row, (uint32_t)(item * kBlocks + b)), *reinterpret_cast<const uint32_t(*)[N]>(&w[b * N]),
              *reinterpret_cast<const uint32_t(*)[N]>(&r[b * N]), *reinterpret_cast<uint32_t(*)[N]>(&out[b * N]));
    if (n >= 8 * kBlocks) {
      store32(dst, out);
    } else {
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) store_some(dst + 8 * b, 0, n - 8 * b, *reinterpret_cast<const uint32_t(*)[N]>(&out[b * N]));
    }
    long long rows = a.row_step;
    int items = a.item_step;
    if (item + items >= a.per_row) {
      items -= a.per_row;
      ++rows;
    }
    row += rows;
    item += items;
    x += rows * a.ld_x + items * 8 * kBlocks;
    residual += rows * a.ld_residual + items * 8 * kBlocks;
    dst += rows * a.ld_out + items * 8 * kBlocks;
  }
}

// Rows that begin anywhere, but x, residual and output at the same place within 16 bytes: a warp per 31 whole vectors (pairs of them
// for fp32) of memory, whose elements begin in one block of 8 columns and end in the next.  Each lane works out the random numbers of
// one block and takes the end of the one before from its neighbour (lane 0 does nothing else), so that only these are shifted,
// and memory is read and written by whole vectors but at a row's ends.
template <typename T>
__global__ void __launch_bounds__(kThreads) dropout_shifted_kernel(const DropoutArgs a) {
  pdl_sync();
  constexpr int N = Words<T>::n;
  const int lane = threadIdx.x & 31;
  long long i = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  long long row = i / a.per_row;
  int segment = (int)(i - row * a.per_row);
  const long long step = (long long)gridDim.x * (kThreads / 32);
  for (; i < a.items; i += step) {
    const int block = segment * 31 + lane - 1;
    const T *x = static_cast<const T *>(a.x) + row * a.ld_x;
    const int before = (int)(reinterpret_cast<uintptr_t>(x) & 15) / (int)sizeof(T);  // elements of the row's first vector that are not its own
    const int first = block * 8 - before, end = min(first + 8, a.columns);
    uint32_t w[N] = {}, r[N] = {}, out[N];
    const bool mine = lane > 0 && end > 0 && first < a.columns, full = mine && first >= 0 && end == first + 8;
    const T *residual = static_cast<const T *>(a.residual) + row * a.ld_residual + first;
    if (full) {
      load_whole(x + first, w);
      if (a.residual) load_whole(residual, r);
    } else if (mine) {
      load_between(x + first, max(0, -first), end - first, w);
      if (a.residual) load_between(residual, max(0, -first), end - first, r);
    }
    uint32_t bits[8], of[4];
    const Keep8 here = dropout_keep8(a.key, (uint64_t)row, (uint32_t)block);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      bits[j] = __shfl_up_sync(0xffffffffu, here.w[j], 1);
      bits[4 + j] = here.w[j];
    }
    shift_words<4>(bits, 16 - 2 * before, of);
    const Keep8 keep = {{of[0], of[1], of[2], of[3]}, here.limit};
    drop<T>(a, keep, w, r, out);
    T *dst = static_cast<T *>(a.out) + row * a.ld_out + first;
    if (full) store_whole(dst, out);
    else if (mine) store_some(dst, max(0, -first), end - first, out);
    row += a.row_step;
    segment += a.item_step;
    if (segment >= a.per_row) {
      segment -= a.per_row;
      ++row;
    }
  }
}

// Anything else, element by element.
template <typename T>
__global__ void __launch_bounds__(kThreads) dropout_loose_kernel(const DropoutArgs a) {
  pdl_sync();
  constexpr int N = Words<T>::n;
  const long long step = (long long)gridDim.x * kThreads;
  for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < a.items; i += step) {
    const long long row = i / a.per_row;
    const int block = (int)(i - row * a.per_row), n = a.columns - block * 8;
    uint32_t w[N], r[N] = {}, out[N];
    load_some(static_cast<const T *>(a.x) + row * a.ld_x + block * 8, n, w);
    if (a.residual) load_some(static_cast<const T *>(a.residual) + row * a.ld_residual + block * 8, n, r);
    drop<T>(a, dropout_keep8(a.key, (uint64_t)row, (uint32_t)block), w, r, out);
    store_some(static_cast<T *>(a.out) + row * a.ld_out + block * 8, 0, n, out);
  }
}

enum Rows { kVectors, kShifted, kLoose };

template <typename T>
cudaError_t launch_dropout(DropoutArgs a, Rows rows, int sms, cudaStream_t stream) {
  constexpr long long kItem = 32 / sizeof(T);  // columns
  const int each = rows == kShifted ? kThreads / 32 : kThreads;
  // (a row that begins within a vector has one vector of 8 elements more)
  a.per_row = (int)(rows == kVectors ? (a.columns + kItem - 1) / kItem : rows == kShifted ? ((a.columns + 14ll) / 8 + 30) / 31 : (a.columns + 7ll) / 8);
  a.items = a.rows * a.per_row;
  const long long work = (a.items + each - 1) / each, most = (long long)sms * (rows == kVectors ? kResident : 8);
  const unsigned grid = (unsigned)(work < most ? work : most);
  const long long step = (long long)grid * each;
  a.row_step = step / a.per_row;
  a.item_step = (int)(step % a.per_row);
  return launch_k(rows == kVectors ? dropout_kernel<T> : rows == kShifted ? dropout_shifted_kernel<T> : dropout_loose_kernel<T>, grid, kThreads, 0,
                  stream, a);
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
  const MatrixSpan o(out, cfg->rows, cfg->columns, ld_out, e);
  if ((out != x || (ld_out != ld_x && cfg->rows > 1)) && !apart(o, MatrixSpan(x, cfg->rows, cfg->columns, ld_x, e))) return NGC_ERR_INVALID;
  if (residual && (out != residual || (ld_out != ld_residual && cfg->rows > 1)) &&
      !apart(o, MatrixSpan(residual, cfg->rows, cfg->columns, ld_residual, e)))
    return NGC_ERR_INVALID;
  const int sms = device_sm_count();
  if (sms <= 0) return NGC_ERR_CUDA;
  DropoutArgs a = {};
  a.x = x; a.residual = residual; a.out = out;
  a.ld_x = ld_x; a.ld_residual = ld_residual; a.ld_out = ld_out;
  a.rows = cfg->rows; a.columns = cfg->columns;
  const uint32_t t = dropout_threshold(cfg->p);
  a.stretch = t < 65536 ? (float)(65536.0 / (65536 - t)) : 0.f;
  a.key = dropout_key(cfg->p, cfg->seed, cfg->first_row, cfg->step);
  Rows rows = kVectors;
  const uintptr_t at = reinterpret_cast<uintptr_t>(x) & 15, turn = cfg->rows == 1 ? 0 : (uintptr_t)ld_x * e & 15;
  for (auto [p, ld] : {std::make_pair(x, ld_x), std::make_pair(residual, ld_residual), std::make_pair((const void *)out, ld_out)}) {
    if (!p) continue;
    if (rows == kVectors && !(aligned(p, 32) && (cfg->rows == 1 || (size_t)ld * e % 32 == 0))) rows = kShifted;
    if ((reinterpret_cast<uintptr_t>(p) & 15) != at || (cfg->rows > 1 && ((uintptr_t)ld * e & 15) != turn)) rows = kLoose;
  }
  // (the last warp of a shifted row counts up to 31 blocks beyond it, in 32 bits)
  if (rows == kShifted && cfg->columns > 0x7fffffff - 32 * 8) rows = kLoose;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t rc = cfg->dtype == NGC_F32 ? launch_dropout<float>(a, rows, sms, stream)
                                               : launch_dropout<__nv_bfloat16>(a, rows, sms, stream);
  return rc == cudaSuccess ? NGC_OK : NGC_ERR_CUDA;
}

}  // extern "C"

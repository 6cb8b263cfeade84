// ngc_dropout: dropout whose mask is worked out again wherever it is needed, from seed, step, row and column.
//
// A thread takes blocks of 8 elements of a row, which share one call of the generator (ten rounds of two 32 x 32 -> 64-bit
// products for eight 16-bit numbers).  One read (two with a residual), one write.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

#include "ngc.h"
#include "ngc_device.h"
#include "ngc_pdl.cuh"
#include "ngc_philox.cuh"
#include "ngc_spans.h"

namespace ngc {

namespace {

struct DropoutArgs {
  const void *x, *residual;
  void *out;
  long long ld_x, ld_residual, ld_out;
  long long rows;
  int columns, blocks;  // blocks of 8 columns
  float stretch;
  DropoutKey key;
};

__device__ __forceinline__ void load8(const float *p, int n, float (&v)[8]) {
  if (n >= 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
    const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.f;
  }
}
__device__ __forceinline__ void load8(const __nv_bfloat16 *p, int n, float (&v)[8]) {
  if (n >= 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
    const uint4 q = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? __bfloat162float(p[i]) : 0.f;
  }
}
__device__ __forceinline__ void store8(float *p, int n, const float (&v)[8]) {
  if (n >= 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
    reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = v[i];
  }
}
__device__ __forceinline__ void store8(__nv_bfloat16 *p, int n, const float (&v)[8]) {
  if (n >= 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = __float2bfloat16_rn(v[i]);
  }
}

template <typename T>
__global__ void __launch_bounds__(256) dropout_kernel(const DropoutArgs a) {
  pdl_sync();
  const long long total = a.rows * a.blocks;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
    const long long row = i / a.blocks;
    const int block = (int)(i - row * a.blocks), n = a.columns - block * 8;
    float v[8], r[8];
    load8(static_cast<const T *>(a.x) + row * a.ld_x + block * 8, n, v);
    if (a.residual) load8(static_cast<const T *>(a.residual) + row * a.ld_residual + block * 8, n, r);
    const uint32_t keep = dropout_keep8(a.key, (uint64_t)row, (uint32_t)block);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[j] = (keep >> j) & 1 ? v[j] * a.stretch : 0.f;
      if (a.residual) v[j] += r[j];
    }
    store8(static_cast<T *>(a.out) + row * a.ld_out + block * 8, n, v);
  }
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
  DropoutArgs a;
  a.x = x; a.residual = residual; a.out = out;
  a.ld_x = ld_x; a.ld_residual = ld_residual; a.ld_out = ld_out;
  a.rows = cfg->rows; a.columns = cfg->columns; a.blocks = (int)(((long long)cfg->columns + 7) / 8);
  const uint32_t t = dropout_threshold(cfg->p);
  a.stretch = t < 65536 ? (float)(65536.0 / (65536 - t)) : 0.f;
  a.key = {cfg->seed, cfg->first_row, cfg->step, t};
  const long long work = (a.rows * a.blocks + 255) / 256;
  const unsigned grid = (unsigned)(work < sms * 8ll ? work : sms * 8ll);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t rc = cfg->dtype == NGC_F32 ? launch_k(dropout_kernel<float>, grid, 256, 0, stream, a)
                                               : launch_k(dropout_kernel<__nv_bfloat16>, grid, 256, 0, stream, a);
  return rc == cudaSuccess ? NGC_OK : NGC_ERR_CUDA;
}

}  // extern "C"

// ngc_linear_cross_entropy: softmax cross entropy over a large vocabulary straight from features X [rows][d] and weights W
// [classes][d] (or [d][classes]), with the gradients of both.
//
//   z = scale X W^T,  lse = log sum_v e^z,  G = scale w (e^(z - lse) - onehot),  dX = G W,  dW_j = G_j^T X_j.
//
// The logits are never stored.  The first contraction's epilogue turns each tile of them, straight from tensor memory, into
// its rows' maxima and sums of powers over 128 classes and, for a gradient, into 16-bit powers relative to those maxima (a
// relative error of 2^-12, whatever the logits' size).  One pass over the powers then has lse, losses, and G in their place
// in bf16 (the one rounding to 8 bits; operands of the two gradient contractions are bf16).  Taking the logits a second time
// from X and W instead would need no room for the powers, but a fourth contraction beside three (a third more time);
// the room is bounded by passing the rows through in pieces.
//
// Rows that do not count (labels outside the classes, weight 0) cost nothing: the others are packed first, each
// partition's from a multiple of 64 rows on (so that a K chunk of the weights' gradient never holds two partitions).  The
// packed copy also takes away strides and alignments that bulk copies cannot read, keeps NaN in left-out rows out of
// the products, and is where dropout is applied to the features.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>

#include "ngc.h"
#include "ngc_device.h"
#include "ngc_pdl.cuh"
#include "ngc_philox.cuh"
#include "ngc_spans.h"
#include "ngc_tc.cuh"

namespace ngc {

namespace {

using namespace tc;

constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLn2 = 0.6931471805599453f;
// Powers are stored times 2^14, so that fp16 holds from 2^-38 on, with all its digits from 2^-28 on, and the largest one, which
// the rounding of a maximum of 2^24 may make 2 instead of 1.
constexpr int kPowerBits = 14;
constexpr int kAlign = 64;      // packed rows of a partition are a multiple of a K chunk

// ---- contraction on CTA pairs --------------------------------------------------------------------
// C[M x N] = A B over tiles of 256 x BN (BN = 256 or 128): two CTAs of a cluster drive one 256-row MMA, each loads its own 128
// rows of A and half of B's columns, and keeps its 128 rows of C in its own tensor memory, where two accumulators take
// turns so that a tile's epilogue runs beside the next one's contraction.  Operands come through six stages of 64 along K,
// with 128-byte swizzle, either K-major or M/N-major (X^T, or W in the other layout, is never made).
constexpr int kStages = 6;
constexpr int kHalfBytes = 16384;  // 128 x 64 bf16
constexpr int kStageBytes = 2 * kHalfBytes;
constexpr int kThreads = 320;      // loads, MMA, 8 epilogue warps (two per quadrant of the 128 rows, half of the columns each)
constexpr int kStageTile = 32 * 128;  // a warp's 32 rows of 128 bytes on their way out
constexpr int kSmem = kStages * kStageBytes + 8 * kStageTile + 256 + 1024;
constexpr int kTmem = 512;

enum { kLogits = 0, kFeatureGrad = 1, kWeightGrad = 2 };

struct GemmArgs {
  int m, n;                // extents of C (m: of the buffer, where m_dev says how many rows are in use)
  const int *m_dev;
  int k;                   // extent of the contraction
  const int *k_begin;      // per batch: first row of K (k_begin[batch + 1]: end), multiples of 64; null: 0 .. k
  int batch, splits;       // splits: contiguous shares of K, each with its own output
  int group;               // M tiles that share B tiles while these are in L2
  int *status;
  // kLogits
  const int *label;        // packed rows
  float *label_z;          // scaled logit of the label, times log2(e)
  float2 *stat;            // [row][stats]: largest scaled logit (times log2(e)) and sum of powers, per BN / 2 classes
  int stats;
  float c;                 // scale log2(e)
  __half *power;           // [row][ld_power], null: not wanted
  long long ld_power;
  // kFeatureGrad
  const int *source;       // packed row -> row, -1: none
  __nv_bfloat16 *out;      // also kWeightGrad
  long long ld_out, out_batch;
  float *partial;          // kFeatureGrad: [split][m][n_pad]; kWeightGrad: running sums over pieces of rows, or null
  int n_pad;
  int first, last;         // kWeightGrad: of the pieces that make up a sum
  DropoutKey drop;
};

struct Tile {
  int batch, split, m0, n0, k0, chunks;
};

template <int BN>
__device__ __forceinline__ Tile tile_of(const GemmArgs &p, int m_tiles, int n_tiles, int t) {
  Tile q;
  const int per = m_tiles * n_tiles;
  const int bs = t / per;
  int r = t % per;
  q.batch = bs / p.splits;
  q.split = bs % p.splits;
  const int g = r / (p.group * n_tiles);
  r -= g * p.group * n_tiles;
  const int height = min(p.group, m_tiles - g * p.group);
  q.m0 = (g * p.group + r % height) * 256;
  q.n0 = (r / height) * BN;
  int k0 = 0, k1 = p.k;
  if (p.k_begin) {
    k0 = p.k_begin[q.batch];
    k1 = p.k_begin[q.batch + 1];
  }
  const int chunks = (k1 - k0 + 63) / 64;
  const int a = (int)((long long)chunks * q.split / p.splits), b = (int)((long long)chunks * (q.split + 1) / p.splits);
  q.k0 = k0 + a * 64;
  q.chunks = b - a;
  return q;
}

// 16 bytes of a row's 128 in a warp's staging tile; rows are permuted so that neither writes (a row per lane) nor reads (a
// row per 8 lanes) meet in a bank.
__device__ __forceinline__ uint4 *staged(unsigned char *tile, int row, int piece) {
  return reinterpret_cast<uint4 *>(tile + row * 128 + ((piece ^ (row & 7)) << 4));
}

// Up to 8 16-bit elements at p; whole vectors where p allows.
__device__ __forceinline__ void store8(void *p, const uint4 &v, int n) {
  if (n >= 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
    *static_cast<uint4 *>(p) = v;
    return;
  }
  uint16_t *d = static_cast<uint16_t *>(p);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) d[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ uint32_t pack_half(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t *>(&h);
}

__device__ __forceinline__ float power2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// W columns of one quadrant's 32 rows, from tensor memory to where they belong.
template <int W>
__device__ __forceinline__ void logits_epilogue(const GemmArgs &p, const Tile &q, int nt_half, uint32_t taddr, int row, int n0,
                                                unsigned char *stage, int lane, uint32_t release_bar) {
  uint32_t r[W];
  tmem_ld_chunks<W / 32>(taddr, W / 32, r);
  tc_fence_before();
  mbar_arrive_cluster(release_bar);  // everything is in registers: the accumulator may be written again
  const int valid = p.n - n0;
  const int lab = p.label[row] - n0;
  float top = kNegInf;
  if (valid >= W) {
#pragma unroll
    for (int i = 0; i < W; ++i) top = fmaxf(top, __uint_as_float(r[i]));
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) {
      if (i >= valid) r[i] = __float_as_uint(kNegInf);
      top = fmaxf(top, __uint_as_float(r[i]));
    }
  }
  if (lab >= 0 && lab < min(W, valid)) {
    float z = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) z = i == lab ? __uint_as_float(r[i]) : z;
    p.label_z[row] = z * p.c;
  }
  const float shift = valid > 0 ? top * p.c : 0.f;
  float s0 = 0.f, s1 = 0.f;
  const int row0 = row - lane;
#pragma unroll
  for (int h = 0; h < W / 64; ++h) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = h * 64 + j * 8 + i * 2;
        const float a = power2(fmaf(__uint_as_float(r[at]), p.c, -shift));
        const float b = power2(fmaf(__uint_as_float(r[at + 1]), p.c, -shift));
        s0 += a;
        s1 += b;
        w[i] = pack_half(a * (float)(1 << kPowerBits), b * (float)(1 << kPowerBits));
      }
      if (p.power) *staged(stage, lane, j) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    if (p.power) {
      __syncwarp();
#pragma unroll
      for (int it = 0; it < 8; ++it) {
        const int rr = it * 4 + lane / 8, col = n0 + h * 64 + (lane & 7) * 8;
        if (col < p.ld_power)
          *reinterpret_cast<uint4 *>(p.power + (long long)(row0 + rr) * p.ld_power + col) = *staged(stage, rr, lane & 7);
      }
      __syncwarp();
    }
  }
  // (a NaN among the logits is not the largest, but it is in the sum)
  p.stat[(long long)row * p.stats + nt_half] = make_float2(valid > 0 ? shift : kNegInf, s0 + s1);
}

template <int BN>
__device__ __forceinline__ void feature_epilogue(const GemmArgs &p, const Tile &q, uint32_t taddr, int row, int rows, int n0,
                                                 unsigned char *stage, int lane, uint32_t release_bar) {
  constexpr int W = BN / 2;
  const int row0 = row - lane;
  if (p.splits > 1) {
    float *dst = p.partial + (long long)q.split * p.m * p.n_pad;
#pragma unroll 1
    for (int h = 0; h < W / 32; ++h) {
      uint32_t r[32];
      tmem_ld_chunks<1>(taddr + h * 32, 1, r);
      if (h == W / 32 - 1) {
        tc_fence_before();
        mbar_arrive_cluster(release_bar);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) *staged(stage, lane, j) = make_uint4(r[4 * j], r[4 * j + 1], r[4 * j + 2], r[4 * j + 3]);
      __syncwarp();
#pragma unroll
      for (int it = 0; it < 8; ++it) {
        const int rr = it * 4 + lane / 8, col = n0 + h * 32 + (lane & 7) * 4;
        if (row0 + rr < rows && col < p.n_pad)
          *reinterpret_cast<uint4 *>(dst + (long long)(row0 + rr) * p.n_pad + col) = *staged(stage, rr, lane & 7);
      }
      __syncwarp();
    }
    return;
  }
  const int src = row < rows ? p.source[row] : -1;
  const bool counts = row < rows && p.label[row] >= 0;
#pragma unroll 1
  for (int h = 0; h < W / 64; ++h) {
    uint32_t r[64];
    tmem_ld_chunks<2>(taddr + h * 64, 2, r);
    if (h == W / 64 - 1) {
      tc_fence_before();
      mbar_arrive_cluster(release_bar);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = counts ? pack_bf16(__uint_as_float(r[j * 8 + 2 * i]), __uint_as_float(r[j * 8 + 2 * i + 1])) : 0u;
      if (p.drop.threshold) {
        const Keep8 keep = dropout_keep8(p.drop, (uint64_t)src, (uint32_t)(n0 + h * 64 + j * 8) >> 3);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] &= keep.halves(i);
      }
      *staged(stage, lane, j) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __syncwarp();
#pragma unroll
    for (int it = 0; it < 8; ++it) {
      const int rr = it * 4 + lane / 8, col = n0 + h * 64 + (lane & 7) * 8;
      const int to = __shfl_sync(0xffffffffu, src, rr);
      if (to >= 0 && col < p.n) store8(p.out + (long long)to * p.ld_out + col, *staged(stage, rr, lane & 7), p.n - col);
    }
    __syncwarp();
  }
}

template <int BN>
__device__ __forceinline__ void weight_epilogue(const GemmArgs &p, const Tile &q, uint32_t taddr, int row, int n0,
                                                unsigned char *stage, int lane, uint32_t release_bar) {
  constexpr int W = BN / 2;
  const int row0 = row - lane;
  __nv_bfloat16 *out = p.out + (long long)q.batch * p.out_batch;
  const bool sums = p.partial != nullptr;
#pragma unroll 1
  for (int h = 0; h < W / 64; ++h) {
    uint32_t r[64];
    if (q.chunks > 0) {
      tmem_ld_chunks<2>(taddr + h * 64, 2, r);
    } else {  // no row of this partition counts
#pragma unroll
      for (int i = 0; i < 64; ++i) r[i] = 0u;
    }
    if (h == W / 64 - 1 && q.chunks > 0) {
      tc_fence_before();
      mbar_arrive_cluster(release_bar);
    }
    if (sums) {  // fp32 sums over the pieces of a partition's rows
#pragma unroll
      for (int g = 0; g < 2; ++g) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          *staged(stage, lane, j) = make_uint4(r[g * 32 + 4 * j], r[g * 32 + 4 * j + 1], r[g * 32 + 4 * j + 2], r[g * 32 + 4 * j + 3]);
        __syncwarp();
#pragma unroll
        for (int it = 0; it < 8; ++it) {
          const int rr = it * 4 + lane / 8, col = n0 + h * 64 + g * 32 + (lane & 7) * 4;
          if (row0 + rr < p.m && col < p.n) {
            float4 v = *reinterpret_cast<float4 *>(staged(stage, rr, lane & 7));
            float4 *acc = reinterpret_cast<float4 *>(p.partial + (long long)(row0 + rr) * p.n_pad + col);
            if (!p.first) {
              const float4 old = *acc;
              v.x += old.x; v.y += old.y; v.z += old.z; v.w += old.w;
            }
            if (!p.last) {
              *acc = v;
            } else {
              __nv_bfloat16 *dst = out + (long long)(row0 + rr) * p.ld_out + col;
              const uint32_t lo = pack_bf16(v.x, v.y), hi = pack_bf16(v.z, v.w);
              if (p.n - col >= 4 && (reinterpret_cast<uintptr_t>(dst) & 7) == 0) {
                *reinterpret_cast<uint2 *>(dst) = make_uint2(lo, hi);
              } else {
                uint16_t *d = reinterpret_cast<uint16_t *>(dst);
                d[0] = (uint16_t)lo;
                if (p.n - col > 1) d[1] = (uint16_t)(lo >> 16);
                if (p.n - col > 2) d[2] = (uint16_t)hi;
                if (p.n - col > 3) d[3] = (uint16_t)(hi >> 16);
              }
            }
          }
        }
        __syncwarp();
      }
      continue;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = pack_bf16(__uint_as_float(r[j * 8 + 2 * i]), __uint_as_float(r[j * 8 + 2 * i + 1]));
      *staged(stage, lane, j) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __syncwarp();
#pragma unroll
    for (int it = 0; it < 8; ++it) {
      const int rr = it * 4 + lane / 8, col = n0 + h * 64 + (lane & 7) * 8;
      if (row0 + rr < p.m && col < p.n)
        store8(out + (long long)(row0 + rr) * p.ld_out + col, *staged(stage, rr, lane & 7), p.n - col);
    }
    __syncwarp();
  }
}

template <int EPI, int A_MN, int B_MN, int BN>
__global__ void __launch_bounds__(kThreads, 1)
vocab_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const GemmArgs p) {
  pdl_sync();
  extern __shared__ unsigned char smem_raw[];
  const uint32_t sbase = smem_u32(smem_raw);
  unsigned char *tiles = smem_raw + ((1024u - (sbase & 1023u)) & 1023u);
  unsigned char *staging = tiles + kStages * kStageBytes;
  const uint32_t bars = smem_u32(staging + 8 * kStageTile);
  const uint32_t full = bars, empty = bars + 8 * kStages, tfull = bars + 16 * kStages, tempty = tfull + 16;
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(staging + 8 * kStageTile + 16 * kStages + 32);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(full + 8 * i, 1);
      mbar_init(empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(tfull + 8 * i, 1);
      mbar_init(tempty + 8 * i, 2 * (kThreads - 64));
    }
    mbar_fence_init();
  }
  if (warp == 1) tmem_alloc_pair(smem_u32(tmem_slot), kTmem);
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // the peer's barriers exist before anything is signalled on them
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  bool failed = false;
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const int rows = p.m_dev ? *p.m_dev : p.m;
  const int m_tiles = (rows + 255) / 256, n_tiles = (p.n + BN - 1) / BN;
  const int total = m_tiles * n_tiles * p.batch * p.splits;
  constexpr int kHalf = BN / 2;                       // columns of B that this CTA loads
  constexpr int kLoaded = kHalfBytes + kHalf * 128;  // bytes of a stage

  if (warp == 0) {
    if (lane == 0) {
      int st = 0;
      uint32_t ph = 0;
      for (int t = pair; t < total && !failed; t += pairs) {
        const Tile q = tile_of<BN>(p, m_tiles, n_tiles, t);
        const int m0 = q.m0 + (int)rank * 128, n0 = q.n0 + (int)rank * kHalf;
        for (int kc = 0; kc < q.chunks; ++kc) {
          if (!mbar_wait(empty + 8 * st, ph ^ 1u)) { failed = true; break; }
          if (rank == 0) mbar_expect_tx(full + 8 * st, 2 * kLoaded);
          const uint32_t a = smem_u32(tiles + st * kStageBytes), b = a + kHalfBytes;
          const uint32_t bar = map_to_rank(full + 8 * st, 0);
          const int k = q.k0 + kc * 64;
          if (A_MN) {
            tma_load_2d_pair(a, &tmA, m0, k, bar);
            tma_load_2d_pair(a + 8192, &tmA, m0 + 64, k, bar);
          } else {
            tma_load_2d_pair(a, &tmA, k, m0, bar);
          }
          if (B_MN) {
#pragma unroll
            for (int j = 0; j < kHalf / 64; ++j) tma_load_2d_pair(b + j * 8192, &tmB, n0 + j * 64, k, bar);
          } else {
            tma_load_2d_pair(b, &tmB, k, n0, bar);
          }
          if (++st == kStages) { st = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    if (rank == 0) {  // all 32 lanes walk the loop (uniform operands); one elected lane issues
      const uint32_t idesc = instr_desc_bf16(256, BN, A_MN, B_MN);
      int st = 0, buf = 0;
      uint32_t ph = 0, aph = 0;
      for (int t = pair; t < total && !failed; t += pairs) {
        const Tile q = tile_of<BN>(p, m_tiles, n_tiles, t);
        if (q.chunks == 0) continue;
        if (!mbar_wait_warp(tempty + 8 * buf, aph ^ 1u)) { failed = true; break; }
        tc_fence_after();
        const uint32_t acc = tmem + (uint32_t)buf * 256u;
        for (int kc = 0; kc < q.chunks; ++kc) {
          if (!mbar_wait_warp(full + 8 * st, ph)) { failed = true; break; }
          tc_fence_after();
          const uint32_t a = smem_u32(tiles + st * kStageBytes);
          // K-major: rows 128 bytes apart, 16 elements of K are 32 bytes on.  M/N-major: boxes of 64 elements 8192 bytes
          // apart, 16 elements of K are 16 rows of 128 bytes on.
          const uint64_t ad = smem_desc_sw128(a, A_MN ? 8192 : 16, 1024);
          const uint64_t bd = smem_desc_sw128(a + kHalfBytes, B_MN ? 8192 : 16, 1024);
#pragma unroll
          for (int k4 = 0; k4 < 4; ++k4)
            mma_bf16_pair(acc, ad + (uint64_t)(k4 * (A_MN ? 128 : 2)), bd + (uint64_t)(k4 * (B_MN ? 128 : 2)), idesc,
                          (kc | k4) != 0);
          mma_commit_pair(empty + 8 * st, 3);
          if (++st == kStages) { st = 0; ph ^= 1u; }
        }
        if (failed) break;
        mma_commit_pair(tfull + 8 * buf, 3);
        buf ^= 1;
        if (buf == 0) aph ^= 1u;
      }
    }
  } else {
    const int quad = warp & 3, half = (warp - 2) >> 2;
    unsigned char *stage = staging + (warp - 2) * kStageTile;
    int buf = 0;
    uint32_t aph = 0;
    for (int t = pair; t < total; t += pairs) {
      const Tile q = tile_of<BN>(p, m_tiles, n_tiles, t);
      const int row = q.m0 + (int)rank * 128 + quad * 32 + lane, n0 = q.n0 + half * kHalf;
      const uint32_t taddr = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(buf * 256 + half * kHalf);
      const uint32_t release = map_to_rank(tempty + 8 * buf, 0);
      if (q.chunks > 0) {
        if (!__all_sync(0xffffffffu, mbar_wait(tfull + 8 * buf, aph))) { failed = true; break; }
        tc_fence_after();
      }
      if (EPI == kLogits)
        logits_epilogue<kHalf>(p, q, (q.n0 / BN) * 2 + half, taddr, row, n0, stage, lane, release);
      else if (EPI == kFeatureGrad)
        feature_epilogue<BN>(p, q, taddr, row, rows, n0, stage, lane, release);
      else
        weight_epilogue<BN>(p, q, taddr, row, n0, stage, lane, release);
      if (q.chunks > 0) {
        buf ^= 1;
        if (buf == 0) aph ^= 1u;
      }
    }
  }
  if (failed) atomicExch(p.status, 1);
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // neither CTA leaves while the other may still touch its shared or tensor memory
  if (warp == 1) tmem_dealloc_pair(tmem, kTmem);
}

// ---- which rows count ------------------------------------------------------------------------------
constexpr int kSegment = 1024;  // rows of one block below, within one partition
constexpr int kRowThreads = 256;

struct RowArgs {
  const __nv_bfloat16 *x;
  long long ldx;
  int d, d_pad;
  int rows, each, parts, segments;  // rows of this piece, per partition; segments per partition
  int n_classes, pack;
  const int *labels;
  const float *weight;  // null: 1
  int *header;          // [0] status, [1] packed rows
  int *counts, *begin;  // rows that count per segment; first packed row of each partition (parts + 1)
  int *position;        // row -> packed row, -1: left out
  int *source, *label;  // packed row -> row, its label (-1: left out, or no row)
  float *row_weight;
  __nv_bfloat16 *packed;
  float *logp, *row_loss;
  __nv_bfloat16 *dx;
  long long ld_dx;
  DropoutKey drop;
  int first_piece;
};

__device__ __forceinline__ bool counts_row(const RowArgs &a, int row) {
  const int y = a.labels[row];
  return y >= 0 && y < a.n_classes && (!a.weight || a.weight[row] != 0.f);
}
__device__ __forceinline__ int round_up(int v) { return (v + kAlign - 1) / kAlign * kAlign; }

template <typename T>
__device__ __forceinline__ T block_sum(T v, T *scratch) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  T s = 0;
#pragma unroll
  for (int i = 0; i < kRowThreads / 32; ++i) s += scratch[i];
  return s;
}

// Rows first + 4 t .. + 3 of thread t that count, as bits, and the number of those before them in the segment.
__device__ __forceinline__ uint32_t scan_segment(const RowArgs &a, int first, int n, int *before, int *total, int *scratch) {
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = (int)threadIdx.x * 4 + i;
    if (r < n && counts_row(a, first + r)) bits |= 1u << i;
  }
  int v = __popc(bits);
  const int lane = threadIdx.x & 31, mine = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  __syncthreads();
  if (lane == 31) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  int base = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kRowThreads / 32; ++i) {
    if (i < (int)(threadIdx.x >> 5)) base += scratch[i];
    all += scratch[i];
  }
  *before = base + v - mine;
  *total = all;
  return bits;
}

__global__ void __launch_bounds__(kRowThreads) vocab_count_kernel(const RowArgs a) {
  pdl_sync();
  __shared__ int scratch[kRowThreads / 32];
  const int part = blockIdx.x / a.segments, first = part * a.each + (int)(blockIdx.x % a.segments) * kSegment;
  const int n = min(min(kSegment, (part + 1) * a.each - first), a.rows - first);
  int v = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = (int)threadIdx.x * 4 + i;
    if (r < n) v += counts_row(a, first + r) ? 1 : 0;
  }
  v = block_sum(v, scratch);
  if (threadIdx.x == 0) a.counts[blockIdx.x] = v;
}

// A left-out row's outputs.
__device__ __forceinline__ void leave_out(const RowArgs &a, int row) {
  a.logp[row] = 0.f;
  a.row_loss[row] = 0.f;
}

// What a segment's rows become: numbers of the packed rows and, for those, row, label and weight.
__device__ __forceinline__ void place_rows(const RowArgs &a, int first, int n, uint32_t bits, int at, int *position) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = (int)threadIdx.x * 4 + i, row = first + r;
    if (r >= n) break;
    const bool live = (bits >> i) & 1;
    position[r] = live ? at : -1;
    if (live) {
      a.source[at] = row;
      a.label[at] = a.labels[row];
      a.row_weight[at] = a.weight ? a.weight[row] : 1.f;
      ++at;
    } else {
      leave_out(a, row);
    }
  }
}
__device__ __forceinline__ void place_padding(const RowArgs &a, int from, int to) {
  for (int i = from + (int)threadIdx.x; i < to; i += kRowThreads) {
    a.source[i] = -1;
    a.label[i] = -1;
    a.row_weight[i] = 0.f;
  }
}

__global__ void __launch_bounds__(kRowThreads) vocab_place_kernel(const RowArgs a) {
  pdl_sync();
  __shared__ int scratch[kRowThreads / 32];
  const int part = blockIdx.x / a.segments, segment = blockIdx.x % a.segments;
  int base = 0;
  for (int p = threadIdx.x; p < part; p += kRowThreads) {
    int in = 0;
    for (int s = 0; s < a.segments; ++s) in += a.counts[p * a.segments + s];
    base += round_up(in);
  }
  for (int s = threadIdx.x; s < segment; s += kRowThreads) base += a.counts[part * a.segments + s];
  base = block_sum(base, scratch);
  const int first = part * a.each + segment * kSegment;
  const int n = max(0, min(min(kSegment, (part + 1) * a.each - first), a.rows - first));
  int before, total;
  const uint32_t bits = scan_segment(a, first, n, &before, &total, scratch);
  place_rows(a, first, n, bits, base + before, a.position + first);
  if (segment == a.segments - 1) {
    // (every partition begins at a multiple of 64)
    const int end = round_up(base + total);
    place_padding(a, base + total, end);
    if (threadIdx.x == 0) {
      a.begin[part + 1] = end;
      if (part == 0) a.begin[0] = 0;
      if (part == a.parts - 1) {
        a.header[1] = end;
        if (a.first_piece) a.header[0] = 0;
      }
    }
  }
}

// Rows stay where they are.
__global__ void __launch_bounds__(kRowThreads) vocab_keep_kernel(const RowArgs a) {
  pdl_sync();
  const int end = round_up(a.rows);
  for (int i = (int)(blockIdx.x * kRowThreads + threadIdx.x); i < end; i += (int)(gridDim.x * kRowThreads)) {
    const bool live = i < a.rows && counts_row(a, i);
    a.source[i] = i < a.rows ? i : -1;
    a.label[i] = live ? a.labels[i] : -1;
    a.row_weight[i] = live ? (a.weight ? a.weight[i] : 1.f) : 0.f;
    if (i < a.rows && !live) leave_out(a, i);
  }
  for (int i = (int)(blockIdx.x * kRowThreads + threadIdx.x); i <= a.parts; i += (int)(gridDim.x * kRowThreads))
    a.begin[i] = (int)min((long long)i * a.each, (long long)end);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.header[1] = end;
    if (a.first_piece) a.header[0] = 0;
  }
}

__device__ __forceinline__ uint4 load8(const __nv_bfloat16 *p, int n) {
  if (n >= 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) return *reinterpret_cast<const uint4 *>(p);
  const uint16_t *s = reinterpret_cast<const uint16_t *>(p);
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = 2 * i < n ? s[2 * i] : 0, hi = 2 * i + 1 < n ? s[2 * i + 1] : 0;
    w[i] = lo | hi << 16;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// One row by a warp: to its place among the packed rows (dropped features are zero there; the others are stretched in
// the scale of the logits and of G instead, which rounds nothing), or, left out, its gradient to zero.
__device__ __forceinline__ void move_row(const RowArgs &a, int row, int to, int lane) {
  if (to >= 0) {
    const __nv_bfloat16 *src = a.x + (long long)row * a.ldx;
    uint4 *dst = reinterpret_cast<uint4 *>(a.packed + (long long)to * a.d_pad);
    const int blocks = a.d_pad / 8;
    for (int b = lane; b < blocks; b += 32) {
      const int n = a.d - b * 8;
      uint4 v = n > 0 ? load8(src + b * 8, n) : make_uint4(0u, 0u, 0u, 0u);
      if (a.drop.threshold && n > 0) {
        const Keep8 keep = dropout_keep8(a.drop, (uint64_t)row, (uint32_t)b);
        uint32_t *w = &v.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] &= keep.halves(i);
      }
      dst[b] = v;
    }
  } else if (a.dx) {
    __nv_bfloat16 *dst = a.dx + (long long)row * a.ld_dx;
    for (int b = lane; b < (a.d + 7) / 8; b += 32) store8(dst + b * 8, make_uint4(0u, 0u, 0u, 0u), a.d - b * 8);
  }
}
__device__ __forceinline__ void clear_row(const RowArgs &a, int at, int lane) {
  uint4 *dst = reinterpret_cast<uint4 *>(a.packed + (long long)at * a.d_pad);
  for (int b = lane; b < a.d_pad / 8; b += 32) dst[b] = make_uint4(0u, 0u, 0u, 0u);
}

// A warp per row, then per row of padding that a partition may have.
__global__ void __launch_bounds__(kRowThreads) vocab_move_kernel(const RowArgs a) {
  pdl_sync();
  const int lane = threadIdx.x & 31;
  const long long job = (long long)blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5);
  if (job < a.rows) {
    move_row(a, (int)job, a.position[job], lane);
  } else {
    const long long part = (job - a.rows) / kAlign;
    if (part >= a.parts) return;
    const int at = a.begin[part + 1] - 1 - (int)((job - a.rows) % kAlign);
    if (at >= a.begin[part] && a.source[at] < 0) clear_row(a, at, lane);
  }
}

// The same in one launch for one partition of one segment: every block works out all positions.
__global__ void __launch_bounds__(kRowThreads) vocab_pack_kernel(const RowArgs a) {
  pdl_sync();
  __shared__ int scratch[kRowThreads / 32], position[kSegment];
  int before, total;
  const uint32_t bits = scan_segment(a, 0, a.rows, &before, &total, scratch);
  const int end = round_up(total);
  if (blockIdx.x == 0) {
    place_rows(a, 0, a.rows, bits, before, position);
    place_padding(a, total, end);
    if (threadIdx.x == 0) {
      a.begin[0] = 0;
      a.begin[1] = end;
      a.header[1] = end;
      if (a.first_piece) a.header[0] = 0;
    }
  } else {
    int at = before;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool live = (bits >> i) & 1;
      position[threadIdx.x * 4 + i] = live ? at : -1;
      at += live ? 1 : 0;
    }
  }
  __syncthreads();
  const int lane = threadIdx.x & 31, job = (int)blockIdx.x * (kRowThreads / 32) + (int)(threadIdx.x >> 5);
  if (job < a.rows) {
    move_row(a, job, position[job], lane);
  } else if (total + job - a.rows < end) {
    clear_row(a, total + job - a.rows, lane);
  }
}

// A matrix with rows that bulk copies cannot read, to one with rows of whole 128 bytes; a warp per row.
__global__ void __launch_bounds__(kRowThreads)
vocab_copy_kernel(const __nv_bfloat16 *src, long long ld, int rows, int columns, __nv_bfloat16 *dst, int ld_dst) {
  pdl_sync();
  const int lane = threadIdx.x & 31;
  for (int row = (int)(blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5)); row < rows; row += (int)gridDim.x * (kRowThreads / 32))
    for (int b = lane; b < ld_dst / 8; b += 32) {
      const int n = columns - b * 8;
      reinterpret_cast<uint4 *>(dst + (long long)row * ld_dst)[b] =
          n > 0 ? load8(src + (long long)row * ld + b * 8, n) : make_uint4(0u, 0u, 0u, 0u);
    }
}

// ---- losses, and powers to G ------------------------------------------------------------------------
struct LossArgs {
  const int *header, *source, *label;
  const float *weight, *label_z;
  const float2 *stat;
  int stats, width;  // width: classes per statistic
  float *logp, *row_loss;
  __half *power;
  long long ld_power;
  float factor;  // scale (and what dropout stretches features by)
};

__device__ __forceinline__ float2 join(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x);
  // (an empty set's maximum is -infinity; two of them must not be subtracted)
  return make_float2(m, (a.x == kNegInf ? a.y : a.y * power2(a.x - m)) + (b.x == kNegInf ? b.y : b.y * power2(b.x - m)));
}

// T threads per packed row: the row's statistics joined, its loss, and its powers e turned into
// G = factor w (e 2^(m - lse) - onehot), each group of classes with its own m.
template <int T>
__global__ void __launch_bounds__(256) vocab_loss_kernel(const LossArgs a) {
  pdl_sync();
  __shared__ float2 part[8];
  const int row = (int)(blockIdx.x * (256 / T) + threadIdx.x / T), t = threadIdx.x % T;
  if (row >= a.header[1]) return;  // (T = 256: the whole block; T = 32: whole warps)
  const int label = a.label[row];
  uint4 *power = reinterpret_cast<uint4 *>(a.power + (long long)row * a.ld_power);
  const int vectors = (int)(a.ld_power / 8);
  if (label < 0) {  // padding, or left out
    if (a.power)
      for (int v = t; v < vectors; v += T) power[v] = make_uint4(0u, 0u, 0u, 0u);
    return;
  }
  const float2 *stat = a.stat + (long long)row * a.stats;
  float2 s = make_float2(kNegInf, 0.f);
  for (int i = t; i < a.stats; i += T) s = join(s, stat[i]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    s = join(s, make_float2(__shfl_xor_sync(0xffffffffu, s.x, o), __shfl_xor_sync(0xffffffffu, s.y, o)));
  if (T > 32) {
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
    __syncthreads();
    s = part[0];
#pragma unroll
    for (int i = 1; i < T / 32; ++i) s = join(s, part[i]);
  }
  const float lse = s.x + log2f(s.y), logp = (a.label_z[row] - s.x - log2f(s.y)) * kLn2, w = a.weight[row];
  if (t == 0) {
    a.logp[a.source[row]] = logp;
    a.row_loss[a.source[row]] = -w * logp;
  }
  if (!a.power) return;
  const float g = a.factor * w, at_label = g * expm1f(logp);
  const int per = a.width / 8;  // vectors per statistic
  for (int v = t; v < vectors; v += T) {
    uint4 q = power[v];
    const int group = v / per;
    const float f = group < a.stats ? g * power2(stat[group].x - lse - (float)kPowerBits) : 0.f;
    uint32_t *x = &q.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 e = __half22float2(*reinterpret_cast<const __half2 *>(&x[i]));
      const int c = v * 8 + 2 * i;
      x[i] = pack_bf16(c == label ? at_label : e.x * f, c + 1 == label ? at_label : e.y * f);
    }
    power[v] = q;
  }
}

// dX from the shares of K: their sum, dropped features zero; a thread per 8 columns.
struct JoinArgs {
  const int *header, *source, *label;
  const float *partial;
  int m, n, n_pad, splits;
  __nv_bfloat16 *out;
  long long ld_out;
  DropoutKey drop;
};
__global__ void __launch_bounds__(256) vocab_join_kernel(const JoinArgs a) {
  pdl_sync();
  const int blocks = (a.n + 7) / 8, rows = a.header[1];
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < (long long)rows * blocks; i += (long long)gridDim.x * 256) {
    const int row = (int)(i / blocks), b = (int)(i % blocks), src = a.source[row];
    if (src < 0) continue;
    float v[8] = {};
    if (a.label[row] >= 0) {
      for (int s = 0; s < a.splits; ++s) {
        const float4 *p = reinterpret_cast<const float4 *>(a.partial + ((long long)s * a.m + row) * a.n_pad + b * 8);
        const float4 lo = p[0], hi = p[1];
        v[0] += lo.x; v[1] += lo.y; v[2] += lo.z; v[3] += lo.w;
        v[4] += hi.x; v[5] += hi.y; v[6] += hi.z; v[7] += hi.w;
      }
      if (a.drop.threshold) {
        const Keep8 keep = dropout_keep8(a.drop, (uint64_t)src, (uint32_t)b);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = keep[j] ? v[j] : 0.f;
      }
    }
    store8(a.out + (long long)src * a.ld_out + b * 8,
           make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])), a.n - b * 8);
  }
}

}  // namespace
}  // namespace ngc

// ---- host -------------------------------------------------------------------------------------------
namespace ngc {
namespace {

constexpr size_t kPieceBytes = (size_t)1 << 30;  // room for powers (without a gradient: statistics and features) of a piece
constexpr long long kMostPiece = 1ll << 24;      // rows of a piece

inline long long up(long long v, long long a) { return (v + a - 1) / a * a; }

struct VocabPlan {
  long long each;      // rows per partition, as the weights' gradient sees them
  long long parts;     // partitions
  long long piece_parts, subs, sub_rows;  // partitions of a piece, or pieces of a partition and their rows
  long long cap;       // packed rows of a piece at most, a multiple of 256
  int bn, stats, d_pad, ld_power, splits;
  int w_inner, w_outer, w_pad;  // the weights' rows: elements, number, elements of a copied one (0: not copied)
  int sums_m, sums_pad;
  size_t header, counts, begin, position, source, label, weight, label_z, stat, packed, copy, power, partial, sums, bytes;
};

// How the products of a shape are cut for `pairs` CTA pairs.  The narrower tile reads the features twice as often per class; it
// is taken where it leaves fewer pairs idle in the last round.
inline int logits_width(long long rows, int classes, int pairs) {
  const long long m = (rows + 255) / 256;
  const long long wide = (m * ((classes + 255) / 256) + pairs - 1) / pairs * 256;
  const long long narrow = (m * ((classes + 127) / 128) + pairs - 1) / pairs * 128;
  return narrow * 10 < wide * 9 ? 128 : 256;
}
// Shares of K for the features' gradient, whose tiles are few when rows are: the fewest rounds of work, a share at least
// 16 chunks long.
inline int feature_splits(long long rows, int d, int classes, int pairs) {
  const long long tiles = (rows + 255) / 256 * ((d + 255) / 256), chunks = (classes + 63) / 64;
  int best = 1;
  double best_time = 1e300;
  for (int s = 1; s <= 64 && s * 16 <= chunks; ++s) {
    const double rounds = (double)((tiles * s + pairs - 1) / pairs) / s;
    const double time = rounds * (s > 1 ? 1.02 + 0.01 * s : 1.0);
    if (time < best_time) { best_time = time; best = s; }
  }
  return best;
}

VocabPlan vocab_plan(const ngc_linear_ce_t &c, const void *W, long long ld_w, bool dx, bool dw, int sms) {
  VocabPlan p = {};
  const bool grads = dx || dw;
  const int pairs = std::max(1, sms / 2);
  p.each = dw ? std::min<long long>(c.rows_per_partition, std::max<int64_t>(1, c.rows)) : std::max<int64_t>(1, c.rows);
  p.parts = (c.rows + p.each - 1) / p.each;
  p.d_pad = (int)up(c.d, 64);
  p.ld_power = (int)up(c.n_classes, 64);
  const size_t per_row = grads ? (size_t)p.ld_power * 2 : (size_t)(c.n_classes + 127) / 128 * 16 + (size_t)p.d_pad * 2;
  long long most = c.piece_rows > 0 ? c.piece_rows : (long long)std::max<size_t>(256, kPieceBytes / per_row / 256 * 256);
  most = std::min(most, kMostPiece);
  long long rows;  // of a piece
  if (p.each <= most) {
    const long long taken = c.keep_rows ? p.each : up(p.each, kAlign);
    p.piece_parts = std::min(std::max<long long>(1, most / taken), std::max<long long>(1, p.parts));
    p.subs = 1;
    p.sub_rows = p.each;
    rows = std::min<long long>(p.piece_parts * p.each, std::max<int64_t>(1, c.rows));
    p.cap = c.keep_rows ? rows : p.piece_parts * taken;
  } else {
    p.piece_parts = 1;
    p.subs = (p.each + most - 1) / most;
    p.sub_rows = up((p.each + p.subs - 1) / p.subs, kAlign);
    p.subs = (p.each + p.sub_rows - 1) / p.sub_rows;
    rows = p.sub_rows;
    p.cap = rows;
  }
  p.cap = up(p.cap, 256);
  p.bn = logits_width(rows, c.n_classes, pairs);
  p.stats = 2 * ((c.n_classes + p.bn - 1) / p.bn);
  p.splits = dx ? feature_splits(rows, c.d, c.n_classes, pairs) : 1;
  p.w_inner = c.feature_major ? c.n_classes : c.d;
  p.w_outer = c.feature_major ? c.d : c.n_classes;
  const bool copy = !aligned(W, 16) || ld_w % 8 != 0;
  p.w_pad = copy ? (int)up(p.w_inner, 64) : 0;
  p.sums_m = c.feature_major ? c.d : c.n_classes;
  p.sums_pad = (int)up(p.w_inner, 8);
  const long long segments = (std::min(p.each, rows) + kSegment - 1) / kSegment;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  p.header = take(256);
  p.counts = take((size_t)(p.piece_parts * segments) * 4);
  p.begin = take((size_t)(p.piece_parts + 1) * 4);
  p.position = take((size_t)rows * 4);
  p.source = take((size_t)p.cap * 4);
  p.label = take((size_t)p.cap * 4);
  p.weight = take((size_t)p.cap * 4);
  p.label_z = take((size_t)p.cap * 4);
  p.stat = take((size_t)p.cap * p.stats * sizeof(float2));
  p.packed = take(c.keep_rows ? 0 : (size_t)p.cap * p.d_pad * 2);
  p.copy = take((size_t)p.w_pad * p.w_outer * 2);
  p.power = take(grads ? (size_t)p.cap * p.ld_power * 2 : 0);
  p.partial = take(p.splits > 1 ? (size_t)p.splits * p.cap * p.d_pad * 4 : 0);
  p.sums = take(dw && p.subs > 1 ? (size_t)p.sums_m * p.sums_pad * 4 : 0);
  p.bytes = at;
  return p;
}

typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {
  static const EncodeTiled fn = [] {
    void *ptr = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      ptr = nullptr;
    return reinterpret_cast<EncodeTiled>(ptr);
  }();
  return fn;
}

// bf16 rows of `inner` elements, `ld` apart; boxes of 64 x `box` in 128-byte swizzle; zero outside.
bool row_map(CUtensorMap *m, const void *base, long long inner, long long rows, long long ld, int box) {
  const EncodeTiled fn = encode_tiled();
  if (!fn) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)rows}, stride[1] = {(cuuint64_t)ld * 2};
  const cuuint32_t boxes[2] = {64, (cuuint32_t)box}, steps[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(base), dims, stride, boxes, steps,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int EPI, int A_MN, int B_MN, int BN>
cudaError_t launch_gemm(const CUtensorMap &a, const CUtensorMap &b, const GemmArgs &p, long long tiles, int sms,
                        cudaStream_t stream) {
  auto kern = vocab_gemm_kernel<EPI, A_MN, B_MN, BN>;
  // (the opt-in shared-memory size is set once per device; setting it twice does no harm)
  static std::atomic<uint64_t> ready{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (!(ready.load(std::memory_order_acquire) & bit)) {
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
    ready.fetch_or(bit, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(2 * std::max<long long>(1, std::min<long long>(tiles, sms / 2))));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kern, a, b, p);
}

// What dropout multiplies the features by (where nothing is left of them: by anything).
inline double vocab_stretch(double p) {
  const uint32_t t = dropout_threshold(p);
  return t < 65536 ? 65536.0 / (65536 - t) : 1.0;
}

struct VocabCall {
  const ngc_linear_ce_t *cfg;
  const __nv_bfloat16 *x, *w;
  long long ldx, ldw;
  const int *labels;
  const float *row_weight;
  __nv_bfloat16 *dx, *dw;
  long long ld_dx, ld_dw, dw_part;
  float *logp, *row_loss;
  unsigned char *ws;
  int sms;
  cudaStream_t stream;
};

// One piece: `rows` rows from `first` on, `parts` partitions of `each` rows (the last may be short), the number of the
// first; begin / end: of the pieces that a partition is cut into.
cudaError_t vocab_piece(const VocabCall &q, const VocabPlan &p, long long first, int rows, int each, int parts,
                        long long first_part, bool begin, bool end) {
  const ngc_linear_ce_t &c = *q.cfg;
  const DropoutKey drop = {c.seed, c.first_row + (uint64_t)first, c.step, dropout_threshold(c.dropout)};
  const double stretch = vocab_stretch(c.dropout);
  int *header = reinterpret_cast<int *>(q.ws + p.header);
  RowArgs r = {};
  r.x = q.x + first * q.ldx;
  r.ldx = q.ldx; r.d = c.d; r.d_pad = p.d_pad;
  r.rows = rows; r.each = each; r.parts = parts; r.segments = (std::min(each, rows) + kSegment - 1) / kSegment;
  r.n_classes = c.n_classes; r.pack = !c.keep_rows;
  r.labels = q.labels + first;
  r.weight = q.row_weight ? q.row_weight + first : nullptr;
  r.header = header;
  r.counts = reinterpret_cast<int *>(q.ws + p.counts);
  r.begin = reinterpret_cast<int *>(q.ws + p.begin);
  r.position = reinterpret_cast<int *>(q.ws + p.position);
  r.source = reinterpret_cast<int *>(q.ws + p.source);
  r.label = reinterpret_cast<int *>(q.ws + p.label);
  r.row_weight = reinterpret_cast<float *>(q.ws + p.weight);
  r.packed = reinterpret_cast<__nv_bfloat16 *>(q.ws + p.packed);
  r.logp = q.logp + first;
  r.row_loss = q.row_loss + first;
  r.dx = q.dx ? q.dx + first * q.ld_dx : nullptr;
  r.ld_dx = q.ld_dx;
  r.drop = drop;
  r.first_piece = first == 0;
  cudaError_t e;
  constexpr int kWarps = kRowThreads / 32;
  if (c.keep_rows) {
    e = launch_k(vocab_keep_kernel, std::max(1, std::min(1024, (rows + kRowThreads - 1) / kRowThreads)), kRowThreads, 0, q.stream, r);
  } else if (parts == 1 && rows <= kSegment) {
    e = launch_k(vocab_pack_kernel, (rows + kAlign - 1 + kWarps - 1) / kWarps, kRowThreads, 0, q.stream, r);
  } else {
    e = launch_k(vocab_count_kernel, parts * r.segments, kRowThreads, 0, q.stream, r);
    if (e == cudaSuccess) e = launch_k(vocab_place_kernel, parts * r.segments, kRowThreads, 0, q.stream, r);
    const long long jobs = (long long)rows + (long long)parts * kAlign;
    if (e == cudaSuccess) e = launch_k(vocab_move_kernel, (unsigned)((jobs + kWarps - 1) / kWarps), kRowThreads, 0, q.stream, r);
  }
  if (e != cudaSuccess) return e;

  const bool grads = q.dx || q.dw;
  const void *xp = c.keep_rows ? (const void *)r.x : (const void *)r.packed;
  const long long x_rows = c.keep_rows ? rows : p.cap, x_ld = c.keep_rows ? q.ldx : p.d_pad;
  const void *w = p.w_pad ? (const void *)(q.ws + p.copy) : (const void *)q.w;
  const long long w_ld = p.w_pad ? p.w_pad : q.ldw;
  void *power = q.ws + p.power;
  CUtensorMap a, b;
  GemmArgs g = {};
  g.batch = 1; g.splits = 1; g.group = 16;
  g.status = header;
  g.source = r.source; g.label = r.label;
  const int m_tiles = (int)((up(rows, kAlign) + (long long)(parts - 1) * kAlign + 255) / 256);

  // logits
  g.m = (int)p.cap; g.m_dev = header + 1; g.n = c.n_classes; g.k = c.d;
  g.label_z = reinterpret_cast<float *>(q.ws + p.label_z);
  g.stat = reinterpret_cast<float2 *>(q.ws + p.stat);
  g.stats = p.stats;
  g.c = (float)(c.scale * stretch * 1.4426950408889634);
  g.power = grads ? static_cast<__half *>(power) : nullptr;
  g.ld_power = p.ld_power;
  if (!row_map(&a, xp, c.d, x_rows, x_ld, 128)) return cudaErrorInvalidValue;
  if (!row_map(&b, w, p.w_inner, p.w_outer, w_ld, c.feature_major ? 64 : p.bn / 2)) return cudaErrorInvalidValue;
  const long long logit_tiles = (long long)m_tiles * ((c.n_classes + p.bn - 1) / p.bn);
  if (c.feature_major)
    e = p.bn == 256 ? launch_gemm<kLogits, 0, 1, 256>(a, b, g, logit_tiles, q.sms, q.stream)
                    : launch_gemm<kLogits, 0, 1, 128>(a, b, g, logit_tiles, q.sms, q.stream);
  else
    e = p.bn == 256 ? launch_gemm<kLogits, 0, 0, 256>(a, b, g, logit_tiles, q.sms, q.stream)
                    : launch_gemm<kLogits, 0, 0, 128>(a, b, g, logit_tiles, q.sms, q.stream);
  if (e != cudaSuccess) return e;

  LossArgs l = {};
  l.header = header; l.source = r.source; l.label = r.label; l.weight = r.row_weight; l.label_z = g.label_z; l.stat = g.stat;
  l.stats = p.stats; l.width = p.bn / 2;
  l.logp = r.logp; l.row_loss = r.row_loss;
  l.power = g.power; l.ld_power = p.ld_power;
  l.factor = (float)(c.scale * stretch);
  const long long most = up(rows, kAlign) + (c.keep_rows ? 0 : (long long)(parts - 1) * kAlign);
  e = c.n_classes <= 2048 ? launch_k(vocab_loss_kernel<32>, (unsigned)((most + 7) / 8), 256, 0, q.stream, l)
                          : launch_k(vocab_loss_kernel<256>, (unsigned)most, 256, 0, q.stream, l);
  if (e != cudaSuccess) return e;

  if (q.dx) {
    g.n = c.d; g.k = c.n_classes; g.splits = p.splits;
    g.out = r.dx; g.ld_out = q.ld_dx;
    g.partial = reinterpret_cast<float *>(q.ws + p.partial);
    g.n_pad = p.d_pad;
    g.drop = drop;
    if (!row_map(&a, power, p.ld_power, p.cap, p.ld_power, 128)) return cudaErrorInvalidValue;
    if (!row_map(&b, w, p.w_inner, p.w_outer, w_ld, c.feature_major ? 128 : 64)) return cudaErrorInvalidValue;
    const long long tiles = (long long)m_tiles * ((c.d + 255) / 256) * p.splits;
    e = c.feature_major ? launch_gemm<kFeatureGrad, 0, 0, 256>(a, b, g, tiles, q.sms, q.stream)
                        : launch_gemm<kFeatureGrad, 0, 1, 256>(a, b, g, tiles, q.sms, q.stream);
    if (e == cudaSuccess && p.splits > 1) {
      JoinArgs j = {header, r.source, r.label, g.partial, (int)p.cap, c.d, p.d_pad, p.splits, r.dx, q.ld_dx, drop};
      const long long work = (most * ((c.d + 7) / 8) + 255) / 256;
      e = launch_k(vocab_join_kernel, (unsigned)std::min<long long>(work, q.sms * 16), 256, 0, q.stream, j);
    }
    if (e != cudaSuccess) return e;
  }
  if (q.dw) {
    g.splits = 1; g.m_dev = nullptr;
    g.k_begin = r.begin; g.batch = parts;
    g.out = q.dw + first_part * q.dw_part; g.ld_out = q.ld_dw; g.out_batch = q.dw_part;
    g.partial = p.subs > 1 ? reinterpret_cast<float *>(q.ws + p.sums) : nullptr;
    g.n_pad = p.sums_pad;
    g.first = begin; g.last = end;
    g.m = p.w_outer; g.n = p.w_inner;
    CUtensorMap powers, features;
    if (!row_map(&powers, power, p.ld_power, p.cap, p.ld_power, 64)) return cudaErrorInvalidValue;
    if (!row_map(&features, xp, c.d, x_rows, x_ld, 64)) return cudaErrorInvalidValue;
    const long long tiles = (long long)((g.m + 255) / 256) * ((g.n + 255) / 256) * parts;
    e = launch_gemm<kWeightGrad, 1, 1, 256>(c.feature_major ? features : powers, c.feature_major ? powers : features, g, tiles,
                                            q.sms, q.stream);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

bool vocab_config_ok(const ngc_linear_ce_t *c, const void *W, int64_t ld_w) {
  if (!c || c->rows < 0 || c->rows > 0x7fffffffll || c->rows_per_partition < 1 || c->piece_rows < 0 || c->d < 1 ||
      c->d > (1 << 20) || c->n_classes < 1 || c->n_classes > (1 << 24))
    return false;
  if (!(c->dropout >= 0.0 && c->dropout <= 1.0)) return false;
  const float coef = (float)(c->scale * vocab_stretch(c->dropout) * 1.4426950408889634);
  if (!(c->scale > 0.0) || !std::isfinite(coef) || !((float)c->scale > 0.f)) return false;
  const long long inner = c->feature_major ? c->n_classes : c->d;
  return W && aligned(W, 2) && ld_w >= inner && ld_w <= 1ll << 32;
}

}  // namespace
}  // namespace ngc

extern "C" {

size_t ngc_linear_cross_entropy_workspace_bytes(const ngc_linear_ce_t *cfg, const void *W, int64_t ld_w, int with_dx, int with_dw) {
  using namespace ngc;
  if (!vocab_config_ok(cfg, W, ld_w)) return 0;
  return vocab_plan(*cfg, W, ld_w, with_dx != 0, with_dw != 0, std::max(2, device_sm_count())).bytes;
}

int ngc_linear_cross_entropy(const ngc_linear_ce_t *cfg, const void *X, int64_t ld_x, const void *W, int64_t ld_w,
                             const int32_t *labels, const float *row_weight, void *dX, int64_t ld_dx, void *dW, int64_t ld_dw,
                             int64_t dw_stride, float *logp, float *row_loss, float *loss, void *workspace,
                             size_t workspace_bytes, void *cuda_stream) {
  using namespace ngc;
  if (!vocab_config_ok(cfg, W, ld_w)) return NGC_ERR_INVALID;
  const ngc_linear_ce_t &c = *cfg;
  const long long rows = c.rows, far = (1ll << 44) / (rows + 1);
  const long long inner = c.feature_major ? c.n_classes : c.d, outer = c.feature_major ? c.d : c.n_classes;
  const long long all_parts = rows == 0 ? 1 : (rows - 1) / c.rows_per_partition + 1;
  if (!aligned(dW, 2) || (dW && (ld_dw < inner || ld_dw > 1ll << 32 || (all_parts > 1 && dw_stride < (outer - 1) * ld_dw + inner) ||
                                 dw_stride > (1ll << 44) / all_parts)))
    return NGC_ERR_INVALID;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  if (rows == 0) {
    if (dW && cudaMemset2DAsync(dW, (size_t)ld_dw * 2, 0, (size_t)inner * 2, (size_t)outer, stream) != cudaSuccess) return NGC_ERR_CUDA;
    return NGC_OK;
  }
  if (!X || !labels || !logp || !row_loss || !workspace || !aligned(workspace, 256) || !aligned(X, 2) || !aligned(dX, 2) ||
      ld_x < c.d || ld_x > far || (dX && (ld_dx < c.d || ld_dx > far)))
    return NGC_ERR_INVALID;
  for (const void *p : {(const void *)labels, (const void *)row_weight, (const void *)logp, (const void *)row_loss, (const void *)loss})
    if (!aligned(p, 4)) return NGC_ERR_INVALID;
  const int sms = device_sm_count();
  if (sms <= 0) return NGC_ERR_CUDA;
  if (sms < 2) return NGC_ERR_INVALID;
  const VocabPlan p = vocab_plan(c, W, ld_w, dX != nullptr, dW != nullptr, sms);
  if (workspace_bytes < p.bytes) return NGC_ERR_INVALID;
  // rows that stay where they are: bulk copies have to be able to read them, dropout would change them, and a K chunk of
  // 64 rows must not hold two partitions
  if (c.keep_rows && (!aligned(X, 16) || ld_x % 8 != 0 || c.dropout != 0.0 || (p.parts > 1 && p.each % kAlign != 0)))
    return NGC_ERR_INVALID;
  const size_t vec = (size_t)rows * 4;
  const Span x = matrix_span(X, rows, c.d, ld_x, 2), w = matrix_span(W, outer, (int)inner, ld_w, 2);
  const Span gx = matrix_span(dX, rows, c.d, ld_dx, 2);
  const Span gw(dW, (size_t)((all_parts - 1) * dw_stride + (outer - 1) * ld_dw + inner) * 2);
  const Span lab(labels, vec), weight(row_weight, vec), lp(logp, vec), row(row_loss, vec), sum(loss, (size_t)all_parts * 4);
  const Span ws(workspace, p.bytes);
  if (!apart(ws, {x, w, gx, gw, lab, weight, lp, row, sum}) || !apart(gx, {x, w, gw, lab, weight, lp, row, sum}) ||
      !apart(gw, {x, w, lab, weight, lp, row, sum}) || !apart(lp, {x, w, lab, weight, row, sum}) ||
      !apart(row, {x, w, lab, weight, sum}) || !apart(sum, {x, w, lab, weight}))
    return NGC_ERR_INVALID;
  VocabCall q = {cfg, static_cast<const __nv_bfloat16 *>(X), static_cast<const __nv_bfloat16 *>(W), ld_x, ld_w, labels, row_weight,
                 static_cast<__nv_bfloat16 *>(dX), static_cast<__nv_bfloat16 *>(dW), ld_dx, ld_dw, dw_stride, logp, row_loss,
                 static_cast<unsigned char *>(workspace), sms, stream};
  if (p.w_pad) {
    const unsigned blocks = (unsigned)std::min<long long>((outer + kRowThreads / 32 - 1) / (kRowThreads / 32), sms * 8);
    if (launch_k(vocab_copy_kernel, blocks, kRowThreads, 0, stream, q.w, (long long)ld_w, (int)outer, (int)inner,
                 reinterpret_cast<__nv_bfloat16 *>(q.ws + p.copy), p.w_pad) != cudaSuccess)
      return NGC_ERR_CUDA;
  }
  if (p.subs == 1) {
    for (long long part = 0; part < p.parts; part += p.piece_parts) {
      const long long n = std::min(p.piece_parts, p.parts - part), first = part * p.each;
      const long long here = std::min(rows - first, n * p.each);
      if (vocab_piece(q, p, first, (int)here, (int)std::min(p.each, here), (int)n, part, true, true) != cudaSuccess) return NGC_ERR_CUDA;
    }
  } else {
    for (long long part = 0; part < p.parts; ++part) {
      const long long first = part * p.each, last = std::min<long long>(rows, first + p.each);
      for (long long at = first; at < last; at += p.sub_rows) {
        const int here = (int)std::min(p.sub_rows, last - at);
        if (vocab_piece(q, p, at, here, here, 1, part, at == first, at + here == last) != cudaSuccess) return NGC_ERR_CUDA;
      }
    }
  }
  if (loss && launch_partition_sums(row_loss, (int)rows, c.rows_per_partition, loss, stream) != cudaSuccess) return NGC_ERR_CUDA;
  return NGC_OK;
}

}  // extern "C"

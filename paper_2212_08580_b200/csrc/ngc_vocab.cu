// ngc_linear_cross_entropy: softmax cross entropy over a large vocabulary straight from features X [rows][d] and weights W
// [classes][d] (or [d][classes]), with the gradients of both.
//
//   z = scale X W^T,  lse = log sum_v e^z,  G = scale w (e^(z - lse) - onehot),  dX = G W,  dW_j = G_j^T X_j.
//
// The logits are never stored.  The first contraction's epilogue turns each tile of them, straight from tensor memory, into
// its rows' maxima and sums of powers over 128 classes and, for a gradient, into 16-bit powers relative to those maxima (an
// error of 2^-11 of a power, or 2^-39 of the largest of its 128, whatever the logits' size: differences are taken before anything
// is multiplied).  One pass over the powers then has lse, losses, and G in their place in bf16: operands of the two gradient
// contractions are bf16, so its rounding to 8 bits is paid for their rate; dX and dW are rounded once more, to their type, and are 1.2 to
// 1.45 times as far off as by that alone (dW of a few rows up to 2.5 times, as a label's G scales all of its class's).  Taking the logits a
// second time from X and W instead would need no room for the powers, but a fourth contraction beside three (a third more time);
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
#include "ngc_words.cuh"

namespace ngc {

namespace {

using namespace tc;

constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLn2 = 0.6931471805599453f;
// A set's largest logit is stored as no less than this, so that a maximum of -infinity means an empty set and nothing else, and logits
// of -infinity have a difference to it.
constexpr float kLowest = -3.4028234663852886e38f;
// Powers are at most 1.  They are stored times 2^14, so that fp16 holds from 2^-38 on, with all its digits from 2^-28 on.
constexpr int kPowerBits = 14;
constexpr int kAlign = 64;      // packed rows of a partition are a multiple of a K chunk

// ---- contraction on CTA pairs --------------------------------------------------------------------
// C[M x N] = A B over tiles of 256 x BN (BN = 256 or 128).  Two CTAs of a cluster drive one 256-row MMA: each loads its own 128 rows of A
// and half of B's columns, and keeps its 128 rows of C in its own tensor memory.  Operands come through a ring of stages of 64 along K
// with 128-byte swizzle, either K-major or M/N-major (X^T, or W in the other layout, is never made).
//
// Single tiles (Wide false): the two accumulators take turns, so that a tile's epilogue runs beside the next one's contraction; six stages.
// The tensor cores are busy 94 % of the cycles in the gradients' contractions, and the clock falls to 1.3-1.45 GHz under the power limit:
// 4096 x 4096 x 16000 in 331 us, 1.62 PFLOP/s, where a library product reaches 1.64.  The logits' are busy 90 % (345 us), 74 % at 1024 features
// (2048 x 1024 x 65536 in 205 us): their accumulators are handed over every 256 features, and a tile's last epilogue takes longer
// than the next tile's first two runs.
// Units of two tiles that share an operand (Wide true): side by side, which share A, for the features' gradient, above each other, which
// share B, for the weights'.  A quarter less goes from L2 to shared memory, but the unit after waits until its first accumulator has been
// read out, and runs ahead on that one alone as far as its four stages go: busy 88 %, at 1.5 GHz.  This pays where a contraction is
// long: features' gradient of 6144 x 4096 x 32000 1078 -> 982 us, weights' 1058 -> 1018 us; but K = 512 139 instead of 113 us.  Units that
// would not fill a round of pairs are taken as single tiles.
constexpr int kHalfBytes = 16384;  // 128 x 64 bf16
constexpr int kMostFewRows = 128;  // packed ones too (two groups of 32 for each half of the epilogue's warps)
constexpr int kLongContraction = 96;  // chunks of 64: the weights' gradient takes units of two tiles from here on (64: 95 instead of 88 us)
// The tensor cores cut what does not fit into an accumulator instead of rounding it, once for every 16 products.  How much that is depends on
// the data: a sum that grows evenly to z loses (d / 16) 1.5e-8 of itself, features with one non-zero element lose nothing.  So the
// logits' accumulators begin anew every kSumChunks chunks of 64, and the epilogue adds what they held in fp32, rounding: at most 16 cuts in a
// row at any d.  (log p of 512 rows, standard normal features, d = 1024 .. 8192: 1.0e-6 off rms, where an fp32 product is 0.7e-6 .. 2.3e-6;
// logits that grow evenly to 100: 3e-6 .. 1.1e-5, fp32 2e-5 .. 2e-4.  Runs of 8 chunks are 1.9e-6 off and 1-2 % faster, 7 % at 256 classes; of 2,
// 0.7e-6 and 1-4 % slower, 8 % scoring 350 rows.)
constexpr int kSumChunks = 4;
constexpr int kThreads = 320;      // loads, MMA, 8 epilogue warps (two per quadrant of the 128 rows, half of the columns each)
constexpr int kStageTile = 32 * 128;  // a warp's 32 rows of 128 bytes on their way out
constexpr int kExchange = 2 * 128 * 8;  // kGradient: a row's statistics between the warps that share it (in place of a stage)
constexpr int kSmem = 12 * kHalfBytes + 8 * kStageTile + 256 + 1024;
constexpr int kTmem = 512;

// kLogits: statistics and powers; kGradient: losses and G at once, where a row's classes are one tile; kFeatureGrad, kWeightGrad.
// kFewRows: kLogits of few rows.  Classes take the M side and rows the N side, which is as wide as there are rows (in 32s).  How many
// classes a tile has (up to 256) is chosen so that the last round of pairs is full, as reading the weights is all that counts: one row
// of 4096 x 32000 69 -> 63 us, 64 rows of 1024 x 131072 68 -> 57 us; 200 rows 67 -> 89 us, as its epilogue (32 classes of a row lie
// in the lanes of a warp) costs more.
enum { kLogits = 0, kFeatureGrad = 1, kWeightGrad = 2, kGradient = 3, kFewRows = 4 };

// A row's outputs; loss: where a partition is one row, else null (sums are taken at the end).
struct RowOut {
  float *logp, *row_loss, *loss;
  __device__ __forceinline__ void put(int row, float lp, float l) const {
    logp[row] = lp;
    row_loss[row] = l;
    if (loss) loss[row] = l;
  }
};

struct GemmArgs {
  int m, n;                // extents of C; m_dev, where there is one, says how many packed rows there are (m, or kFewRows's n)
  const int *m_dev;
  int classes_each;        // kFewRows: of a CTA's tile, at most 128
  int few_rows;            // kFewRows: number of rows, where m_dev is null
  int k;                   // extent of the contraction
  const int *k_begin;      // per batch: first row of K (k_begin[batch + 1]: end), multiples of 64; null: 0 .. k
  int batch;
  int group;               // units along M that share B while it is in L2
  int store;               // kWeightGrad: results leave by bulk stores (the third map); kFeatureGrad: rows of `out` are aligned
  int *rest;               // kLogits, kGradient, kFewRows: how the features' gradient will be cut goes here, for `rest_pairs`; kFeatureGrad: it is here
  int rest_pairs, rest_wide;
  int *status;
  // kLogits, kGradient
  const int *label;        // packed rows
  float2 *label_sums;      // sum of products of the label's class, and the sum of powers of its 128 (or 32) classes without its own
  float2 *stat;            // [row][stats]: largest sum of products (a logit without its scale) and sum of powers, per 128 classes
  int stats;
  float c;                 // scale log2(e): differences of sums of products become exponents of 2
  __half *power;           // [row][ld_power], null: not wanted
  long long ld_power;
  // kGradient
  const float *weight;     // packed rows
  float factor;            // of G
  RowOut rows_out;
  // kFeatureGrad (source: also kGradient)
  const int *source;       // packed row -> row, -1: none
  __nv_bfloat16 *out;      // also kWeightGrad
  long long ld_out, out_batch;
  float *partial;          // kFeatureGrad: tiles of 256 x 256, [rest][share]; kWeightGrad: running sums over pieces of rows, or null
  int n_pad;               // row stride of these
  int first, last;         // kWeightGrad: of the pieces that make up a sum; kFewRows without m_dev: first piece of the call
  DropoutKey drop;
};

// How the units of a problem are dealt to pairs: `whole` ones, then `rest` single tiles (the two of a unit one after the other; one
// that does not exist is passed over), each cut along K into `shares`.
// The features' gradient has long contractions and few tiles: what would not fill a round is cut, ends up side by side as fp32 tiles,
// and is added by vocab_join_kernel (8192 x 4096 features of 32000 classes, a quarter left out: 192 units on 74 pairs).
struct Rest {
  int whole, rest, shares;
};
constexpr int kMostShares = 32, kShareChunks = 16, kMostRounds = 8;
__host__ __device__ inline Rest rest_of(int units, int pairs) {
  const int left = units % pairs;
  Rest r = {units, 0, 1};
  if (2 * left <= pairs) {
    r.whole = units - left;
    r.rest = 2 * left;
  }
  return r;
}
__host__ __device__ inline Rest cut_rest_of(int units, int pairs, int chunks, bool wide) {
  const int rest = units % pairs * (wide ? 2 : 1);
  int best = 1;
  long long best_cost = -1;
  for (int s = 1; s <= kMostShares; ++s) {
    if (s > 1 && (s * kShareChunks > chunks || rest * s > kMostRounds * pairs)) break;
    const long long rounds = (rest * s + pairs - 1) / pairs;
    // in fifths of a chunk's time: every share fills the stages anew, joining costs a launch and the tiles' traffic
    const long long cost = rounds * ((chunks + s - 1) / s + 6) * 5 + (s > 1 ? 75 + rest * s : 0);
    if (best_cost < 0 || cost < best_cost) {
      best_cost = cost;
      best = s;
    }
  }
  if (best > 1) return {units - units % pairs, rest, best};
  return wide ? rest_of(units, pairs) : Rest{units, 0, 1};
}

struct Unit {
  int batch, share, rest, m0, n0, k0, chunks, tiles;  // rest: number among the tiles that are cut, -1: whole; tiles: 0, 1 or 2
};

__device__ __forceinline__ void unit_place(int group, int m_units, int n_units, int ms, int ns, int r, int *m0, int *n0) {
  int first = 0, height = m_units;
  if (m_units > group) {
    const int per = group * n_units, g = r / per;
    r -= g * per;
    first = g * group;
    height = min(group, m_units - first);
  }
  const int n = r / height;
  *m0 = (first + r - n * height) * ms;
  *n0 = n * ns;
}

// (Divisions are 32 bits wide and as few as can be: the loading thread goes through this for every unit.)
template <int EPI, bool Wide>
__device__ __forceinline__ Unit unit_of(const GemmArgs &p, int rows, int columns, int ms, int bn, int m_units, int n_units, const Rest &rest,
                                        int t) {
  constexpr bool above = EPI == kWeightGrad;  // the two tiles of a unit differ in M
  const int ns = Wide && !above ? 2 * bn : bn;
  Unit q;
  q.share = 0;
  q.rest = -1;
  q.batch = 0;
  q.k0 = 0;
  int second = 0;
  const bool single = t >= rest.whole;
  if (single) {
    int u = t - rest.whole;
    if (EPI == kFeatureGrad) {
      q.share = u / rest.rest;
      u -= q.share * rest.rest;
    }
    q.rest = u;
    second = Wide ? u & 1 : 0;
    t = rest.whole + (Wide ? u >> 1 : u);
  }
  if (EPI == kWeightGrad && p.batch > 1) {
    const int per = m_units * n_units;
    q.batch = t / per;
    t -= q.batch * per;
  }
  unit_place(p.group, m_units, n_units, ms, ns, t, &q.m0, &q.n0);
  if (second) {
    if (above) q.m0 += 256;
    else q.n0 += bn;
  }
  const int left = above ? rows - q.m0 : columns - q.n0;  // (of the side along which the tiles lie)
  q.tiles = left <= 0 ? 0 : !Wide || single || left <= (above ? 256 : bn) ? 1 : 2;
  int k1 = p.k;
  if (EPI == kWeightGrad) {
    q.k0 = p.k_begin[q.batch];
    k1 = p.k_begin[q.batch + 1];
  }
  q.chunks = (k1 - q.k0 + 63) >> 6;
  if (EPI == kFeatureGrad && single && rest.shares > 1) {
    const int a = q.chunks * q.share / rest.shares, b = q.chunks * (q.share + 1) / rest.shares;
    q.k0 = a * 64;
    q.chunks = b - a;
  } else {
    q.rest = -1;
  }
  return q;
}

// 16 bytes of a row's 128 in a warp's staging tile; rows are permuted so that neither writes (a row per lane) nor reads (a
// row per 8 lanes) meet in a bank.
__device__ __forceinline__ uint4 *staged(unsigned char *tile, int row, int piece) {
  return reinterpret_cast<uint4 *>(tile + row * 128 + ((piece ^ (row & 7)) << 4));
}

// A warp's tile on its way out by bulk copies: the last one's copy has read it before it is written again.
struct Outgoing {
  unsigned char *tile;
  __device__ __forceinline__ unsigned char *claim(int lane) {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
    return tile;
  }
  __device__ __forceinline__ void send(const CUtensorMap *map, int c0, int c1, int c2, int lane) {
    fence_async_smem();
    __syncwarp();
    if (lane == 0) {
      tma_store_3d(map, c0, c1, c2, smem_u32(tile));
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
  }
};

// Up to 8 16-bit elements at p; whole vectors where p allows.
__device__ __forceinline__ void store8(void *p, const uint4 &v, int n) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  if (n >= 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) store_whole(p, w);
  else store_some(static_cast<__nv_bfloat16 *>(p), 0, n, w);
}

// The first `n` of a staged row's 64 16-bit elements to p, which is a multiple of 2 bytes: a warp, a word per lane, so that a row is one
// store.
__device__ __forceinline__ void store_row(__nv_bfloat16 *p, int n, const unsigned char *tile, int row, int lane) {
  const uint32_t w = *reinterpret_cast<const uint32_t *>(tile + row * 128 + (((lane >> 2) ^ (row & 7)) << 4) + (lane & 3) * 4);
  const int at = 2 * lane;
  if ((reinterpret_cast<uintptr_t>(p) & 2) == 0) {
    if (at + 1 < n) *reinterpret_cast<uint32_t *>(p + at) = w;
    else if (at < n) *reinterpret_cast<uint16_t *>(p + at) = (uint16_t)w;
  } else {  // a word of memory is the end of the lane before's and the beginning of this one's
    const uint32_t before = __shfl_up_sync(0xffffffffu, w, 1), both = before >> 16 | w << 16;
    if (lane > 0 && at < n) *reinterpret_cast<uint32_t *>(p + at - 1) = both;
    else if (lane > 0 && at - 1 < n) *reinterpret_cast<uint16_t *>(p + at - 1) = (uint16_t)both;
    else if (lane == 0 && n > 0) *reinterpret_cast<uint16_t *>(p) = (uint16_t)w;
    if (lane == 31 && n > 63) *reinterpret_cast<uint16_t *>(p + 63) = (uint16_t)(w >> 16);
  }
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

// What an epilogue warp works on: W columns from n0 of one quadrant's 32 rows.
struct Part {
  uint32_t taddr, release;  // accumulator, and the barrier that gives it back
  int row, lane, half;
  Outgoing *out;
};
// (The whole warp, one arrival, which orders nothing but the tensor memory's reads, as the fence before it does: with release semantics it
// waited for everything else that the warp had under way, some 2400 cycles in every run.)
__device__ __forceinline__ void give_back(const Part &w) {
  tc_fence_before();
  __syncwarp();
  if (w.lane == 0) mbar_arrive_cluster_relaxed(w.release);
}

// The two accumulators, which hold the runs of a tile's contraction in turn.
struct Accumulators {
  uint32_t taddr, full, release;  // of the first one
  uint32_t turn;
  // Waits for the next one (the whole warp).
  __device__ __forceinline__ bool next(Part *w) {
    const uint32_t a = turn & 1u, phase = turn >> 1 & 1u;
    ++turn;
    if (!__all_sync(0xffffffffu, mbar_wait(full + 8 * a, phase))) return false;
    tc_fence_after();
    w->taddr = taddr + 256u * a;
    w->release = release + 8u * a;
    return true;
  }
};

// The sums of a tile's W columns over all of its runs; false: a wait gave up.
template <int W>
__device__ __forceinline__ bool add_runs(Accumulators *in, Part w, int chunks, uint32_t (&r)[W]) {
  if (!in->next(&w)) return false;
  tmem_ld_chunks<W / 32>(w.taddr, W / 32, r);
  give_back(w);  // everything is in registers: the accumulator may be written again
#pragma unroll 1
  for (int k = kSumChunks; k < chunks; k += kSumChunks) {
    if (!in->next(&w)) return false;
#pragma unroll
    for (int h = 0; h < W / 16; ++h) {  // (32 at a time would spill)
      uint32_t x[16];
      tmem_ld16_nowait(w.taddr + h * 16, x);
      tmem_ld_wait(x);
      if (h == W / 16 - 1) give_back(w);
#pragma unroll
      for (int i = 0; i < 16; ++i) r[h * 16 + i] = __float_as_uint(__uint_as_float(r[h * 16 + i]) + __uint_as_float(x[i]));
    }
  }
  return true;
}
// The same of 32 columns out of every 64, `groups` of them in all, from the warp's half on.
__device__ __forceinline__ bool add_few_runs(Accumulators *in, Part w, int chunks, int groups, uint32_t (&r)[2][32]) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 32; ++i) r[h][i] = 0u;
#pragma unroll 1
  for (int k = 0; k < chunks; k += kSumChunks) {
    if (!in->next(&w)) return false;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (w.half + 2 * h >= groups) break;
      uint32_t x[32];
      tmem_ld_chunks<1>(w.taddr + (w.half + 2 * h) * 32, 1, x);
#pragma unroll
      for (int i = 0; i < 32; ++i) r[h][i] = __float_as_uint(__uint_as_float(r[h][i]) + __uint_as_float(x[i]));
    }
    give_back(w);
  }
  return true;
}

// A row's W sums of products (columns from `valid` on are behind the last class), and its label if it is one of them.
template <int W>
struct Row {
  float top;   // the largest; no less than kLowest
  bool here;   // the label
  float z;     // its sum of products, which is taken out: its power is not needed where it lies, as G is put there from log p
  __device__ __forceinline__ Row(uint32_t (&r)[W], int valid, int lab) : top(kNegInf), here(lab >= 0 && lab < min(W, valid)), z(0.f) {
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
    top = fmaxf(top, kLowest);
    if (here) {
#pragma unroll
      for (int i = 0; i < W; ++i) {
        z = i == lab ? __uint_as_float(r[i]) : z;
        r[i] = i == lab ? __float_as_uint(kNegInf) : r[i];
      }
    }
  }
  // Powers of N of the columns in place of their sums of products, and their sum.  (The difference first: the largest power is 1 whatever
  // the logits' size.  As a product less a rounded product it was 2 to the rounding error of top c, which fp16 did not hold from 2^26 on.)
  template <int N, int From>
  __device__ __forceinline__ float powers(uint32_t (&r)[W], float c) const {
    float s[4] = {};
#pragma unroll
    for (int i = From; i < From + N; ++i) {
      const float e = power2((__uint_as_float(r[i]) - top) * c);
      s[i & 3] += e;
      r[i] = __float_as_uint(e);
    }
    return (s[0] + s[1]) + (s[2] + s[3]);
  }
  // Maximum and sum of powers, the label's own among them.  (A NaN among the logits is not the largest, but it is in the sum.)
  __device__ __forceinline__ float2 stat(float others, int valid, float c) const {
    return make_float2(valid > 0 ? top : kNegInf, here ? others + power2((z - top) * c) : others);
  }
};

// log p of a label with sum of products z, from the largest one of its row and the sum of all other classes' powers relative to that; *total:
// the sum with its own.  Differences first, and by the scale itself (times log2(e) one may leave fp32); above a half, p by how far it is from 1, of
// which a sum near 1 would keep nothing below 2^-24.  So log p is below 0, with its digits, at any p.
__device__ __forceinline__ float log_p(float z, float top, float others, float c, float factor, float *total) {
  const float own = power2((z - top) * c);
  *total = others + own;
  return others <= own ? -log1pf(others / own) : (z - top) * factor - log2f(*total) * kLn2;
}

// 64 columns' powers on their way.
template <int W, int From>
__device__ __forceinline__ void send_powers(const GemmArgs &p, const CUtensorMap *map, const Part &w, const uint32_t (&r)[W], int n0) {
  constexpr float k = (float)(1 << kPowerBits);
  unsigned char *tile = w.out->claim(w.lane);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    uint32_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      x[i] = pack_half(__uint_as_float(r[From + j * 8 + 2 * i]) * k, __uint_as_float(r[From + j * 8 + 2 * i + 1]) * k);
    *staged(tile, w.lane, j) = make_uint4(x[0], x[1], x[2], x[3]);
  }
  if (n0 + From < p.ld_power) w.out->send(map, n0 + From, w.row - w.lane, 0, w.lane);
}

template <int W>
__device__ __forceinline__ void logits_epilogue(const GemmArgs &p, const CUtensorMap *map, const Part &w, uint32_t (&r)[W], int group, int n0) {
  const Row<W> row(r, p.n - n0, p.label[w.row] - n0);
  // (The second half's powers while the first half's store is read from shared memory: contraction of 2048 x 1024 x 65536 230 -> 208 us.  The
  // sums are the same without powers to store, to the bit.)
  float others = row.template powers<64, 0>(r, p.c);
  if (p.power) send_powers<W, 0>(p, map, w, r, n0);
  others += row.template powers<W - 64, 64>(r, p.c);
  if (p.power) send_powers<W, 64>(p, map, w, r, n0);
  if (row.here) p.label_sums[w.row] = make_float2(row.z, others);
  p.stat[(long long)w.row * p.stats + group] = row.stat(others, p.n - n0, p.c);
}

// For each of 32 columns, `op` over the 32 lanes: lane l ends up with column l's.  Every step halves what a lane holds.
template <typename Op>
__device__ __forceinline__ float across_lanes(const uint32_t (&r)[32], int lane, Op op) {
  float v[32];
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const bool upper = lane & o;
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const float mine = upper ? v[i + o] : v[i], theirs = upper ? v[i] : v[i + o];
      v[i] = op(mine, __shfl_xor_sync(0xffffffffu, theirs, o));
    }
  }
  return v[0];
}

// Statistics (and powers) of rows n0 .. n0 + bn - 1 (columns here) over a warp's 32 classes, one per lane.
__device__ __forceinline__ void few_rows_epilogue(const GemmArgs &p, const Part &w, const uint32_t (&sums)[2][32], bool inside, int group, int n0,
                                                  int rows, int groups) {
  const bool real = inside && w.row < p.m;
  const int classes = __popc(__ballot_sync(0xffffffffu, real));  // the warp's, in its first lanes
  // (A loop: the instructions are fetched for a tile or two of a warp, so twice as many would take longer.)
#pragma unroll 1
  for (int g = w.half; g < groups; g += 2) {
    uint32_t r[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) r[i] = g < 2 ? sums[0][i] : sums[1][i];
    const int row = n0 + g * 32 + w.lane;
    const int lab = (row < rows ? p.label[row] : -1) - (w.row - w.lane);  // lane of the label's class
    const bool has_label = lab >= 0 && lab < classes;
    if (!real) {
#pragma unroll
      for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(kNegInf);
    }
    // (of a group without classes: nothing is read later, or zeros)
    const float top = classes > 0 ? fmaxf(across_lanes(r, w.lane, [](float a, float b) { return fmaxf(a, b); }), kLowest) : 0.f;
    float z = 0.f;  // of this lane's row
    for (unsigned has = __ballot_sync(0xffffffffu, has_label); has; has &= has - 1) {
      const int column = __ffs(has) - 1, at = __shfl_sync(0xffffffffu, lab, column);
      float here = 0.f;
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        here = i == column ? __uint_as_float(r[i]) : here;
        if (i == column && w.lane == at) r[i] = __float_as_uint(kNegInf);
      }
      here = __shfl_sync(0xffffffffu, here, at);
      if (w.lane == column) z = here;
    }
#pragma unroll
    for (int i = 0; i < 32; ++i)
      r[i] = __float_as_uint(power2((__uint_as_float(r[i]) - __shfl_sync(0xffffffffu, top, i)) * p.c));
    if (p.power && inside && w.row < p.ld_power) {  // (a row's classes lie side by side in the lanes)
      __half *dst = p.power + (long long)(n0 + g * 32) * p.ld_power + w.row;
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (n0 + g * 32 + i < rows) dst[i * p.ld_power] = __float2half_rn(__uint_as_float(r[i]) * (float)(1 << kPowerBits));
    }
    float sum = across_lanes(r, w.lane, [](float a, float b) { return a + b; });
    if (has_label) {
      p.label_sums[row] = make_float2(z, sum);
      sum += power2((z - top) * p.c);
    }
    if (row < rows) p.stat[(long long)row * p.stats + group] = make_float2(classes > 0 ? top : kNegInf, sum);
  }
}

// Losses and G of rows whose classes are this tile's: what the two warps of a row have found is exchanged.  They go on, or give up, together:
// one that has no sums sends a maximum that is not a number, which no set has.
template <int W>
__device__ __forceinline__ bool gradient_epilogue(const GemmArgs &p, const CUtensorMap *map, const Part &w, uint32_t (&r)[W], bool ok, int rows,
                                                  int n0, float2 *exchange) {
  const int quad = (threadIdx.x >> 5) & 3, mine = quad * 32 + w.lane;
  const bool counts = w.row < rows && p.label[w.row] >= 0;
  const int lab = counts ? p.label[w.row] - n0 : -1;
  const Row<W> row(r, p.n - n0, lab);
  const float others = row.template powers<W, 0>(r, p.c);
  const float2 s = ok ? row.stat(others, p.n - n0, p.c) : make_float2(__int_as_float(0x7fffffff), 0.f);
  exchange[w.half * 128 + mine] = s;
  asm volatile("bar.sync %0, 64;" ::"r"(1 + quad) : "memory");
  const float2 o = exchange[(w.half ^ 1) * 128 + mine];
  asm volatile("bar.sync %0, 64;" ::"r"(1 + quad) : "memory");  // (read before the next tile's are written)
  if (!ok || __any_sync(0xffffffffu, isnan(o.x))) return false;
  const float top = fmaxf(s.x, o.x);
  // (an empty half's maximum is -infinity: 2^-infinity = 0)
  const float mine_up = power2((s.x - top) * p.c), theirs = o.y * power2((o.x - top) * p.c), sum = s.y * mine_up + theirs;
  const float weight = counts ? p.weight[w.row] : 0.f, g = p.factor * weight;
  const bool here = lab >= 0 && lab < W;
  float at_label = 0.f;
  if (here) {
    float total;
    const float logp = log_p(row.z, top, others * mine_up + theirs, p.c, p.factor, &total);
    at_label = g * expm1f(logp);
    p.rows_out.put(p.source[w.row], logp, -weight * logp);
  }
  if (!p.power) return true;
  const float f = g * mine_up / sum;
#pragma unroll
  for (int h = 0; h < W / 64; ++h) {
    unsigned char *tile = w.out->claim(w.lane);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        x[i] = counts ? pack_bf16(__uint_as_float(r[h * 64 + j * 8 + 2 * i]) * f, __uint_as_float(r[h * 64 + j * 8 + 2 * i + 1]) * f) : 0u;
      *staged(tile, w.lane, j) = make_uint4(x[0], x[1], x[2], x[3]);
    }
    if (here && lab / 64 == h)
      reinterpret_cast<__nv_bfloat16 *>(staged(tile, w.lane, (lab & 63) >> 3))[lab & 7] = __float2bfloat16_rn(at_label);
    if (n0 + h * 64 < p.ld_power) w.out->send(map, n0 + h * 64, w.row - w.lane, 0, w.lane);
  }
  return true;
}

template <int W>
__device__ __forceinline__ void feature_epilogue(const GemmArgs &p, const Part &w, const Unit &q, int shares, int rows, int n0) {
  const int row0 = w.row - w.lane;
  if (row0 >= rows) {  // (the same in the whole warp)
    give_back(w);
    return;
  }
  if (q.rest >= 0) {
    float *dst = p.partial + ((long long)q.rest * shares + q.share) * 65536 + (row0 - q.m0) * 256 + (n0 - q.n0);
#pragma unroll 1
    for (int h = 0; h < W / 32; ++h) {
      uint32_t r[32];
      tmem_ld_chunks<1>(w.taddr + h * 32, 1, r);
      if (h == W / 32 - 1) give_back(w);
      unsigned char *tile = w.out->claim(w.lane);
#pragma unroll
      for (int j = 0; j < 8; ++j) *staged(tile, w.lane, j) = make_uint4(r[4 * j], r[4 * j + 1], r[4 * j + 2], r[4 * j + 3]);
      __syncwarp();
#pragma unroll
      for (int it = 0; it < 8; ++it) {
        const int rr = it * 4 + w.lane / 8;
        *reinterpret_cast<uint4 *>(dst + rr * 256 + h * 32 + (w.lane & 7) * 4) = *staged(tile, rr, w.lane & 7);
      }
      __syncwarp();
    }
    return;
  }
  const int src = w.row < rows ? p.source[w.row] : -1;
  const bool counts = w.row < rows && p.label[w.row] >= 0;
#pragma unroll 1
  for (int h = 0; h < W / 64; ++h) {
    uint32_t r[64];
    tmem_ld_chunks<2>(w.taddr + h * 64, 2, r);
    if (h == W / 64 - 1) give_back(w);
    unsigned char *tile = w.out->claim(w.lane);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        x[i] = counts ? pack_bf16(__uint_as_float(r[j * 8 + 2 * i]), __uint_as_float(r[j * 8 + 2 * i + 1])) : 0u;
      if (p.drop.threshold) {
        const Keep8 keep = dropout_keep8(p.drop, (uint64_t)src, (uint32_t)(n0 + h * 64 + j * 8) >> 3);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] &= keep.halves(i);
      }
      *staged(tile, w.lane, j) = make_uint4(x[0], x[1], x[2], x[3]);
    }
    __syncwarp();
    const int col0 = n0 + h * 64;
    if (p.store) {  // rows begin at multiples of 16 bytes
#pragma unroll
      for (int it = 0; it < 8; ++it) {
        const int rr = it * 4 + w.lane / 8, col = col0 + (w.lane & 7) * 8;
        const int to = __shfl_sync(0xffffffffu, src, rr);
        if (to >= 0 && col < p.n) store8(p.out + (long long)to * p.ld_out + col, *staged(tile, rr, w.lane & 7), p.n - col);
      }
    } else if (col0 < p.n) {
#pragma unroll 4
      for (int rr = 0; rr < 32; ++rr) {
        const int to = __shfl_sync(0xffffffffu, src, rr);
        if (to >= 0) store_row(p.out + (long long)to * p.ld_out + col0, p.n - col0, tile, rr, w.lane);
      }
    }
    __syncwarp();
  }
}

// All of a staged tile to rows `ld` apart, by the same words.  (8 warps have the instructions of this to themselves but little to hide
// their latency with: eight rows are read before the first is written.  Gradient of 3 x 10007 x 1021 from 600 rows each: 37 us where
// bulk stores can be used, 75 us with a row after the other.)
__device__ __forceinline__ void store_rows(__nv_bfloat16 *p, long long ld, const unsigned char *tile, int lane) {
  const uint32_t in_vector = (lane & 3) * 4, vector = lane >> 2;
#pragma unroll 1
  for (int r = 0; r < 32; r += 8) {
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = *reinterpret_cast<const uint32_t *>(tile + (r + j) * 128 + ((vector ^ j) << 4) + in_vector);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if ((reinterpret_cast<uintptr_t>(p) & 2) == 0) {
        *reinterpret_cast<uint32_t *>(p + 2 * lane) = w[j];
      } else {
        const uint32_t before = __shfl_up_sync(0xffffffffu, w[j], 1);
        if (lane > 0) *reinterpret_cast<uint32_t *>(p + 2 * lane - 1) = __funnelshift_r(before, w[j], 16);
        if (lane == 0) *reinterpret_cast<uint16_t *>(p) = (uint16_t)w[j];
        if (lane == 31) *reinterpret_cast<uint16_t *>(p + 63) = (uint16_t)(w[j] >> 16);
      }
      p += ld;
    }
  }
}

template <int W>
__device__ __forceinline__ void weight_epilogue(const GemmArgs &p, const CUtensorMap *map, const Part &w, const Unit &q, int n0) {
  const int row0 = w.row - w.lane;
  __nv_bfloat16 *out = p.out + (long long)q.batch * p.out_batch;
  const bool sums = p.partial != nullptr;
#pragma unroll 1
  for (int h = 0; h < W / 64; ++h) {
    uint32_t r[64];
    if (q.chunks > 0) {
      tmem_ld_chunks<2>(w.taddr + h * 64, 2, r);
      if (h == W / 64 - 1) give_back(w);
    } else {  // no row of this partition counts
#pragma unroll
      for (int i = 0; i < 64; ++i) r[i] = 0u;
    }
    const int col0 = n0 + h * 64;
    if (col0 >= p.n || row0 >= p.m) continue;  // (the same in the whole warp)
    if (sums) {  // fp32 sums over the pieces of a partition's rows
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        unsigned char *tile = w.out->claim(w.lane);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          *staged(tile, w.lane, j) = make_uint4(r[g * 32 + 4 * j], r[g * 32 + 4 * j + 1], r[g * 32 + 4 * j + 2], r[g * 32 + 4 * j + 3]);
        __syncwarp();
#pragma unroll
        for (int it = 0; it < 8; ++it) {
          const int rr = it * 4 + w.lane / 8, col = col0 + g * 32 + (w.lane & 7) * 4;
          if (row0 + rr >= p.m || col >= p.n) continue;
          float4 v = *reinterpret_cast<float4 *>(staged(tile, rr, w.lane & 7));
          float4 *acc = reinterpret_cast<float4 *>(p.partial + (long long)(row0 + rr) * p.n_pad + col);
          if (!p.first) {
            const float4 old = *acc;
            v.x += old.x; v.y += old.y; v.z += old.z; v.w += old.w;
          }
          if (!p.last) {
            *acc = v;
            continue;
          }
          __nv_bfloat16 *dst = out + (long long)(row0 + rr) * p.ld_out + col;
          const uint32_t lo = pack_bf16(v.x, v.y), hi = pack_bf16(v.z, v.w);
          if (p.n - col >= 4 && (reinterpret_cast<uintptr_t>(dst) & 7) == 0) *reinterpret_cast<uint2 *>(dst) = make_uint2(lo, hi);
          else store_some(dst, 0, min(4, p.n - col), {lo, hi, 0u, 0u});
        }
        __syncwarp();
      }
      continue;
    }
    unsigned char *tile = w.out->claim(w.lane);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = pack_bf16(__uint_as_float(r[j * 8 + 2 * i]), __uint_as_float(r[j * 8 + 2 * i + 1]));
      *staged(tile, w.lane, j) = make_uint4(x[0], x[1], x[2], x[3]);
    }
    if (p.store) {
      w.out->send(map, col0, row0, q.batch, w.lane);
      continue;
    }
    __syncwarp();
    __nv_bfloat16 *dst = out + (long long)row0 * p.ld_out + col0;
    const int here = p.m - row0;
    if (here >= 32 && p.n - col0 >= 64) {
      store_rows(dst, p.ld_out, tile, w.lane);
    } else {
#pragma unroll 1
      for (int rr = 0; rr < min(32, here); ++rr) store_row(dst + (long long)rr * p.ld_out, p.n - col0, tile, rr, w.lane);
    }
    __syncwarp();
  }
}

template <int EPI, int A_MN, int B_MN, int BN, bool Wide>
__global__ void __launch_bounds__(kThreads, 1)
vocab_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                  const __grid_constant__ CUtensorMap tmC, const GemmArgs p) {
  constexpr bool above = EPI == kWeightGrad, runs = EPI == kLogits || EPI == kGradient || EPI == kFewRows;
  static_assert(!(runs && Wide), "runs take the accumulators in turn");
  constexpr int kRing = Wide ? 4 : EPI == kGradient ? 5 : 6, kStageBytes = (Wide ? 3 : 2) * kHalfBytes;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t sbase = smem_u32(smem_raw);
  unsigned char *tiles = smem_raw + ((1024u - (sbase & 1023u)) & 1023u);
  unsigned char *staging = tiles + kRing * kStageBytes;
  unsigned char *behind = staging + 8 * kStageTile;
  const uint32_t bars = smem_u32(behind);
  const uint32_t full = bars, empty = bars + 8 * kRing, tfull = bars + 16 * kRing, tempty = tfull + 16;
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(behind + 16 * kRing + 32);
  float2 *exchange = reinterpret_cast<float2 *>(behind + 256);
  static_assert(kRing * kStageBytes + 8 * kStageTile + 256 + (EPI == kGradient ? kExchange : 0) + 1024 <= kSmem, "shared memory");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  // (up to here, and the barriers and tensor memory below, nothing of the kernel before is touched)
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (threadIdx.x == 0) {
    for (int i = 0; i < kRing; ++i) {
      mbar_init(full + 8 * i, 1);
      mbar_init(empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(tfull + 8 * i, 1);
      mbar_init(tempty + 8 * i, 2 * (kThreads / 32 - 2));
    }
    mbar_fence_init();
  }
  if (warp == 1) tmem_alloc_pair(smem_u32(tmem_slot), kTmem);
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();  // the peer's barriers exist before anything is signalled on them
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  bool failed = false;
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const int in_use = p.m_dev ? *p.m_dev : EPI == kFewRows ? p.few_rows : p.m;
  if (EPI == kFewRows && !p.m_dev && p.first && blockIdx.x == 0 && threadIdx.x == 0) *p.status = 0;  // (no kernel before this one did)
  const int rows = EPI == kFewRows ? p.m : in_use, columns = EPI == kFewRows ? in_use : p.n;
  int bn = BN;  // columns of a tile
  if (EPI == kFewRows) bn = max(32, (columns + 31) / 32 * 32);
  const int each = EPI == kFewRows ? p.classes_each : 128;  // rows of A that this CTA loads
  const int ms = EPI == kFewRows ? 2 * each : Wide && above ? 512 : 256, ns = Wide && !above ? 2 * bn : bn;
  const int m_units = (rows + ms - 1) / ms, n_units = EPI == kFewRows && columns == 0 ? 0 : (columns + ns - 1) / ns;
  Rest rest = {m_units * n_units * p.batch, 0, 1};
  if (EPI == kFeatureGrad) rest = *reinterpret_cast<const Rest *>(p.rest);
  else if (Wide) rest = rest_of(rest.whole, pairs);
  const int total = rest.whole + rest.rest * rest.shares;
  constexpr int kHalf = BN / 2;             // columns of a tile's B that this CTA loads
  const int own = EPI == kFewRows ? bn / 2 : kHalf;
  const uint32_t b_bytes = (uint32_t)own * 128u, third_bytes = above ? (uint32_t)kHalfBytes : b_bytes;

  if (warp == 0) {
    if (lane == 0) {
      int st = 0;
      uint32_t ph = 0;
      for (int t = pair; t < total && !failed; t += pairs) {
        const Unit q = unit_of<EPI, Wide>(p, rows, columns, ms, bn, m_units, n_units, rest, t);
        if (q.tiles == 0) continue;
        const int m0 = q.m0 + (int)rank * each, n0 = q.n0 + (int)rank * own;
        const bool both = Wide && q.tiles == 2;
        const uint32_t bytes = 2 * ((uint32_t)each * 128u + b_bytes + (both ? third_bytes : 0u));  // both CTAs signal the leader's barrier
        for (int kc = 0; kc < q.chunks; ++kc) {
          if (!mbar_wait(empty + 8 * st, ph ^ 1u)) { failed = true; break; }
          if (rank == 0) mbar_expect_tx(full + 8 * st, bytes);
          const uint32_t a = smem_u32(tiles + st * kStageBytes), b = a + kHalfBytes;
          const uint32_t bar = map_to_rank(full + 8 * st, 0);
          const int k = q.k0 + kc * 64;
          auto load_a = [&](uint32_t dst, int m) {
            if (A_MN) {
              tma_load_2d_pair(dst, &tmA, m, k, bar);
              tma_load_2d_pair(dst + 8192, &tmA, m + 64, k, bar);
            } else {
              tma_load_2d_pair(dst, &tmA, k, m, bar);
            }
          };
          auto load_b = [&](uint32_t dst, int n) {
            if (EPI == kFewRows) {  // (as many boxes of 16 rows as there are)
              for (int j = 0; j < own / 16; ++j) tma_load_2d_pair(dst + j * 2048, &tmB, k, n + j * 16, bar);
            } else if (B_MN) {
#pragma unroll
              for (int j = 0; j < kHalf / 64; ++j) tma_load_2d_pair(dst + j * 8192, &tmB, n + j * 64, k, bar);
            } else {
              tma_load_2d_pair(dst, &tmB, k, n, bar);
            }
          };
          load_a(a, m0);
          load_b(b, n0);
          if (both) {
            if (above) load_a(b + kHalfBytes, m0 + 256);
            else load_b(b + kHalfBytes, n0 + bn);
          }
          if (++st == kRing) { st = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    if ((EPI == kLogits || EPI == kGradient || EPI == kFewRows) && blockIdx.x == 1 && lane == 0 && p.rest)  // (a warp that has nothing else to do)
      *reinterpret_cast<Rest *>(p.rest) = cut_rest_of((in_use + 255) / 256 * ((p.k + (p.rest_wide ? 511 : 255)) / (p.rest_wide ? 512 : 256)),
                                                  p.rest_pairs, (p.n + 63) / 64, p.rest_wide);
    if (rank == 0) {  // all 32 lanes walk the loop (uniform operands); one elected lane issues
      const uint32_t idesc = instr_desc_bf16(256, EPI == kFewRows ? bn : BN, A_MN, B_MN);
      int st = 0, singles = 0;
      uint32_t ph = 0, eph[2] = {0u, 0u};
      // one chunk of one tile; K-major: rows 128 bytes apart, 16 elements of K are 32 bytes on; M/N-major: boxes of 64 elements
      // 8192 bytes apart, 16 elements of K are 16 rows of 128 bytes on
      auto contract = [&](uint32_t acc, int stage, bool other, bool go_on) {
        const uint32_t at = smem_u32(tiles + stage * kStageBytes);
        const uint64_t ad = smem_desc_sw128(at + (other && above ? 2 * kHalfBytes : 0), A_MN ? 8192 : 16, 1024);
        const uint64_t bd = smem_desc_sw128(at + (other && !above ? 2 * kHalfBytes : kHalfBytes), B_MN ? 8192 : 16, 1024);
#pragma unroll
        for (int k4 = 0; k4 < 4; ++k4)
          mma_bf16_pair(acc, ad + (uint64_t)(k4 * (A_MN ? 128 : 2)), bd + (uint64_t)(k4 * (B_MN ? 128 : 2)), idesc,
                        go_on || k4 != 0);
      };
      for (int t = pair; t < total && !failed; t += pairs) {
        const Unit q = unit_of<EPI, Wide>(p, rows, columns, ms, bn, m_units, n_units, rest, t);
        if (q.chunks == 0 || q.tiles == 0) continue;
        const bool both = Wide && q.tiles == 2;
        int kc = 0;
        do {  // (a run; where there are none, the whole contraction)
          const int begin = kc, end = runs ? min(q.chunks, begin + kSumChunks) : q.chunks;
          const int a0 = both ? 0 : (singles++ & 1);
          const uint32_t acc0 = tmem + (uint32_t)a0 * 256u, acc1 = tmem + 256u;
          if (!mbar_wait_warp(tempty + 8 * a0, (a0 ? eph[1] : eph[0]) ^ 1u)) { failed = true; break; }
          tc_fence_after();
          if (both) {
            // as many chunks as the ring holds for the first accumulator, while the second one may still be read out
            const int lead = min(q.chunks, kRing);
            const uint32_t ph0 = ph;
            const int st0 = st;
            for (int i = 0; i < lead; ++i) {
              if (!mbar_wait_warp(full + 8 * st, ph)) { failed = true; break; }
              tc_fence_after();
              contract(acc0, st, false, i != 0);
              if (++st == kRing) { st = 0; ph ^= 1u; }
            }
            if (failed || !mbar_wait_warp(tempty + 8, eph[1] ^ 1u)) { failed = true; break; }
            tc_fence_after();
            st = st0;
            ph = ph0;
            for (int i = 0; i < lead; ++i) {
              contract(acc1, st, true, i != 0);
              mma_commit_pair(empty + 8 * st, 3);
              if (++st == kRing) { st = 0; ph ^= 1u; }
            }
            kc = lead;
          }
          for (; kc < end; ++kc) {
            if (!mbar_wait_warp(full + 8 * st, ph)) { failed = true; break; }
            tc_fence_after();
            contract(acc0, st, false, kc != begin);
            if (both) contract(acc1, st, true, true);
            mma_commit_pair(empty + 8 * st, 3);
            if (++st == kRing) { st = 0; ph ^= 1u; }
          }
          if (failed) break;
          mma_commit_pair(tfull + 8 * a0, 3);
          if (both) mma_commit_pair(tfull + 8, 3);
          if (both || a0 == 0) eph[0] ^= 1u;
          if (both || a0 == 1) eph[1] ^= 1u;
        } while (runs && kc < q.chunks);
      }
    }
  } else {
    const int quad = warp & 3, half = (warp - 2) >> 2;
    Outgoing out = {staging + (warp - 2) * kStageTile};
    int singles = 0;
    uint32_t fph[2] = {0u, 0u};
    const uint32_t mine = tmem + ((uint32_t)(quad * 32) << 16);
    Accumulators in = {mine + (uint32_t)(EPI == kFewRows ? 0 : half * kHalf), tfull, map_to_rank(tempty, 0), 0u};
    for (int t = pair; t < total && !failed; t += pairs) {
      const Unit q = unit_of<EPI, Wide>(p, rows, columns, ms, bn, m_units, n_units, rest, t);
      if constexpr (runs) {
        if (q.tiles == 0) continue;
        const int n0 = q.n0 + (EPI == kFewRows ? 0 : half * kHalf);
        Part w = {0, 0, q.m0 + (int)rank * each + quad * 32 + lane, lane, half, &out};
        bool ok;
        if constexpr (EPI == kFewRows) {
          uint32_t r[2][32];
          const int groups = bn / 32;
          ok = add_few_runs(&in, w, q.chunks, groups, r);
          if (ok) few_rows_epilogue(p, w, r, quad * 32 + lane < each, (q.m0 / ms * 2 + (int)rank) * 4 + quad, n0, columns, groups);
        } else {
          uint32_t r[kHalf];
          ok = add_runs<kHalf>(&in, w, q.chunks, r);
          if constexpr (EPI == kGradient) ok = gradient_epilogue<kHalf>(p, &tmC, w, r, ok, rows, n0, exchange);
          else if (ok) logits_epilogue<kHalf>(p, &tmC, w, r, n0 / kHalf, n0);
        }
        failed = !ok;
        continue;
      }
      const int a0 = q.chunks > 0 && q.tiles == 1 ? (singles++ & 1) : 0;
#pragma unroll 1
      for (int i = 0; i < q.tiles; ++i) {
        const int acc = a0 + i, m0 = q.m0 + (above ? i * 256 : 0), n0 = q.n0 + (above ? 0 : i * bn) + half * kHalf;
        const Part w = {mine + (uint32_t)(acc * 256 + half * kHalf), map_to_rank(tempty + 8 * acc, 0), m0 + (int)rank * each + quad * 32 + lane, lane,
                        half, &out};
        if (q.chunks > 0) {
          if (!__all_sync(0xffffffffu, mbar_wait(tfull + 8 * acc, acc ? fph[1] : fph[0]))) { failed = true; break; }
          tc_fence_after();
          if (acc) fph[1] ^= 1u; else fph[0] ^= 1u;
        }
        if (EPI == kFeatureGrad) feature_epilogue<kHalf>(p, w, q, rest.shares, rows, n0);
        else weight_epilogue<kHalf>(p, &tmC, w, q, n0);
      }
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");  // what is on its way out is there
  }
  // (Loads stop when the ring is full and nothing else starts any, so by the time a wait has given up the copies on their way have had
  // its whole limit to arrive; the barrier below keeps both CTAs' memory until every warp is through.)
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
  int n_classes;
  const int *labels;
  const float *weight;  // null: 1
  int *header;          // [0] status, [1] packed rows, [2 .. 4] a Rest
  int *counts, *begin;  // rows that count per segment; first packed row of each partition (parts + 1)
  int *position;        // row -> packed row, -1: left out
  int *source, *label;  // packed row -> row, its label (-1: left out, or no row)
  float *row_weight;
  __nv_bfloat16 *packed;
  RowOut out;
  __nv_bfloat16 *dx;
  long long ld_dx;
  DropoutKey drop;
  int first_piece;
};

__device__ __forceinline__ bool counts_row(const RowArgs &a, int row) {
  const int y = a.labels[row];
  const float w = a.weight ? a.weight[row] : 1.f;  // (asked for beside the label)
  return (y >= 0) & (y < a.n_classes) & (w != 0.f);
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
      a.out.put(row, 0.f, 0.f);
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
    if (i < a.rows && !live) a.out.put(i, 0.f, 0.f);
  }
  for (int i = (int)(blockIdx.x * kRowThreads + threadIdx.x); i <= a.parts; i += (int)(gridDim.x * kRowThreads))
    a.begin[i] = (int)min((long long)i * a.each, (long long)end);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.header[1] = end;
    if (a.first_piece) a.header[0] = 0;
  }
}

// Row `src` of `n` elements (of a matrix that ends at `last`) to whole vectors, zero behind its end; a warp, several vectors
// of a lane in flight.
template <typename Change>
__device__ __forceinline__ void copy_row(const __nv_bfloat16 *src, int n, const void *first, const void *last, uint4 *dst, int vectors,
                                         int lane, Change change) {
  constexpr int kFlight = 8;
  for (int b0 = lane; b0 < vectors; b0 += 32 * kFlight) {
    uint32_t w[kFlight][4];
#pragma unroll
    for (int i = 0; i < kFlight; ++i) {
      const int b = b0 + 32 * i;
      if (b < vectors && b * 8 < n) {
        load_anywhere(src + b * 8, n - b * 8, first, last, w[i]);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) w[i][j] = 0u;
      }
    }
#pragma unroll
    for (int i = 0; i < kFlight; ++i) {
      const int b = b0 + 32 * i;
      if (b < vectors) {
        change(b, w[i]);
        dst[b] = make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]);
      }
    }
  }
}

// One row by a warp: to its place among the packed rows (dropped features are zero there; the others are stretched in
// the scale of the logits and of G instead, which rounds nothing), or, left out, its gradient to zero.
__device__ __forceinline__ void move_row(const RowArgs &a, int row, int to, int lane) {
  if (to >= 0) {
    copy_row(a.x + (long long)row * a.ldx, a.d, a.x, a.x + (long long)(a.rows - 1) * a.ldx + a.d,
             reinterpret_cast<uint4 *>(a.packed + (long long)to * a.d_pad), a.d_pad / 8, lane, [&](int b, uint32_t (&w)[4]) {
               if (a.drop.threshold) {
                 const Keep8 keep = dropout_keep8(a.drop, (uint64_t)row, (uint32_t)b);
#pragma unroll
                 for (int i = 0; i < 4; ++i) w[i] &= keep.halves(i);
               }
             });
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
  const __nv_bfloat16 *last = src + (long long)(rows - 1) * ld + columns;
  for (int row = (int)(blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5)); row < rows; row += (int)gridDim.x * (kRowThreads / 32))
    copy_row(src + (long long)row * ld, columns, src, last, reinterpret_cast<uint4 *>(dst + (long long)row * ld_dst), ld_dst / 8, lane,
             [](int, uint32_t (&)[4]) {});
}

// ---- losses, and powers to G ------------------------------------------------------------------------
struct LossArgs {
  const int *header, *source, *label;  // header, source null: rows where they are, `rows` of them, with the caller's labels and weights
  const float *weight;
  const float2 *label_sums;
  int rows, n_classes;
  const float2 *stat;
  int stats;  // one per 128 classes, or four per few_each
  int few_each;        // kFewRows' classes of a CTA's tile, else 0
  uint32_t few_inverse;  // 2^32 / few_each, rounded up
  RowOut out;
  __half *power;
  long long ld_power;
  float factor;  // scale (and what dropout stretches features by)
  float c;       // factor log2(e)
};

__device__ __forceinline__ float2 join(float2 a, float2 b, float c) {
  const float m = fmaxf(a.x, b.x);
  // (an empty set's maximum is -infinity; two of them must not be subtracted)
  return make_float2(m, (a.x == kNegInf ? a.y : a.y * power2((a.x - m) * c)) + (b.x == kNegInf ? b.y : b.y * power2((b.x - m) * c)));
}

// T threads per packed row (and share of its classes, where there are few rows; 32 up to 2048 classes, else 128: with 256 8000 rows of
// 4000 classes take 40 instead of 26 us, rows of 10000 and more the same): the row's statistics joined, its loss, and its
// powers e turned into G = factor w (e 2^(m - lse) - onehot), each group of classes with its own m (by its distance from the largest: as
// a difference of two scaled maxima it had the rounding of both).
template <int T>
// (32 lanes: the row's arithmetic, and its latency, bound it; more warps help although registers spill: 204800 x 256 123 -> 99 us)
__global__ void __launch_bounds__(T == 32 ? 256 : T, T == 32 ? 8 : 6 * 256 / T) vocab_loss_kernel(const LossArgs a) {
  pdl_sync();
  __shared__ float2 part[T / 32];
  const int row = (int)(T == 32 ? blockIdx.x * 8 + threadIdx.x / 32 : blockIdx.x), t = threadIdx.x % T;
  if (row >= (a.header ? a.header[1] : a.rows)) return;  // (the whole block, or whole warps)
  const int label = a.label[row], src = a.source ? a.source[row] : row;
  const float w = a.weight ? a.weight[row] : 1.f;
  uint4 *power = reinterpret_cast<uint4 *>(a.power + (long long)row * a.ld_power);
  const int all = (int)(a.ld_power / 8);
  const int first = (int)((long long)all * blockIdx.y / gridDim.y), vectors = (int)((long long)all * (blockIdx.y + 1) / gridDim.y);
  if (label < 0 || label >= a.n_classes || w == 0.f) {  // padding, or left out
    if (!a.header && t == 0) a.out.put(row, 0.f, 0.f);
    if (a.power)
      for (int v = first + t; v < vectors; v += T) power[v] = make_uint4(0u, 0u, 0u, 0u);
    return;
  }
  const float2 *stat = a.stat + (long long)row * a.stats;
  const float2 own = a.label_sums[row];
  int own_group = label / 128;
  if (a.few_each) {
    const int tile = (int)__umulhi((uint32_t)label, a.few_inverse);
    own_group = tile * 4 + (label - tile * a.few_each) / 32;
  }
  float2 s = make_float2(kNegInf, 0.f);
  for (int i0 = t; i0 < a.stats; i0 += 8 * T) {  // (eight at a time: a read from L2 takes longer than all of their arithmetic)
    float2 q[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      q[j] = i0 + j * T < a.stats ? stat[i0 + j * T] : make_float2(kNegInf, 0.f);
      if (i0 + j * T == own_group) q[j].y = own.y;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) s = join(s, q[j], a.c);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    s = join(s, make_float2(__shfl_xor_sync(0xffffffffu, s.x, o), __shfl_xor_sync(0xffffffffu, s.y, o)), a.c);
  if (T > 32) {
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
    __syncthreads();
    s = part[0];
#pragma unroll
    for (int i = 1; i < T / 32; ++i) s = join(s, part[i], a.c);
  }
  float total;
  const float logp = log_p(own.x, s.x, s.y, a.c, a.factor, &total), sum = log2f(total);
  if (t == 0 && blockIdx.y == 0) a.out.put(src, logp, -w * logp);
  if (!a.power) return;
  const float g = a.factor * w, at_label = g * expm1f(logp);
  constexpr int kFlight = T == 32 ? 1 : 2;
  for (int v0 = first + t; v0 < vectors; v0 += T * kFlight) {
    uint32_t q[kFlight][4];
    float f[kFlight];
    bool behind[kFlight];  // of the last tile: nothing was written there
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
      const int v = v0 + j * T;
      int group = v / 16;
      if (a.few_each) {
        const int tile = (int)__umulhi((uint32_t)v * 8u, a.few_inverse);
        group = tile * 4 + (v * 8 - tile * a.few_each) / 32;
      }
      if (v < vectors) load_whole(power + v, q[j]);
      f[j] = v < vectors && group < a.stats ? g * power2((stat[group].x - s.x) * a.c - sum - (float)kPowerBits) : 0.f;
      behind[j] = group >= a.stats;
    }
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
      const int v = v0 + j * T;
      if (v >= vectors) break;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 e = __half22float2(*reinterpret_cast<const __half2 *>(&q[j][i]));
        q[j][i] = behind[j] ? 0u : pack_bf16(e.x * f[j], e.y * f[j]);
      }
      store_whole(power + v, q[j]);
    }
  }
  const int mine = label / 8 - first;  // the thread that wrote the label's vector puts its element right
  if (mine >= 0 && label / 8 < vectors && mine % T == t)
    reinterpret_cast<__nv_bfloat16 *>(power)[label] = __float2bfloat16_rn(at_label);
}

// The tiles of dX that were cut along K: their shares' sum, dropped features zero; a warp per row of 256 columns.
struct JoinArgs {
  const int *header, *source, *label;
  const float *partial;
  int n, group, wide;
  __nv_bfloat16 *out;
  long long ld_out;
  DropoutKey drop;
};
__global__ void __launch_bounds__(256) vocab_join_kernel(const JoinArgs a) {
  pdl_sync();
  const int rows = a.header[1], m_units = (rows + 255) / 256, n_units = a.wide ? (a.n + 511) / 512 : (a.n + 255) / 256, lane = threadIdx.x & 31;
  const Rest rest = *reinterpret_cast<const Rest *>(a.header + 2);
  if (rest.shares == 1) return;
  for (int i = (int)(blockIdx.x * 8 + (threadIdx.x >> 5)); i < rest.rest * 256; i += (int)gridDim.x * 8) {
    int m0, n0;
    unit_place(a.group, m_units, n_units, 256, a.wide ? 512 : 256, rest.whole + (a.wide ? i / 512 : i / 256), &m0, &n0);
    const int row = m0 + i % 256, col = n0 + (a.wide ? i / 256 & 1 : 0) * 256 + lane * 8;
    if (row >= rows || col >= a.n) continue;
    const int src = a.source[row];
    if (src < 0) continue;
    float v[8] = {};
    if (a.label[row] >= 0) {
      const float *p = a.partial + (long long)(i / 256) * rest.shares * 65536 + (i % 256) * 256 + lane * 8;
#pragma unroll 4
      for (int s = 0; s < rest.shares; ++s) {
        const float4 lo = reinterpret_cast<const float4 *>(p + (long long)s * 65536)[0];
        const float4 hi = reinterpret_cast<const float4 *>(p + (long long)s * 65536)[1];
        v[0] += lo.x; v[1] += lo.y; v[2] += lo.z; v[3] += lo.w;
        v[4] += hi.x; v[5] += hi.y; v[6] += hi.z; v[7] += hi.w;
      }
      if (a.drop.threshold) {
        const Keep8 keep = dropout_keep8(a.drop, (uint64_t)src, (uint32_t)col >> 3);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = keep[j] ? v[j] : 0.f;
      }
    }
    store8(a.out + (long long)src * a.ld_out + col,
           make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])), a.n - col);
  }
}

}  // namespace
}  // namespace ngc

// ---- host -------------------------------------------------------------------------------------------
namespace ngc {
namespace {

constexpr size_t kPieceBytes = (size_t)2 << 30;  // room for powers (without a gradient: statistics and features) of a piece
constexpr long long kMostPiece = 1ll << 24;      // rows of a piece
constexpr long long kMostParts = 4096;           // partitions of a piece (each block that places rows adds up the earlier ones' counts)

inline long long up(long long v, long long a) { return (v + a - 1) / a * a; }

struct VocabPlan {
  long long each;      // rows per partition, as the weights' gradient sees them
  long long parts;     // partitions
  long long piece_parts, subs, sub_rows;  // partitions of a piece, or pieces of a partition and their rows
  long long cap;       // packed rows of a piece at most, a multiple of 256
  int bn, stats, d_pad, ld_power;
  bool one_tile;       // a row's classes are one tile: losses and G come from the logits' epilogue
  int few_each;        // few rows: classes of a CTA's tile, else 0
  int w_inner, w_outer, w_pad;  // the weights' rows: elements, number, elements of a copied one (0: not copied)
  int sums_m, sums_pad;
  size_t header, counts, begin, position, source, label, weight, label_sums, stat, packed, copy, power, partial, sums, bytes;
};

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
    p.piece_parts = std::min(std::min(std::max<long long>(1, most / taken), kMostParts), std::max<long long>(1, p.parts));
    p.subs = 1;
    p.sub_rows = p.each;
    rows = std::min<long long>(p.piece_parts * p.each, std::max<int64_t>(1, c.rows));
    p.cap = c.keep_rows ? rows : p.piece_parts * taken;
  } else {
    p.piece_parts = 1;
    most = std::max<long long>(most / kAlign * kAlign, kAlign);  // (whole chunks of K, and no more rows than were asked for)
    p.subs = (p.each + most - 1) / most;
    p.sub_rows = up((p.each + p.subs - 1) / p.subs, kAlign);
    p.subs = (p.each + p.sub_rows - 1) / p.sub_rows;
    rows = p.sub_rows;
    p.cap = rows;
  }
  p.one_tile = c.n_classes <= 256;
  p.bn = c.n_classes <= 128 && p.one_tile ? 128 : 256;
  p.stats = 2 * ((c.n_classes + p.bn - 1) / p.bn);
  if (!p.one_tile && c.rows <= kMostFewRows && p.cap <= kMostFewRows) {  // (many partitions are packed to more)
    // (weights whose classes are contiguous come in boxes of 64 classes, so their tiles are whole)
    const int rounds = (c.n_classes + 256 * pairs - 1) / (256 * pairs), each = (c.n_classes + 2 * pairs * rounds - 1) / (2 * pairs * rounds);
    p.few_each = c.feature_major ? 128 : std::min(128, (int)up(each, 8));
    p.stats = 8 * ((c.n_classes + 2 * p.few_each - 1) / (2 * p.few_each));
  }
  p.cap = up(p.cap, 256);
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
  p.label_sums = take((size_t)p.cap * sizeof(float2));
  p.stat = take((size_t)p.cap * p.stats * sizeof(float2));
  p.packed = take(c.keep_rows ? 0 : (size_t)p.cap * p.d_pad * 2);
  p.copy = take((size_t)p.w_pad * p.w_outer * 2);
  p.power = take(grads ? (size_t)p.cap * p.ld_power * 2 : 0);
  const long long chunks = (c.n_classes + 63) / 64, tiles = p.cap / 256 * ((c.d + 511) / 512) * 2;
  const long long cut = std::min<long long>((long long)kMostRounds * pairs, tiles * std::min<long long>(kMostShares, chunks / kShareChunks));
  p.partial = take(dx && chunks >= 2 * kShareChunks ? (size_t)cut * 65536 * 4 : 0);
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

// bf16 rows of `inner` elements, `ld` apart, `batch` such matrices `stride` apart; boxes of 64 x `box` in 128-byte swizzle; zero
// outside, where nothing is written either.
bool matrix_map(CUtensorMap *m, const void *base, long long inner, long long rows, long long ld, long long batch, long long stride, int box) {
  const EncodeTiled fn = encode_tiled();
  if (!fn) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)inner, (cuuint64_t)rows, (cuuint64_t)batch};
  const cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)stride * 2};
  const cuuint32_t boxes[3] = {64, (cuuint32_t)box, 1}, steps[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, batch > 0 ? 3 : 2, const_cast<void *>(base), dims, strides, boxes, steps,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool row_map(CUtensorMap *m, const void *base, long long inner, long long rows, long long ld, int box) {
  return matrix_map(m, base, inner, rows, ld, 0, 0, box);
}

template <int EPI, int A_MN, int B_MN, int BN, bool Wide>
cudaError_t launch_gemm(const CUtensorMap &a, const CUtensorMap &b, const CUtensorMap &out, const GemmArgs &p, long long tiles, int sms,
                        cudaStream_t stream) {
  auto kern = vocab_gemm_kernel<EPI, A_MN, B_MN, BN, Wide>;
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
  return cudaLaunchKernelEx(&cfg, kern, a, b, out, p);
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
  RowOut out;
  unsigned char *ws;
  bool keep;    // rows stay where they are
  bool direct;  // few scored rows: no kernel before the logits'
  int sms;
  cudaStream_t stream;
};

// One piece: `rows` rows from `first` on, `parts` partitions of `each` rows (the last may be short), the number of the
// first; begin / end: of the pieces that a partition is cut into.
cudaError_t vocab_piece(const VocabCall &q, const VocabPlan &p, long long first, int rows, int each, int parts,
                        long long first_part, bool begin, bool end) {
  const ngc_linear_ce_t &c = *q.cfg;
  const DropoutKey drop = dropout_key(c.dropout, c.seed, c.first_row + (uint64_t)first, c.step);
  const double stretch = vocab_stretch(c.dropout);
  int *header = reinterpret_cast<int *>(q.ws + p.header);
  RowArgs r = {};
  r.x = q.x + first * q.ldx;
  r.ldx = q.ldx; r.d = c.d; r.d_pad = p.d_pad;
  r.rows = rows; r.each = each; r.parts = parts; r.segments = (std::min(each, rows) + kSegment - 1) / kSegment;
  r.n_classes = c.n_classes;
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
  r.out = {q.out.logp + first, q.out.row_loss + first, q.out.loss ? q.out.loss + first : nullptr};
  r.dx = q.dx ? q.dx + first * q.ld_dx : nullptr;
  r.ld_dx = q.ld_dx;
  r.drop = drop;
  r.first_piece = first == 0;
  cudaError_t e;
  constexpr int kWarps = kRowThreads / 32;
  if (q.direct) {
    e = cudaSuccess;
  } else if (q.keep) {
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
  const void *xp = q.keep ? (const void *)r.x : (const void *)r.packed;
  const long long x_rows = q.keep ? rows : p.cap, x_ld = q.keep ? q.ldx : p.d_pad;
  const void *w = p.w_pad ? (const void *)(q.ws + p.copy) : (const void *)q.w;
  const long long w_ld = p.w_pad ? p.w_pad : q.ldw;
  void *power = q.ws + p.power;
  CUtensorMap a, b, out;
  GemmArgs g = {};
  g.batch = 1; g.group = 16;
  g.status = header;
  g.rest = q.dx ? header + 2 : nullptr; g.rest_pairs = std::max(1, q.sms / 2);
  g.source = r.source; g.label = r.label;
  const int m_tiles = (int)((up(rows, kAlign) + (long long)(parts - 1) * kAlign + 255) / 256);

  // (units of two tiles for the features' gradient where they fill a round of pairs at least once)
  g.rest_wide = m_tiles * ((c.d + 511ll) / 512) >= q.sms / 2;

  // logits: powers and statistics, or all of G
  g.m = (int)p.cap; g.m_dev = header + 1; g.n = c.n_classes; g.k = c.d;
  g.label_sums = reinterpret_cast<float2 *>(q.ws + p.label_sums);
  g.stat = reinterpret_cast<float2 *>(q.ws + p.stat);
  g.stats = p.stats;
  g.c = (float)(c.scale * stretch * 1.4426950408889634);
  g.power = grads ? static_cast<__half *>(power) : nullptr;
  g.ld_power = p.ld_power;
  g.weight = r.row_weight; g.factor = (float)(c.scale * stretch); g.rows_out = r.out;
  if (p.few_each) {
    g.m = c.n_classes; g.classes_each = p.few_each;
    if (q.direct) {
      g.m_dev = nullptr;
      g.few_rows = rows;
      g.first = r.first_piece;
      g.label = r.labels;
    }
    if (!row_map(&a, w, p.w_inner, p.w_outer, w_ld, c.feature_major ? 64 : p.few_each) || !row_map(&b, xp, c.d, x_rows, x_ld, 16))
      return cudaErrorInvalidValue;
    const long long units = (c.n_classes + 2 * p.few_each - 1) / (2 * p.few_each);
    e = c.feature_major ? launch_gemm<kFewRows, 1, 0, 256, false>(a, b, b, g, units, q.sms, q.stream)
                        : launch_gemm<kFewRows, 0, 0, 256, false>(a, b, b, g, units, q.sms, q.stream);
  } else {
    if (!row_map(&a, xp, c.d, x_rows, x_ld, 128) || !row_map(&b, w, p.w_inner, p.w_outer, w_ld, c.feature_major ? 64 : p.bn / 2))
      return cudaErrorInvalidValue;
    if (!grads) out = a;  // (not used)
    else if (!matrix_map(&out, power, p.ld_power, p.cap, p.ld_power, 1, p.cap * p.ld_power, 32)) return cudaErrorInvalidValue;
    const long long tiles = (long long)m_tiles * ((c.n_classes + p.bn - 1) / p.bn);
    const bool full = p.bn == 256;
    if (p.one_tile && c.feature_major)
      e = full ? launch_gemm<kGradient, 0, 1, 256, false>(a, b, out, g, tiles, q.sms, q.stream)
               : launch_gemm<kGradient, 0, 1, 128, false>(a, b, out, g, tiles, q.sms, q.stream);
    else if (p.one_tile)
      e = full ? launch_gemm<kGradient, 0, 0, 256, false>(a, b, out, g, tiles, q.sms, q.stream)
               : launch_gemm<kGradient, 0, 0, 128, false>(a, b, out, g, tiles, q.sms, q.stream);
    else
      e = c.feature_major ? launch_gemm<kLogits, 0, 1, 256, false>(a, b, out, g, tiles, q.sms, q.stream)
                          : launch_gemm<kLogits, 0, 0, 256, false>(a, b, out, g, tiles, q.sms, q.stream);
  }
  if (e != cudaSuccess) return e;

  if (!p.one_tile) {
    LossArgs l = {};
    l.header = header; l.source = r.source; l.label = r.label; l.weight = r.row_weight; l.label_sums = g.label_sums; l.stat = g.stat;
    l.stats = p.stats;
    l.few_each = p.few_each;
    l.few_inverse = p.few_each ? (uint32_t)((1ull << 32) / p.few_each + ((1ull << 32) % p.few_each != 0)) : 0;
    l.out = r.out; l.n_classes = c.n_classes;
    if (q.direct) {
      l.header = l.source = nullptr;
      l.label = r.labels; l.weight = r.weight; l.rows = rows;
    }
    l.power = g.power; l.ld_power = p.ld_power;
    l.factor = g.factor;
    l.c = g.c;
    const long long most = q.direct ? rows : up(rows, kAlign) + (q.keep ? 0 : (long long)(parts - 1) * kAlign);
    if (c.n_classes <= 2048) {
      e = launch_k(vocab_loss_kernel<32>, (unsigned)((most + 7) / 8), 256, 0, q.stream, l);
    } else {
      // few rows: several blocks for each, of at least one round of vectors
      const long long shares = grads ? std::min<long long>(q.sms * 8ll / rows, p.ld_power / (8 * 128 * 2)) : 1;
      e = launch_k(vocab_loss_kernel<128>, dim3((unsigned)most, (unsigned)std::max<long long>(1, shares)), 128, 0, q.stream, l);
    }
    if (e != cudaSuccess) return e;
  }

  if (q.dx) {
    g.n = c.d; g.k = c.n_classes;
    g.out = r.dx; g.ld_out = q.ld_dx;
    g.store = aligned(r.dx, 16) && q.ld_dx % 8 == 0;
    g.partial = reinterpret_cast<float *>(q.ws + p.partial);
    g.drop = drop;
    if (!row_map(&a, power, p.ld_power, p.cap, p.ld_power, 128)) return cudaErrorInvalidValue;
    if (!row_map(&b, w, p.w_inner, p.w_outer, w_ld, c.feature_major ? 128 : 64)) return cudaErrorInvalidValue;
    // (how many rows count is known on the device alone: with contractions that can be cut, all pairs are there)
    const bool cut = (c.n_classes + 63) / 64 >= 2 * kShareChunks;
    const long long tiles = cut ? q.sms : (long long)m_tiles * ((c.d + 255) / 256);
    if (g.rest_wide)
      e = c.feature_major ? launch_gemm<kFeatureGrad, 0, 0, 256, true>(a, b, a, g, tiles, q.sms, q.stream)
                          : launch_gemm<kFeatureGrad, 0, 1, 256, true>(a, b, a, g, tiles, q.sms, q.stream);
    else
      e = c.feature_major ? launch_gemm<kFeatureGrad, 0, 0, 256, false>(a, b, a, g, tiles, q.sms, q.stream)
                          : launch_gemm<kFeatureGrad, 0, 1, 256, false>(a, b, a, g, tiles, q.sms, q.stream);
    if (e == cudaSuccess && cut) {
      JoinArgs j = {header, r.source, r.label, g.partial, c.d, g.group, g.rest_wide, r.dx, q.ld_dx, drop};
      e = launch_k(vocab_join_kernel, (unsigned)q.sms * 4, 256, 0, q.stream, j);
    }
    if (e != cudaSuccess) return e;
  }
  if (q.dw) {
    g.m_dev = nullptr;
    g.k_begin = r.begin; g.batch = parts;
    g.out = q.dw + first_part * q.dw_part; g.ld_out = q.ld_dw; g.out_batch = q.dw_part;
    g.partial = p.subs > 1 ? reinterpret_cast<float *>(q.ws + p.sums) : nullptr;
    g.n_pad = p.sums_pad;
    g.first = begin; g.last = end;
    g.m = p.w_outer; g.n = p.w_inner;
    // (a bulk store writes whole 16 bytes: with n = 333 the columns 333 .. 335 of a wider buffer were lost)
    g.store = aligned(g.out, 16) && g.n % 8 == 0 && q.ld_dw % 8 == 0 && (parts == 1 || q.dw_part % 8 == 0);
    CUtensorMap powers, features;
    if (!row_map(&powers, power, p.ld_power, p.cap, p.ld_power, 64)) return cudaErrorInvalidValue;
    if (!row_map(&features, xp, c.d, x_rows, x_ld, 64)) return cudaErrorInvalidValue;
    if (g.store && !matrix_map(&out, g.out, g.n, g.m, q.ld_dw, parts, parts == 1 ? q.ld_dw : q.dw_part, 32))
      return cudaErrorInvalidValue;
    const long long tiles = (long long)((g.m + 255) / 256) * ((g.n + 255) / 256) * parts;
    const CUtensorMap &ma = c.feature_major ? features : powers, &mb = c.feature_major ? powers : features;
    if (each >= kLongContraction * 64 && g.m > 256) {
      g.group = 8;
      e = launch_gemm<kWeightGrad, 1, 1, 256, true>(ma, mb, out, g, tiles, q.sms, q.stream);
    } else {
      e = launch_gemm<kWeightGrad, 1, 1, 256, false>(ma, mb, out, g, tiles, q.sms, q.stream);
    }
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
    const MatrixSpan w(W, outer, (int)inner, ld_w, 2), gw(dW, outer, (int)inner, ld_dw, 2);
    const Span status(workspace, workspace_bytes < 4 ? 0 : 4);
    if (!apart(gw, w) || !apart(status, {w.span, gw.span}) || !aligned(workspace, 4)) return NGC_ERR_INVALID;
    if (workspace && workspace_bytes >= 4 && cudaMemsetAsync(workspace, 0, 4, stream) != cudaSuccess) return NGC_ERR_CUDA;
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
  const bool can_keep = aligned(X, 16) && ld_x % 8 == 0 && c.dropout == 0.0 && (p.parts <= 1 || p.each % kAlign == 0);
  if (c.keep_rows && !can_keep) return NGC_ERR_INVALID;
  // (few scored rows cost the same where they are, and a left-out one reaches no other: packing them is not worth a launch)
  const bool direct = can_keep && p.few_each && !dX && !dW, keep = c.keep_rows || direct;
  const size_t vec = (size_t)rows * 4;
  const MatrixSpan x(X, rows, c.d, ld_x, 2), w(W, outer, (int)inner, ld_w, 2), gx(dX, rows, c.d, ld_dx, 2);
  const bool even = all_parts == 1 || dw_stride % std::max<int64_t>(1, ld_dw) == 0;
  const MatrixSpan gw(Span(dW, (size_t)((all_parts - 1) * dw_stride + (outer - 1) * ld_dw + inner) * 2), (uintptr_t)inner * 2,
                      even ? (uintptr_t)ld_dw * 2 : 0);
  const Span lab(labels, vec), weight(row_weight, vec), lp(logp, vec), row(row_loss, vec), sum(loss, (size_t)all_parts * 4);
  const Span ws(workspace, p.bytes);
  if (!apart(ws, {x.span, w.span, gx.span, gw.span, lab, weight, lp, row, sum}) || !apart(gx.span, {lab, weight, lp, row, sum}) ||
      !apart(gw.span, {lab, weight, lp, row, sum}) || !apart(lp, {x.span, w.span, lab, weight, row, sum}) ||
      !apart(row, {x.span, w.span, lab, weight, sum}) || !apart(sum, {x.span, w.span, lab, weight}))
    return NGC_ERR_INVALID;
  for (const MatrixSpan *g : {&gx, &gw})
    if (!apart(*g, x) || !apart(*g, w)) return NGC_ERR_INVALID;
  if (!apart(gx, gw)) return NGC_ERR_INVALID;
  VocabCall q = {cfg, static_cast<const __nv_bfloat16 *>(X), static_cast<const __nv_bfloat16 *>(W), ld_x, ld_w, labels, row_weight,
                 static_cast<__nv_bfloat16 *>(dX), static_cast<__nv_bfloat16 *>(dW), ld_dx, ld_dw, dw_stride,
                 {logp, row_loss, c.rows_per_partition == 1 ? loss : nullptr}, static_cast<unsigned char *>(workspace), keep, direct, sms, stream};
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
  if (loss && c.rows_per_partition > 1 && launch_partition_sums(row_loss, (int)rows, c.rows_per_partition, loss, stream) != cudaSuccess) return NGC_ERR_CUDA;
  return NGC_OK;
}

}  // extern "C"

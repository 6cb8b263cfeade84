// ngc_adamw_update: the AdamW update of many tensors in one launch, states in fp32 or in e4m3 with one fp32 scale
// per 256 elements.
//
// What has to move per parameter (fp32 theta and gradient): theta 4 + 4, gradient 4, and m, v 8 + 8 in fp32 or
// 2 + 2 in 8 bits (plus 16 / 256 for the scales): 28 or 16.06 bytes.  Memory is the bound of the fp32 form; the 8-bit
// form also keeps the schedulers busy (62 instructions per element with two elements per multiplication, 65 without).
// A warp takes one block of 256 elements: lane i holds elements 4 i .. 4 i + 3 and 128 + 4 i .. 128 + 4 i + 3, so that
// every array is read and written in whole 128-byte (e4m3), 256-byte (bf16) or 512-byte (fp32) pieces and the largest
// magnitude of an 8-bit block is a reduction within the warp.
//
// Four warps per thread block and one block of 256 elements per warp, so that occupancy, not a pipeline inside the
// warp, keeps the loads in flight.  302 million parameters, fp32 states: 1.219 ms, 6.94 TB/s; e4m3: 0.804 ms, 6.0 TB/s
// (0.828 ms before two elements shared their multiplications).  Measured at 0.839 ms: four blocks per warp with the
// next one's values prefetched into registers (72-96 instead of 48-56) 0.990 ms, eight 0.903 ms, without prefetch
// 1.168 ms; 8 / 16 warps per thread block 0.862 / 0.886 ms.
//
// The moments are formed with one rounding per product and sum, not with fused multiply-adds: a value that lies on
// the border of two codes then falls on the same side in any fp32 implementation of the formulas, and one flipped
// code is 6 % of an element.  (With packed sums, which the compiler fuses with their products: 0.769 ms.)
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "ngc_device.h"
#include "ngc_f32x2.cuh"
#include "ngc_pdl.cuh"

namespace ngc {
namespace {

constexpr int kBlock = NGC_ADAMW_BLOCK;
constexpr int kWarps = 4;                // per thread block, one block of 256 elements each
constexpr int kGroup = kWarps * kBlock;  // elements of a thread block
constexpr float kE4m3Max = 448.f;
constexpr float kE4m3Tiny = 0x1p-9f;  // smallest positive value of the format
constexpr float kNothing = 0x1p-110f; // a block below this has no scale whose reciprocal is a finite float

struct Entry {
  void *theta;
  const void *grad;
  void *m, *v;
  float *m_scale, *v_scale;
  long long numel;
  float decay;
  int vec;              // every pointer is aligned for four elements at once
  unsigned first_group; // thread blocks that the tensors before this one take
};

// The descriptors travel as the kernel's parameter (32 764 bytes at most), so a launch needs no table in device
// memory, and a captured one keeps its own copy.
template <int N>
struct Table {
  Entry e[N];
  int n;
  float lr, b1, omb1, b2, omb2, grad_scale;
  float den_root, den_eps;     // of the host's step number
  double log_b1, log_b2, eps;  // for the step number in device memory
  const long long *step_dev;
};
constexpr int kFew = 4, kSmall = 48, kLarge = 440;
static_assert(sizeof(Table<kLarge>) <= 32764, "kernel parameters end at 32 764 bytes");
static_assert(sizeof(Table<kSmall>) <= 4096, "the small table fits the classic parameter size");

// Four consecutive values as they lie in memory, and as floats.
template <typename T> struct Four;
template <> struct Four<float> { using type = float4; };
template <> struct Four<__nv_bfloat16> { using type = uint2; };
template <> struct Four<__nv_fp8_storage_t> { using type = uint32_t; };

__device__ __forceinline__ void unpack(const float4 &q, float (&x)[4]) { x[0] = q.x; x[1] = q.y; x[2] = q.z; x[3] = q.w; }
__device__ __forceinline__ void unpack(const uint2 &q, float (&x)[4]) {  // bf16 is the upper half of a float
  x[0] = __uint_as_float(q.x << 16); x[1] = __uint_as_float(q.x & 0xffff0000u);
  x[2] = __uint_as_float(q.y << 16); x[3] = __uint_as_float(q.y & 0xffff0000u);
}
__device__ __forceinline__ void unpack(const uint32_t &q, float (&x)[4]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float2 f = __half22float2(__half2(
        __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(q >> (16 * h)), __NV_E4M3)));
    x[2 * h] = f.x; x[2 * h + 1] = f.y;
  }
}

// The first `left` of four values at `p` (the others zero); `vec`: the address is aligned for all four at once.
template <typename T>
__device__ __forceinline__ typename Four<T>::type load4(const T *p, int left, bool vec) {
  using V = typename Four<T>::type;
  if (vec && left >= 4) return *reinterpret_cast<const V *>(p);
  union { V v; T x[4]; } q;
  memset(&q, 0, sizeof(q));
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < left) q.x[i] = p[i];
  return q.v;
}

template <typename T>
__device__ __forceinline__ void store4(T *p, int left, bool vec, const float (&x)[4]);
template <>
__device__ __forceinline__ void store4<float>(float *p, int left, bool vec, const float (&x)[4]) {
  if (vec && left >= 4) {
    *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) p[i] = x[i];
  }
}
template <>
__device__ __forceinline__ void store4<__nv_bfloat16>(__nv_bfloat16 *p, int left, bool vec, const float (&x)[4]) {
  if (vec && left >= 4) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
    *reinterpret_cast<uint2 *>(p) =
        make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) p[i] = __float2bfloat16_rn(x[i]);
  }
}
template <>
__device__ __forceinline__ void store4<__nv_fp8_storage_t>(__nv_fp8_storage_t *p, int left, bool vec,
                                                           const float (&x)[4]) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(x[0], x[1]), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(x[2], x[3]), __NV_SATFINITE, __NV_E4M3);
  const uint32_t q = lo | (hi << 16);
  if (vec && left >= 4) {
    *reinterpret_cast<uint32_t *>(p) = q;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) p[i] = (__nv_fp8_storage_t)(q >> (8 * i));
  }
}

// Largest of the warp's values, none of them negative: such floats order as their bit patterns do.
__device__ __forceinline__ float warp_max(float a) {
  return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(a)));
}

// What the kernel uses of the table, in registers.  With B1 = 1 - beta1^t and B2 = 1 - beta2^t the step is
// m / (sqrt(v) B1 / sqrt(B2) + eps B1).
struct Step {
  float lr, b1, omb1, b2, omb2, grad_scale, decay, den_root, den_eps;
};
// Within one unit in the last place (it only enters theta, times lr).
__device__ __forceinline__ float reciprocal(float x) {
  float r;
  asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// What a lane reads of one block of 256 elements.
template <typename TT, typename TG, typename TS>
struct Loaded {
  typename Four<TT>::type th[2];
  typename Four<TG>::type g[2];
  typename Four<TS>::type m[2], v[2];
  float m_scale, v_scale;
};
template <typename TT, typename TG, typename TS>
struct Block {  // where a block lies
  TT *theta;
  const TG *grad;
  TS *m, *v;
  float *m_scale, *v_scale;
};

// Whole: no element is missing and every pointer is aligned for four elements.
template <bool Whole, typename TT, typename TG, typename TS>
__device__ __forceinline__ void load_block(const Block<TT, TG, TS> &b, int valid, bool vec, int lane,
                                           Loaded<TT, TG, TS> &x) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int at = h * 128 + lane * 4, left = Whole ? 4 : valid - at;
    x.th[h] = load4<TT>(b.theta + at, left, Whole || vec);
    x.g[h] = load4<TG>(b.grad + at, left, Whole || vec);
    x.m[h] = load4<TS>(b.m + at, left, Whole || vec);
    x.v[h] = load4<TS>(b.v + at, left, Whole || vec);
  }
  if (sizeof(TS) == 1) {
    x.m_scale = *b.m_scale;
    x.v_scale = *b.v_scale;
  }
}

template <bool Whole, typename TT, typename TG, typename TS>
__device__ __forceinline__ void update_block(const Step &t, const Block<TT, TG, TS> &b, const Loaded<TT, TG, TS> &x,
                                             int valid, bool vec, int lane) {
  constexpr bool Small8 = sizeof(TS) == 1;
  float m[2][4], v[2][4];
  float mt = 0.f, vt = 0.f;
  const f32x2 b1 = pack2(t.b1, t.b1), omb1 = pack2(t.omb1, t.omb1), b2 = pack2(t.b2, t.b2), omb2 = pack2(t.omb2, t.omb2);
  const f32x2 gs = pack2(t.grad_scale, t.grad_scale), decay = pack2(t.decay, t.decay), lr = pack2(-t.lr, -t.lr);
  const f32x2 den_root = pack2(t.den_root, t.den_root), den_eps = pack2(t.den_eps, t.den_eps);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float th[4], g[4];
    unpack(x.th[h], th);
    unpack(x.g[h], g);
    unpack(x.m[h], m[h]);
    unpack(x.v[h], v[h]);
#pragma unroll
    for (int i = 0; i < 4; i += 2) {  // two elements per instruction, each operation rounded as alone
      f32x2 mm = pack2(m[h][i], m[h][i + 1]), vv = pack2(v[h][i], v[h][i + 1]);
      if (Small8) {
        mm = mul2(mm, pack2(x.m_scale, x.m_scale));
        vv = mul2(vv, pack2(x.v_scale, x.v_scale));
        vv = mul2(vv, vv);
      }
      const f32x2 gg = mul2(pack2(g[i], g[i + 1]), gs);
      // (the sums one by one: packed ones would be fused with their products)
      float a0, a1, c0, c1;
      unpack2(mul2(mm, b1), a0, a1);
      unpack2(mul2(gg, omb1), c0, c1);
      m[h][i] = __fadd_rn(a0, c0);
      m[h][i + 1] = __fadd_rn(a1, c1);
      unpack2(mul2(vv, b2), a0, a1);
      unpack2(mul2(mul2(gg, gg), omb2), c0, c1);
      v[h][i] = __fadd_rn(a0, c0);
      v[h][i + 1] = __fadd_rn(a1, c1);
      const float r0 = sqrtf(v[h][i]), r1 = sqrtf(v[h][i + 1]);
      float d0, d1;
      unpack2(mad2(pack2(r0, r1), den_root, den_eps), d0, d1);
      const f32x2 step = mul2(pack2(m[h][i], m[h][i + 1]), pack2(reciprocal(d0), reciprocal(d1)));
      const f32x2 old = pack2(th[i], th[i + 1]);
      unpack2(mad2(lr, mad2(decay, old, step), old), th[i], th[i + 1]);
      if (Small8) {
        v[h][i] = r0;
        v[h][i + 1] = r1;
        mt = fmaxf(mt, fmaxf(fabsf(m[h][i]), fabsf(m[h][i + 1])));
        vt = fmaxf(vt, fmaxf(r0, r1));
      }
    }
    const int at = h * 128 + lane * 4;
    store4<TT>(b.theta + at, Whole ? 4 : valid - at, Whole || vec, th);
  }
  if (Small8) {
    mt = warp_max(mt);
    vt = warp_max(vt);
    const bool mo = mt >= kNothing, vo = vt >= kNothing;
    const float mi = mo ? __frcp_rn(mt) * kE4m3Max : 0.f, vi = vo ? __frcp_rn(vt) * kE4m3Max : 0.f;
    const float least = vo ? kE4m3Tiny : 0.f;
    if (lane == 0) {  // (warp_max is a barrier of the warp: every lane has read the old scales)
      *b.m_scale = mo ? mt * (1.f / kE4m3Max) : 0.f;
      *b.v_scale = vo ? vt * (1.f / kE4m3Max) : 0.f;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        m[h][i] *= mi;
        const float q = v[h][i] * vi;
        v[h][i] = v[h][i] > 0.f ? fmaxf(q, least) : q;
      }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int at = h * 128 + lane * 4, left = Whole ? 4 : valid - at;
    store4<TS>(b.m + at, left, Whole || vec, m[h]);
    store4<TS>(b.v + at, left, Whole || vec, v[h]);
  }
}

template <typename TT, typename TG, bool Small8, int N>
__global__ void __launch_bounds__(kWarps * 32)
adamw_kernel(const __grid_constant__ Table<N> t) {
  pdl_sync();
  // the tensor whose thread blocks contain this one
  int lo = 0, hi = t.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.e[mid].first_group <= blockIdx.x) lo = mid; else hi = mid - 1;
  }
  const Entry &e = t.e[lo];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  Step st{t.lr, t.b1, t.omb1, t.b2, t.omb2, t.grad_scale, e.decay, t.den_root, t.den_eps};
  if (t.step_dev) {
    const double s = (double)max(*t.step_dev, 1ll), b1 = -expm1(s * t.log_b1), b2 = -expm1(s * t.log_b2);
    st.den_root = (float)(b1 / sqrt(b2));
    st.den_eps = (float)(t.eps * b1);
  }
  using TS = typename std::conditional<Small8, __nv_fp8_storage_t, float>::type;
  const long long block = (long long)(blockIdx.x - e.first_group) * kWarps + warp, base = block * kBlock;
  const long long left = e.numel - base;
  if (left <= 0) return;  // (the whole warp)
  const Block<TT, TG, TS> b{static_cast<TT *>(e.theta) + base, static_cast<const TG *>(e.grad) + base,
                            static_cast<TS *>(e.m) + base,     static_cast<TS *>(e.v) + base,
                            e.m_scale + block,                 e.v_scale + block};  // (scales: 8-bit states only)
  Loaded<TT, TG, TS> x;
  if (e.vec && left >= kBlock) {
    load_block<true>(b, kBlock, true, lane, x);
    update_block<true>(st, b, x, kBlock, true, lane);
  } else {
    const int valid = left < kBlock ? (int)left : kBlock;
    load_block<false>(b, valid, e.vec != 0, lane, x);
    update_block<false>(st, b, x, valid, e.vec != 0, lane);
  }
}

template <typename TT, typename TG, bool Small8, int N>
cudaError_t launch(const Table<N> &t, unsigned groups, cudaStream_t stream) {
  return launch_k(adamw_kernel<TT, TG, Small8, N>, groups, kWarps * 32, 0, stream, t);
}

template <int N>
cudaError_t launch_types(const ngc_adamw_t &c, const Table<N> &t, unsigned groups, cudaStream_t stream) {
  using B = __nv_bfloat16;
  const bool tb = c.theta_dtype == NGC_BF16, gb = c.grad_dtype == NGC_BF16;
  if (c.state_dtype == NGC_E4M3) {
    if (tb) return gb ? launch<B, B, true>(t, groups, stream) : launch<B, float, true>(t, groups, stream);
    return gb ? launch<float, B, true>(t, groups, stream) : launch<float, float, true>(t, groups, stream);
  }
  if (tb) return gb ? launch<B, B, false>(t, groups, stream) : launch<B, float, false>(t, groups, stream);
  return gb ? launch<float, B, false>(t, groups, stream) : launch<float, float, false>(t, groups, stream);
}

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Bytes [first, last) of tensor i.
struct Range {
  uintptr_t first, last;
  int i;
  bool operator<(const Range &o) const { return first < o.first; }
};
using Ranges = std::vector<Range>;
bool ascending(const Ranges &r) {
  for (size_t i = 1; i < r.size(); ++i)
    if (r[i].first < r[i - 1].last) return false;
  return true;
}
// True when no two of the ranges overlap, over all kinds (theta, m, v and the scales).  Tensors usually come in the order of
// their addresses, and often the kinds one after another; only others are sorted.  `lists`: how many of the vectors, in
// order, hold all ranges afterwards.
bool disjoint(Ranges (&r)[5], int kinds, int &lists) {
  Ranges hulls;
  lists = kinds;
  for (int k = 0; k < kinds; ++k) {
    if (!ascending(r[k])) {
      std::sort(r[k].begin(), r[k].end());
      if (!ascending(r[k])) return false;
    }
    if (!r[k].empty()) hulls.push_back({r[k].front().first, r[k].back().last, 0});
  }
  std::sort(hulls.begin(), hulls.end());
  if (ascending(hulls)) return true;
  for (int k = 1; k < kinds; ++k) r[0].insert(r[0].end(), r[k].begin(), r[k].end());
  std::sort(r[0].begin(), r[0].end());
  lists = 1;
  return ascending(r[0]);
}
// True when what is only read (gradients, which may share memory among themselves, and the step number) shares no byte with
// the written ranges, in order and disjoint, but for a tensor's own range as a whole: a thread reads its elements of
// every array before it writes any.  Other warps would read the rest while it is being written.
bool read_apart(const Ranges &reads, const Ranges &writes) {
  auto w = writes.begin();
  for (const Range &x : reads) {
    while (w != writes.end() && w->last <= x.first) ++w;
    if (w == writes.end()) return true;
    if (w->first < x.last && !(w->first == x.first && w->last == x.last && w->i == x.i)) return false;
  }
  return true;
}

int check(const ngc_adamw_t &c, const ngc_adamw_tensor_t *ts, int n) {
  if ((c.theta_dtype != NGC_F32 && c.theta_dtype != NGC_BF16) || (c.grad_dtype != NGC_F32 && c.grad_dtype != NGC_BF16) ||
      (c.state_dtype != NGC_F32 && c.state_dtype != NGC_E4M3))
    return NGC_ERR_INVALID;
  if (!std::isfinite((float)c.lr) || !std::isfinite((float)c.grad_scale) || !(c.beta1 >= 0.0 && c.beta1 < 1.0) ||
      !(c.beta2 >= 0.0 && c.beta2 < 1.0) || !std::isfinite(c.eps) || !((float)(c.eps * (1.0 - c.beta1)) >= FLT_MIN))
    return NGC_ERR_INVALID;
  if (!c.step_dev && c.step < 1) return NGC_ERR_INVALID;
  if (c.step_dev && !aligned(c.step_dev, 8)) return NGC_ERR_INVALID;
  const size_t tb = c.theta_dtype == NGC_F32 ? 4 : 2, gb = c.grad_dtype == NGC_F32 ? 4 : 2;
  const size_t sb = c.state_dtype == NGC_F32 ? 4 : 1;
  const int kinds = c.state_dtype == NGC_E4M3 ? 5 : 3;
  Ranges r[5];
  for (int k = 0; k < kinds; ++k) r[k].reserve(n);
  Ranges reads;
  reads.reserve(n + 1);
  const auto range = [](const void *p, size_t bytes, int i) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    return Range{a, a + bytes, i};
  };
  for (int i = 0; i < n; ++i) {
    const ngc_adamw_tensor_t &t = ts[i];
    // (2^38 elements: their thread blocks still count in 31 bits)
    if (t.numel < 0 || t.numel > (1ll << 38) || !std::isfinite((float)t.weight_decay)) return NGC_ERR_INVALID;
    if (t.numel == 0) continue;
    if (!t.theta_dev || !t.grad_dev || !t.m_dev || !t.v_dev || !aligned(t.theta_dev, tb) || !aligned(t.grad_dev, gb) ||
        !aligned(t.m_dev, sb) || !aligned(t.v_dev, sb))
      return NGC_ERR_INVALID;
    if (c.state_dtype == NGC_E4M3 &&
        (!t.m_scale_dev || !t.v_scale_dev || !aligned(t.m_scale_dev, 4) || !aligned(t.v_scale_dev, 4)))
      return NGC_ERR_INVALID;
    const void *p[5] = {t.theta_dev, t.m_dev, t.v_dev, t.m_scale_dev, t.v_scale_dev};
    const size_t whole = (size_t)t.numel, blocks = (whole + kBlock - 1) / kBlock;
    const size_t bytes[5] = {whole * tb, whole * sb, whole * sb, blocks * 4, blocks * 4};
    for (int k = 0; k < kinds; ++k) r[k].push_back(range(p[k], bytes[k], i));
    reads.push_back(range(t.grad_dev, whole * gb, i));
  }
  int lists;
  if (!disjoint(r, kinds, lists)) return NGC_ERR_INVALID;
  if (c.step_dev) reads.push_back(range(c.step_dev, 8, -1));
  if (!std::is_sorted(reads.begin(), reads.end())) std::sort(reads.begin(), reads.end());
  for (int k = 0; k < lists; ++k)
    if (!read_apart(reads, r[k])) return NGC_ERR_INVALID;
  return NGC_OK;
}

template <int N>
int run(const ngc_adamw_t &c, const ngc_adamw_tensor_t *ts, int n, cudaStream_t stream) {
  Table<N> t = {};
  t.lr = (float)c.lr; t.b1 = (float)c.beta1; t.omb1 = (float)(1.0 - c.beta1);
  t.b2 = (float)c.beta2; t.omb2 = (float)(1.0 - c.beta2);
  t.eps = c.eps; t.grad_scale = (float)c.grad_scale;
  t.log_b1 = std::log(c.beta1); t.log_b2 = std::log(c.beta2);  // (-inf for 0: the correction is then 1)
  t.step_dev = reinterpret_cast<const long long *>(c.step_dev);
  if (!c.step_dev) {
    const double b1 = -std::expm1((double)c.step * t.log_b1), b2 = -std::expm1((double)c.step * t.log_b2);
    t.den_root = (float)(b1 / std::sqrt(b2));
    t.den_eps = (float)(c.eps * b1);
  }
  const size_t tb = c.theta_dtype == NGC_F32 ? 16 : 8, gb = c.grad_dtype == NGC_F32 ? 16 : 8;
  const size_t sb = c.state_dtype == NGC_F32 ? 16 : 4;
  long long groups = 0;
  for (int i = 0; i < n; ++i) {
    const ngc_adamw_tensor_t &s = ts[i];
    if (s.numel > 0) {
      const long long mine = (s.numel + (long long)kGroup - 1) / kGroup;
      if (t.n == N || groups + mine > 0x7fffffffll) {
        if (launch_types(c, t, (unsigned)groups, stream) != cudaSuccess) return NGC_ERR_CUDA;
        t.n = 0;
        groups = 0;
      }
      Entry &e = t.e[t.n++];
      e.theta = s.theta_dev; e.grad = s.grad_dev; e.m = s.m_dev; e.v = s.v_dev;
      e.m_scale = s.m_scale_dev; e.v_scale = s.v_scale_dev;
      e.numel = s.numel;
      e.decay = (float)s.weight_decay;
      e.vec = aligned(s.theta_dev, tb) && aligned(s.grad_dev, gb) && aligned(s.m_dev, sb) && aligned(s.v_dev, sb);
      e.first_group = (unsigned)groups;
      groups += mine;
    }
  }
  if (t.n > 0 && launch_types(c, t, (unsigned)groups, stream) != cudaSuccess) return NGC_ERR_CUDA;
  return NGC_OK;
}

}  // namespace
}  // namespace ngc

extern "C" int ngc_adamw_update(const ngc_adamw_t *cfg, const ngc_adamw_tensor_t *tensors, int n_tensors,
                                void *cuda_stream) {
  if (!cfg || n_tensors < 0 || (n_tensors > 0 && !tensors)) return NGC_ERR_INVALID;
  try {
    const int rc = ngc::check(*cfg, tensors, n_tensors);
    if (rc != NGC_OK) return rc;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (n_tensors <= ngc::kFew) return ngc::run<ngc::kFew>(*cfg, tensors, n_tensors, stream);
    if (n_tensors <= ngc::kSmall) return ngc::run<ngc::kSmall>(*cfg, tensors, n_tensors, stream);
    return ngc::run<ngc::kLarge>(*cfg, tensors, n_tensors, stream);
  } catch (const std::bad_alloc &) {
    return NGC_ERR_NOMEM;
  }
}

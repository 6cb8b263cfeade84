// ngc_policy_loss and ngc_preference_loss: losses on rows of logits and their gradients.
//
// One row.  With x its logits, c = scale log2(e) in fp32 and M = max x, the probabilities are
// p_v = 2^(c (x_v - M)) / s.  The label's term is kept out of the sum: s = rest + e_y.  Then
// log p_y = ln2 c (x_y - M) - ln(rest + e_y), and 1 - p_y = rest / s is exact where p_y is close to one.  The difference
// x - M comes first (it is exact near the maximum, and finite where c x alone would overflow), one rounding each for it
// and its product.  A thread sums its terms relative to the maximum of its own logits; threads are then joined pairwise
// in a fixed order.  All that happens once per row (logarithm, ratio, KL term) is done in fp64.
#include <cuda_bf16.h>

#include <cmath>

#include "ngc_device.h"
#include "ngc_pdl.cuh"

namespace ngc {
namespace {

constexpr float kNegInf = -INFINITY;
constexpr double kLn2 = 0.693147180559945309417232121458;

__device__ __forceinline__ float exp2_fast(float x) {  // relative error 2^-22, results below 2^-126 become zero
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 16 bytes of logits.
template <typename T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int n = 4;
  static __device__ __forceinline__ void unpack(const uint4 &q, float (&x)[4]) {
    x[0] = __uint_as_float(q.x); x[1] = __uint_as_float(q.y); x[2] = __uint_as_float(q.z); x[3] = __uint_as_float(q.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};
template <>
struct Vec<__nv_bfloat16> {
  static constexpr int n = 8;
  static __device__ __forceinline__ void unpack(const uint4 &q, float (&x)[8]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t *>(&b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// Elements between the last 16-byte boundary at or before `p` and `p`.
template <typename T>
__device__ __forceinline__ int misalignment(const T *p) {
  return (int)((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T));
}

// Maximum m of a set of logits and the sum s of 2^(c (x - m)) over it; an empty set is (-infinity, 0).
struct Sum {
  float m, s;
};
__device__ __forceinline__ float shift_of(float m) { return m == kNegInf ? 0.f : m; }
__device__ __forceinline__ Sum join(const Sum &a, const Sum &b, float c) {
  const float m = fmaxf(a.m, b.m), at = shift_of(m);
  return {m, a.s * exp2_fast(c * (a.m - at)) + b.s * exp2_fast(c * (b.m - at))};
}
template <int N>
__device__ __forceinline__ Sum join_values(const Sum &a, const float (&x)[N], float c) {
  float m = a.m;
#pragma unroll
  for (int i = 0; i < N; ++i) m = fmaxf(m, x[i]);
  const float at = shift_of(m);
  float s = a.s * exp2_fast(c * (a.m - at));
#pragma unroll
  for (int i = 0; i < N; ++i) s += exp2_fast(c * (x[i] - at));
  return {m, s};
}
__device__ __forceinline__ Sum warp_join(Sum a, float c) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const Sum b{__shfl_xor_sync(0xffffffffu, a.m, o), __shfl_xor_sync(0xffffffffu, a.s, o)};
    a = join(a, b, c);  // (symmetric: every lane ends with the same bits)
  }
  return a;
}

// What a row leaves behind: top = max over all logits, e_y and rest (the sum without the label) relative to it.
struct Row {
  float top, e_y, rest, x_y;
  __device__ __forceinline__ Row(const Sum &others, float x_label, float c) {
    top = fmaxf(others.m, x_label);
    const float at = shift_of(top);
    rest = others.s * exp2_fast(c * (others.m - at));
    e_y = exp2_fast(c * (x_label - at));
    x_y = x_label;
  }
  // all logits -infinity (a NaN among them is in `rest`)
  __device__ __forceinline__ bool nothing() const { return top == kNegInf && rest == 0.f && !(x_y != x_y); }
  __device__ __forceinline__ double logp(float c) const {
    if (x_y == top) return -log1p((double)rest);
    return kLn2 * (double)c * ((double)x_y - (double)top) - log((double)rest + (double)e_y);
  }
};

struct PolicyArgs {
  const void *logits;
  void *grad;  // may be null
  long long ld, ld_grad;
  int rows, n_classes;
  const int *actions;
  const float *old_logp, *ref_logp, *advantage, *weight;
  float *logp, *row_loss;
  float c;  // scale log2(e)
  double scale, low, high, kl;
};

// Loss of a row and the factor k of its gradient k (onehot - p).
__device__ __forceinline__ void policy_terms(const PolicyArgs &a, const Row &r, int row, float &logp, float &loss,
                                             float &k) {
  const double w = a.weight ? (double)a.weight[row] : 1.0, adv = a.advantage[row];
  const double lp = r.logp(a.c), ratio = exp(lp - (double)a.old_logp[row]);
  const double free_ = ratio * adv, held = fmin(fmax(ratio, a.low), a.high) * adv;
  double value = -fmin(free_, held), slope = free_ <= held ? -free_ : 0.0;
  if (a.ref_logp) {
    const double d = (double)a.ref_logp[row] - lp, q = expm1(d);
    value += a.kl * (isinf(q) ? q : q - d);
    slope -= a.kl * q;
  }
  logp = (float)lp;
  loss = (float)(w * value);
  k = (float)(w * slope * a.scale);
}

constexpr int kRowThreads = 256;

// One row over a thread block: f(i, n) for whole vectors i < n, g(v) for the single elements before and after them.
template <typename T, typename F, typename G>
__device__ __forceinline__ void for_row(const T *row, int n_classes, F whole, G single) {
  constexpr int N = Vec<T>::n;
  const int mis = misalignment(row), head = min(n_classes, mis ? N - mis : 0), vecs = (n_classes - head) / N;
  for (int i = threadIdx.x; i < vecs; i += blockDim.x) whole(head + i * N);
  const int loose = n_classes - vecs * N;  // at most 2 N - 2
  if ((int)threadIdx.x < loose) single((int)threadIdx.x < head ? (int)threadIdx.x : vecs * N + (int)threadIdx.x);
}

// Sum over a row without its label, the same in every thread.  `part`: shared, one Sum per warp.
template <typename T>
__device__ __forceinline__ Sum block_sum(const T *row, int n_classes, int label, float c, Sum *part) {
  constexpr int N = Vec<T>::n;
  Sum a{kNegInf, 0.f};
  for_row(
      row, n_classes,
      [&](int v) {
        float x[N];
        Vec<T>::unpack(*reinterpret_cast<const uint4 *>(row + v), x);
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (v + i == label) x[i] = kNegInf;
        a = join_values(a, x, c);
      },
      [&](int v) {
        if (v != label) {
          const float x[1] = {to_float(row[v])};
          a = join_values(a, x, c);
        }
      });
  a = warp_join(a, c);
  const int warps = blockDim.x >> 5;
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = a;
  __syncthreads();
  a = part[0];
  for (int w = 1; w < warps; ++w) a = join(a, part[w], c);
  return a;
}

// grad = k (onehot - p): `neg` = -k / s, `at_label` = k rest / s.  Without `live` zeros.
template <typename T>
__device__ __forceinline__ void write_gradient(const T *row, T *grad, int n_classes, int label, float c, float top,
                                               float neg, float at_label, bool live) {
  constexpr int N = Vec<T>::n;
  const bool same = misalignment(row) == misalignment(grad);
  const float at = shift_of(top);
  auto one = [&](float x, int v) { return v == label ? at_label : neg * exp2_fast(c * (x - at)); };
  for_row(
      grad, n_classes,
      [&](int v) {
        float x[N];
        if (!live) {
#pragma unroll
          for (int i = 0; i < N; ++i) x[i] = 0.f;
        } else {
          if (same) {
            Vec<T>::unpack(*reinterpret_cast<const uint4 *>(row + v), x);
          } else {
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = to_float(row[v + i]);
          }
#pragma unroll
          for (int i = 0; i < N; ++i) x[i] = one(x[i], v + i);
        }
        *reinterpret_cast<uint4 *>(grad + v) = Vec<T>::pack(x);
      },
      [&](int v) { grad[v] = from_float<T>(live ? one(to_float(row[v]), v) : 0.f); });
}

// Reads the row a second time for the gradient.
template <typename T>
__global__ void __launch_bounds__(kRowThreads) policy_kernel(const PolicyArgs a) {
  pdl_sync();
  __shared__ Sum part[kRowThreads / 32];
  __shared__ float out[2];  // neg, at_label
  const int r = blockIdx.x, label = a.actions[r];
  const T *row = static_cast<const T *>(a.logits) + (size_t)r * a.ld;
  T *grad = a.grad ? static_cast<T *>(a.grad) + (size_t)r * a.ld_grad : nullptr;
  bool live = label >= 0 && label < a.n_classes && (!a.weight || a.weight[r] != 0.f);
  float logp = 0.f, loss = 0.f, top = 0.f;
  if (live) {
    const float x_y = to_float(row[label]);
    const Row stat(block_sum(row, a.n_classes, label, a.c, part), x_y, a.c);
    top = stat.top;
    live = !stat.nothing();
    if (threadIdx.x == 0) {
      float k = 0.f;
      if (live) policy_terms(a, stat, r, logp, loss, k);
      const float s = stat.rest + stat.e_y;
      out[0] = -k / s;
      out[1] = k * (stat.rest / s);
      if (k == 0.f) out[0] = out[1] = 0.f;
    }
    __syncthreads();
    live = live && !(out[0] == 0.f && out[1] == 0.f);
  }
  if (threadIdx.x == 0) {
    if (a.logp) a.logp[r] = logp;
    a.row_loss[r] = loss;
  }
  if (grad) write_gradient(row, grad, a.n_classes, label, a.c, top, live ? out[0] : 0.f, live ? out[1] : 0.f, live);
}

// Sums of row_loss over the partitions, one thread block each, in fp64 and a fixed order.
__global__ void __launch_bounds__(256) partition_sum_kernel(const float *row_loss, int rows, long long each,
                                                            float *loss) {
  pdl_sync();
  __shared__ double part[256];
  const long long first = blockIdx.x * each, last = min((long long)rows, first + each);
  double s = 0.0;
  for (long long r = first + threadIdx.x; r < last; r += 256) s += (double)row_loss[r];
  part[threadIdx.x] = s;
  __syncthreads();
#pragma unroll
  for (int o = 128; o > 0; o >>= 1) {
    if ((int)threadIdx.x < o) part[threadIdx.x] += part[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) loss[blockIdx.x] = (float)part[0];
}

// ---- preference loss: statistics of every row, then pairs, then gradients

struct Stat {  // of a row, 32 bytes
  double logp;       // of the label
  float top, inv_s;  // max, 1 / s
  float rest;        // 1 - p_y
  float k;           // factor of the gradient, written for the pair
  int live, pad;
};

struct PreferenceArgs {
  const void *logits;
  void *grad;
  long long ld, ld_grad;
  int rows, pairs, n_classes, length_mean;
  const int *labels;
  const long long *begin;
  const float *ref_logp, *pair_weight;
  float *seq_logp, *pair_loss;
  Stat *stat;
  float c;
  double scale, beta, smooth;
};

__device__ __forceinline__ int row_bound(const PreferenceArgs &a, int s) {
  const long long b = a.begin[s];
  return b < 0 ? 0 : b > a.rows ? a.rows : (int)b;
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads) row_stat_kernel(const PreferenceArgs a) {
  pdl_sync();
  __shared__ Sum part[kRowThreads / 32];
  const int r = blockIdx.x;
  if (r < row_bound(a, 0) || r >= row_bound(a, 2 * a.pairs)) return;
  const int label = a.labels[r];
  const T *row = static_cast<const T *>(a.logits) + (size_t)r * a.ld;
  Stat st = {};
  if (label >= 0 && label < a.n_classes) {
    const float x_y = to_float(row[label]);
    const Row stat(block_sum(row, a.n_classes, label, a.c, part), x_y, a.c);
    if (!stat.nothing()) {
      const float s = stat.rest + stat.e_y;
      st.live = 1;
      st.top = stat.top;
      st.inv_s = 1.f / s;
      st.rest = stat.rest / s;
      if (threadIdx.x == 0) st.logp = stat.logp(a.c);
    }
  }
  if (threadIdx.x == 0) a.stat[r] = st;
}

__device__ __forceinline__ double log_sigmoid(double x) { return fmin(x, 0.0) - log1p(exp(-fabs(x))); }
__device__ __forceinline__ double sigmoid(double x) {
  const double e = exp(-fabs(x));
  return (x >= 0.0 ? 1.0 : e) / (1.0 + e);
}

// One thread block per pair.
__global__ void __launch_bounds__(256) pair_kernel(const PreferenceArgs a) {
  pdl_sync();
  __shared__ double sum[2][8];
  __shared__ int count[2][8];
  const int q = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int first[2], last[2];
  double lp[2], n[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    first[h] = row_bound(a, 2 * q + h);
    last[h] = row_bound(a, 2 * q + h + 1);
    double s = 0.0;
    int c = 0;
    for (int r = first[h] + (int)threadIdx.x; r < last[h]; r += 256) {
      const Stat &st = a.stat[r];
      if (st.live) { s += st.logp; ++c; }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      s += __shfl_xor_sync(0xffffffffu, s, o);
      c += __shfl_xor_sync(0xffffffffu, c, o);
    }
    if (lane == 0) { sum[h][warp] = s; count[h][warp] = c; }
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    double s = 0.0;
    int c = 0;
    for (int w = 0; w < 8; ++w) { s += sum[h][w]; c += count[h][w]; }
    n[h] = a.length_mean && c > 1 ? (double)c : 1.0;
    lp[h] = s / n[h];
  }
  const double x = a.beta * ((lp[0] - (double)a.ref_logp[2 * q]) - (lp[1] - (double)a.ref_logp[2 * q + 1]));
  const double w = a.pair_weight ? (double)a.pair_weight[q] : 1.0;
  const double slope = a.beta * w * a.scale * (a.smooth * sigmoid(x) - (1.0 - a.smooth) * sigmoid(-x));
  if (threadIdx.x == 0) {
    a.seq_logp[2 * q] = (float)lp[0];
    a.seq_logp[2 * q + 1] = (float)lp[1];
    a.pair_loss[q] = (float)(-w * ((1.0 - a.smooth) * log_sigmoid(x) + a.smooth * log_sigmoid(-x)));
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float k = (float)((h ? -slope : slope) / n[h]);
    for (int r = first[h] + (int)threadIdx.x; r < last[h]; r += 256) a.stat[r].k = k;
  }
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads) row_gradient_kernel(const PreferenceArgs a) {
  pdl_sync();
  const int r = blockIdx.x;
  if (r < row_bound(a, 0) || r >= row_bound(a, 2 * a.pairs)) return;
  const Stat st = a.stat[r];
  const bool live = st.live && st.k != 0.f;
  write_gradient(static_cast<const T *>(a.logits) + (size_t)r * a.ld, static_cast<T *>(a.grad) + (size_t)r * a.ld_grad,
                 a.n_classes, live ? a.labels[r] : -1, a.c, st.top, -st.k * st.inv_s, st.k * st.rest, live);
}

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// What both entry points ask of the logits and their gradient.
bool logits_ok(long long rows, int n_classes, int dtype, double scale, const void *logits, long long ld, const void *grad,
               long long ld_grad) {
  if (rows < 0 || rows > 0x7fffffffll || n_classes < 1 || (dtype != NGC_F32 && dtype != NGC_BF16)) return false;
  if (!(scale > 0.0) || !std::isfinite(scale) || !((float)(scale * 1.4426950408889634) > 0.f) ||
      !std::isfinite((float)(scale * 1.4426950408889634)))
    return false;
  const size_t e = dtype == NGC_F32 ? 4 : 2;
  if (ld < n_classes || ld > (1ll << 40) || (rows > 0 && !logits) || !aligned(logits, e)) return false;
  if (grad && (ld_grad < n_classes || ld_grad > (1ll << 40) || !aligned(grad, e))) return false;
  return !(grad == logits && grad && ld != ld_grad);
}

}  // namespace
}  // namespace ngc

extern "C" {

int ngc_policy_loss(const ngc_policy_loss_t *cfg, const void *logits, int64_t ld, const int32_t *actions,
                    const float *old_logp, const float *ref_logp, const float *advantage, const float *weight,
                    void *dlogits, int64_t ld_grad, float *logp, float *row_loss, float *loss, void *cuda_stream) {
  using namespace ngc;
  if (!cfg || !logits_ok(cfg->rows, cfg->n_classes, cfg->dtype, cfg->scale, logits, ld, dlogits, ld_grad))
    return NGC_ERR_INVALID;
  if (!(cfg->clip_low >= 0.0 && cfg->clip_low <= 1.0) || !(cfg->clip_high >= 0.0) || !std::isfinite(cfg->clip_high) ||
      !(cfg->kl_coef >= 0.0) || !std::isfinite(cfg->kl_coef) || cfg->rows_per_partition < 1)
    return NGC_ERR_INVALID;
  if (cfg->rows == 0) return NGC_OK;
  if (!actions || !old_logp || !advantage || !row_loss) return NGC_ERR_INVALID;
  for (const void *p : {(const void *)actions, (const void *)old_logp, (const void *)ref_logp, (const void *)advantage,
                        (const void *)weight, (const void *)logp, (const void *)row_loss, (const void *)loss})
    if (!aligned(p, 4)) return NGC_ERR_INVALID;
  PolicyArgs a;
  a.logits = logits; a.grad = dlogits; a.ld = ld; a.ld_grad = ld_grad;
  a.rows = (int)cfg->rows; a.n_classes = cfg->n_classes;
  a.actions = actions; a.old_logp = old_logp; a.ref_logp = cfg->kl_coef > 0.0 ? ref_logp : nullptr;
  a.advantage = advantage; a.weight = weight; a.logp = logp; a.row_loss = row_loss;
  a.c = (float)(cfg->scale * 1.4426950408889634);
  a.scale = cfg->scale; a.low = 1.0 - cfg->clip_low; a.high = 1.0 + cfg->clip_high; a.kl = cfg->kl_coef;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = cfg->dtype == NGC_F32
                            ? launch_k(policy_kernel<float>, a.rows, kRowThreads, 0, stream, a)
                            : launch_k(policy_kernel<__nv_bfloat16>, a.rows, kRowThreads, 0, stream, a);
  if (e != cudaSuccess) return NGC_ERR_CUDA;
  if (loss) {
    const long long each = cfg->rows_per_partition, parts = (a.rows - 1) / each + 1;
    if (launch_k(partition_sum_kernel, (unsigned)parts, 256, 0, stream, (const float *)row_loss, a.rows, each, loss) !=
        cudaSuccess)
      return NGC_ERR_CUDA;
  }
  return NGC_OK;
}

size_t ngc_preference_workspace_bytes(int64_t rows, int32_t pairs) {
  (void)pairs;
  return rows < 0 ? 0 : ((size_t)rows + 1) * sizeof(ngc::Stat);
}

int ngc_preference_loss(const ngc_preference_loss_t *cfg, const void *logits, int64_t ld, const int32_t *labels,
                        const int64_t *seq_begin, const float *ref_logp, const float *pair_weight, void *dlogits,
                        int64_t ld_grad, float *seq_logp, float *pair_loss, void *workspace, size_t workspace_bytes,
                        void *cuda_stream) {
  using namespace ngc;
  if (!cfg || !logits_ok(cfg->rows, cfg->n_classes, cfg->dtype, cfg->scale, logits, ld, dlogits, ld_grad))
    return NGC_ERR_INVALID;
  if (cfg->pairs < 0 || cfg->pairs > 0x3ffffffe || !std::isfinite(cfg->beta) ||
      !(cfg->label_smoothing >= 0.0 && cfg->label_smoothing <= 1.0))
    return NGC_ERR_INVALID;
  if (cfg->pairs == 0) return NGC_OK;
  if ((cfg->rows > 0 && !labels) || !seq_begin || !ref_logp || !seq_logp || !pair_loss || !workspace ||
      !aligned(workspace, 16) || workspace_bytes < ngc_preference_workspace_bytes(cfg->rows, cfg->pairs) ||
      !aligned(seq_begin, 8))
    return NGC_ERR_INVALID;
  for (const void *p : {(const void *)labels, (const void *)ref_logp, (const void *)pair_weight, (const void *)seq_logp,
                        (const void *)pair_loss})
    if (!aligned(p, 4)) return NGC_ERR_INVALID;
  PreferenceArgs a;
  a.logits = logits; a.grad = dlogits; a.ld = ld; a.ld_grad = ld_grad;
  a.rows = (int)cfg->rows; a.pairs = cfg->pairs; a.n_classes = cfg->n_classes; a.length_mean = cfg->length_mean != 0;
  a.labels = labels; a.begin = reinterpret_cast<const long long *>(seq_begin);
  a.ref_logp = ref_logp; a.pair_weight = pair_weight; a.seq_logp = seq_logp; a.pair_loss = pair_loss;
  a.stat = static_cast<Stat *>(workspace);
  a.c = (float)(cfg->scale * 1.4426950408889634);
  a.scale = cfg->scale; a.beta = cfg->beta; a.smooth = cfg->label_smoothing;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const bool f32 = cfg->dtype == NGC_F32;
  if (a.rows > 0 && launch_k(f32 ? row_stat_kernel<float> : row_stat_kernel<__nv_bfloat16>, a.rows, kRowThreads, 0, stream,
                             a) != cudaSuccess)
    return NGC_ERR_CUDA;
  if (launch_k(pair_kernel, a.pairs, 256, 0, stream, a) != cudaSuccess) return NGC_ERR_CUDA;
  if (a.rows > 0 && a.grad &&
      launch_k(f32 ? row_gradient_kernel<float> : row_gradient_kernel<__nv_bfloat16>, a.rows, kRowThreads, 0, stream, a) !=
          cudaSuccess)
    return NGC_ERR_CUDA;
  return NGC_OK;
}

}  // extern "C"

// ngc_policy_loss and ngc_preference_loss: losses on rows of logits and their gradients.
//
// One row.  With x its logits and c = scale log2(e), the probabilities are p_v = 2^(c x_v - t) / s for any shift t; t is
// the largest c x, rounded up to a whole number, so a term costs a fused multiply-add or two (rounding only the small
// result) and one 2^x.  The label's term is kept out of the sum: s = rest + e_y.  Then log p_y = ln2 (c x_y - t) - ln(rest + e_y), and
// 1 - p_y = rest / s is exact where p_y is close to one.  Threads sum in a fixed order relative to their warp's
// maximum and are then joined.  Rows whose largest c x is 2^18 or more from zero (a mask in every class, or -infinity in
// every class) take a slower way that subtracts the largest logit before it multiplies.
// Of what happens once per row, the logarithm and the differences between log-probabilities are pairs of floats; ratio,
// clip and KL term are formed from them in single ones, each within a few units in its last place.  Sums over the rows of
// a sequence, and what follows from them, are in fp64.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <cfloat>
#include <cmath>
#include <initializer_list>

#include "ngc_device.h"
#include "ngc_f32x2.cuh"
#include "ngc_pdl.cuh"

namespace ngc {
namespace {

constexpr float kNegInf = -INFINITY;
constexpr float kFloor = -0x1p126f;  // shift of a set without any logit
// Rows with a shift from here on are left to the slow_ functions.  x times the 16 bits of Coef::big misses c x by up to
// 2^-16 of it, which the sum with the shift rounds to 2^-22 here and to more beyond; from 2^24 on the shift itself is no
// longer every whole number.  Such rows are read three times, one element per load: 8192 rows of 32000 bf16 logits around 1e6
// 1.12 ms instead of 0.17, 102400 of 256 fp32 124 us instead of 35.
constexpr float kSlow = 0x1p18f;

// Relative error at most 2^-22, measured 1.4e-7, for x below -1 on average 5.0e-8 too low (4.95e-8 to 5.1e-8 by octave down
// to -17, for x from -1 to 0 2.2e-8), which sums over thousands of rows would show: label_logp corrects that; whole powers
// are exact.  Results below 2^-126 become zero.
constexpr float kExp2Low = 5.0e-8f;
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Within one unit in the last place (it only scales gradients, of which each is rounded anyway).
__device__ __forceinline__ float reciprocal(float x) {
  float r;
  asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// 16 bytes of logits.
template <typename T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int n = 4;
  static constexpr uint32_t neg_inf = 0xff800000u;
};
template <>
struct Vec<__nv_bfloat16> {
  static constexpr int n = 8;
  static constexpr uint32_t neg_inf = 0xff80ff80u;
};
__device__ __forceinline__ uint32_t word(const uint4 &q, int i) { return i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w; }
// Elements 2 i and 2 i + 1 of a vector.
__device__ __forceinline__ void pair_of(float, const uint4 &q, int i, float &a, float &b) {
  a = __uint_as_float(word(q, 2 * i));
  b = __uint_as_float(word(q, 2 * i + 1));
}
__device__ __forceinline__ void pair_of(__nv_bfloat16, const uint4 &q, int i, float &a, float &b) {
  a = __uint_as_float(word(q, i) << 16);  // bf16 is the upper half of a float
  b = __uint_as_float(word(q, i) & 0xffff0000u);
}
__device__ __forceinline__ uint32_t max_words(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// The largest element of NV vectors.
template <int NV>
__device__ __forceinline__ float max_of(float, const uint4 (&q)[NV]) {
  float m = kNegInf;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) m = fmaxf(m, __uint_as_float(word(q[j], i)));
  return m;
}
template <int NV>
__device__ __forceinline__ float max_of(__nv_bfloat16, const uint4 (&q)[NV]) {
  uint32_t w[4] = {q[0].x, q[0].y, q[0].z, q[0].w};
#pragma unroll
  for (int j = 1; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = max_words(w[i], word(q[j], i));
  const uint32_t m = max_words(max_words(w[0], w[1]), max_words(w[2], w[3]));
  return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
}
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// The compiler keeps nothing that it worked out from these registers, and takes them for new values.
__device__ __forceinline__ void pin(uint4 &q) { asm volatile("" : "+r"(q.x), "+r"(q.y), "+r"(q.z), "+r"(q.w)); }
// x = (x & ~mask) | in where w == at.
__device__ __forceinline__ void drop_bits(uint32_t &x, int w, int at, uint32_t mask, uint32_t in) {
  asm("{\n\t.reg .pred p;\n\tsetp.eq.s32 p, %1, %2;\n\t@p lop3.b32 %0, %0, %3, %4, 0xba;\n\t}"
      : "+r"(x) : "r"(w), "r"(at), "r"(mask), "r"(in));
}
// Takes element `i` of vector `at` out of the set (word by word: an index into registers would put them all into memory).
template <typename T, int NV>
__device__ __forceinline__ void drop_element(uint4 (&q)[NV], int at, int i) {
  constexpr int per_word = sizeof(T) == 2 ? 2 : 1;
  const uint32_t mask = per_word == 1 ? 0xffffffffu : i % 2 ? 0xffff0000u : 0x0000ffffu, in = Vec<T>::neg_inf & mask;
  const int w = at * 4 + i / per_word;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    drop_bits(q[j].x, w, 4 * j, mask, in);
    drop_bits(q[j].y, w, 4 * j + 1, mask, in);
    drop_bits(q[j].z, w, 4 * j + 2, mask, in);
    drop_bits(q[j].w, w, 4 * j + 3, mask, in);
  }
}

// A row as whole 16-byte vectors and the loose elements before and after them (at most 2 N - 2), which lanes or
// threads below `loose` take one each.
template <typename T>
struct Layout {
  static constexpr int N = Vec<T>::n;
  int head, vecs, loose;
  __device__ __forceinline__ Layout(const T *row, int n_classes) {
    head = min(n_classes, (int)((0u - (unsigned)(reinterpret_cast<uintptr_t>(row) / sizeof(T))) % N));
    vecs = (n_classes - head) / N;
    loose = n_classes - vecs * N;
  }
  __device__ __forceinline__ int loose_at(int i) const { return i < head ? i : vecs * N + i; }
  // which vector holds an element (none: negative), and which loose element it is (none: negative)
  __device__ __forceinline__ int vec_of(int v) const { return v >= head && v - head < vecs * N ? (v - head) / N : -1; }
  __device__ __forceinline__ int loose_of(int v) const {
    return v < head ? v : v - head >= vecs * N ? v - vecs * N : -1;
  }
};
// Whether two rows have the same place between 16-byte boundaries.
template <typename T>
__device__ __forceinline__ bool same_alignment(const T *a, const T *b) {
  return ((reinterpret_cast<uintptr_t>(a) ^ reinterpret_cast<uintptr_t>(b)) & 15u) == 0;
}

// The sum s of 2^(c x - t) over a set of logits, NaN or finite.  A set of nothing but masks (-1e10 and the like) has a shift
// so far from zero that its rounding is hundreds, and powers anywhere between 0 and infinity.  Next to any logit that
// counts its share is zero as long as it is not infinite; a row of nothing else is left to the slow_ functions.
struct Sum {
  float t, s;
};
__device__ __forceinline__ float no_infinity(float s) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(s), "f"(FLT_MAX));
  return r;
}
// c = scale log2(e) in two parts: with c rounded to fp32 alone, a sequence's log-probability would be off by up to 6e-8 of
// the sum of its logits' distances.  For the powers the first part has 16 bits, so that what the second one adds is many
// units in the last place of the sum; the rest of a whole fp32 would mostly be rounded away, always to the same side (the
// mean error of log p over 631 classes was 2.3e-8).  Both parts are rounded towards zero or positive: -infinity stays that.
struct Coef {
  float hi, lo;      // 24 and 24 bits
  float big, small;  // 16 and 24 bits
  float lo_share;    // lo / hi
  float scale;
  // What powers with the first part alone lack next to a shift t: 2^(lo x) where hi x = t.
  __device__ __forceinline__ float lacking(float t) const { return exp2_fast(t * lo_share); }
  __device__ __forceinline__ float power(float x, float minus_t) const { return fmaf(x, small, fmaf(x, big, minus_t)); }
};
Coef coef_of(double scale) {
  const double c = scale * 1.4426950408889634;
  int e;
  const double f = std::frexp(c, &e);
  const float hi = (float)std::ldexp(std::floor(std::ldexp(f, 24)), e - 24);
  const float big = (float)std::ldexp(std::floor(std::ldexp(f, 16)), e - 16);
  const auto rest = [c](float part) {  // (not zero: -infinity times zero would be NaN)
    const float r = (float)(c - (double)part);
    return r > 0.f ? r : std::fmax(part * 0x1p-60f, FLT_TRUE_MIN);
  };
  // (a coefficient of few digits, below 1e-30, has shifts of 1 and 2 whatever its second part)
  return {hi, rest(hi), big, rest(big), hi > 1e-30f ? rest(hi) / hi : 0.f, (float)scale};
}
// The shift for a set of logits: whole numbers, so that bringing sums together multiplies by powers of two, one above the
// least, so that all powers are taken below -1 (see exp2_fast).
__device__ __forceinline__ float shift_of(float max_logit, const Coef &c) { return fmaxf(ceilf(c.hi * max_logit) + 1.f, kFloor); }
__device__ __forceinline__ float warp_max(float m) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(m));
  return r;
}
__device__ __forceinline__ float warp_sum(float s) {
#pragma unroll
  for (int o = 16; o > 0; o /= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}
__device__ __forceinline__ Sum warp_join(const Sum &a) {
  const float t = warp_max(a.t);
  return {t, no_infinity(warp_sum(a.s * exp2_fast(a.t - t)))};
}

// 2^(c x - t) of the elements of a vector; Fine: with both parts of c.
template <typename T, bool Fine>
__device__ __forceinline__ void exp_vec(const uint4 &q, const Coef &c, float minus_t, f32x2 (&e)[Vec<T>::n / 2]) {
#pragma unroll
  for (int i = 0; i < Vec<T>::n / 2; ++i) {
    float a, b;
    pair_of(T(), q, i, a, b);
    const f32x2 x = pack2(a, b);
    f32x2 u = mad2(x, Fine ? pack2(c.big, c.big) : pack2(c.hi, c.hi), pack2(minus_t, minus_t));
    if (Fine) u = mad2(x, pack2(c.small, c.small), u);
    unpack2(u, a, b);
    e[i] = pack2(exp2_fast(a), exp2_fast(b));
  }
}
// `start` and the sum of 2^(c x - t) over NV vectors; the powers stay in `e`.
template <typename T, int NV>
__device__ __forceinline__ float held_sum(const uint4 (&q)[NV], float start, const Coef &c, float t,
                                          f32x2 (&e)[NV][Vec<T>::n / 2]) {
  f32x2 s = pack2(start, 0.f);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    exp_vec<T, true>(q[j], c, -t, e[j]);
#pragma unroll
    for (int i = 0; i < Vec<T>::n / 2; ++i) s = add2(s, e[j][i]);
  }
  float lo, hi;
  unpack2(s, lo, hi);
  return lo + hi;
}
template <typename T, int NV>
__device__ __forceinline__ float held_sum(const uint4 (&q)[NV], float start, const Coef &c, float t) {
  f32x2 e[NV][Vec<T>::n / 2];
  return held_sum<T, NV>(q, start, c, t, e);
}

// A number as the sum of two floats, the second a few units in the last place of the first, or of what it was made of.
struct Pair {
  float hi, lo;
};
__device__ __forceinline__ Pair two_sum(float a, float b) {  // exact (Knuth)
  const float s = __fadd_rn(a, b), t = __fsub_rn(s, a);
  return {s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t))};
}
__device__ __forceinline__ Pair add(const Pair &a, float b) {
  const Pair s = two_sum(a.hi, b);
  return {s.hi, s.lo + a.lo};
}
// With all that fits in the first.
__device__ __forceinline__ Pair tidy(const Pair &a) {
  const float s = __fadd_rn(a.hi, a.lo);
  return {s, __fsub_rn(a.lo, __fsub_rn(s, a.hi))};
}

// a - b; infinities keep their meaning (an action of probability 0 now, before or under the reference).
__device__ __forceinline__ Pair minus(const Pair &a, float b) {
  const Pair r = add(a, -b);
  return fabsf(r.hi) < INFINITY ? r : Pair{a.hi - b, 0.f};
}

// log p of a label: d = log2 of its term, as a pair, e_y = 2^d, and rest, the sum of the other terms.  Within about 4e-8
// (and a few units of 2^-48 of the parts it is made of): fp64 would need some 2000 cycles here, while the row's
// threads wait.  `far`: scale times what the label's logit is below the others', for a logit whose d would be 1e30 or infinite
// (the type's lowest value).  `low`: how much of rest + e_y has been through exp2_fast, as often as it has.
__device__ __forceinline__ Pair label_logp(const Pair &d, float e_y, float rest, float low, float far) {
  constexpr float kLn2Hi = 0.693147182464599609375f, kLn2Lo = -1.904654323148236e-9f;
  // p_y above 8/9: from what it lacks of one, so that a small log p is as good as a large one
  if (rest < 0.125f * e_y) return {-log1pf(__fdividef(rest, e_y)), -kExp2Low * __fdividef(low, rest + e_y)};
  const float p = kLn2Hi * d.hi;
  if (!(fabsf(p) <= 1e30f)) return {far - logf(rest + e_y), 0.f};  // infinities and NaN keep their meaning
  const float pe = fmaf(kLn2Hi, d.hi, -p) + (kLn2Hi * d.lo + kLn2Lo * d.hi);
  // - log s, s = f 2^e with f in [3/4, 3/2): e ln 2 in two parts, the first with 13 bits, so that its product is exact.
  // Where p_y is close to one, s is a little over one, and both halves of it tell how much.
  const Pair s = two_sum(rest, e_y);
  const int e = ((__float_as_int(s.hi) - 0x3f400000) >> 23);
  const float f = __int_as_float(__float_as_int(s.hi) - (e << 23));
  const float log_f = log1pf(f - 1.f) + __fdividef(fmaf(kExp2Low, low, s.lo), s.hi);
  const float ef = (float)e;
  Pair r = add(two_sum(p, -ef * 0.693115234375f), pe);
  r = add(r, -log_f);
  return add(r, -ef * 3.194618495e-5f);
}

// What the sum over the other classes and the label's logit make of a row.
struct Row {
  float t, e_y, rest, low;
  Pair d;
  __device__ __forceinline__ Row(const Sum &others, float x_y, const Coef &c) {
    const float p = c.hi * x_y;
    t = fmaxf(others.t, p);
    rest = others.s * exp2_fast(others.t - t);
    d = tidy(add(two_sum(p, -t), fmaf(c.hi, x_y, -p) + c.lo * x_y));
    if (!(p >= kFloor)) d = {p - t, 0.f};  // (-infinity, NaN)
    // the likeliest class: d is what t has lost of c x_y, and e_y as exact as the difference to one has to be
    const bool near = fabsf(d.hi) < 0x1p-12f;
    e_y = near ? fmaf(d.hi, 0.693147182f, 1.f) : exp2_fast(d.hi);
    low = near ? 2.f * rest : rest + e_y;
  }
  __device__ __forceinline__ bool slow() const { return !(fabsf(t) < kSlow); }
  __device__ __forceinline__ Pair logp(float x_y, const Coef &c) const { return label_logp(d, e_y, rest, low, c.scale * x_y); }
};

// Gradient of a row: k (onehot - p) = factor 2^(c x - t), and at_label = k rest / s for the label.
struct Gradient {
  float t, factor, at_label;
  __device__ __forceinline__ bool zero() const { return factor == 0.f && at_label == 0.f; }
};
template <bool Exact>
__device__ __forceinline__ Gradient gradient_of(float k, float t, float rest, float e_y) {
  // Exact: true divisions.  Where bf16 logits are unpacked again for the gradient, their branches also keep the compiler
  // from spreading the row's scalars over the loops around them, which took 8 % longer on rows of 32000 logits (11 % on
  // 4000); where the powers are kept, or in fp32, the reciprocal is shorter (2000 fp32 logits: 131 against 139 us).
  const float s = rest + e_y;
  if (k == 0.f) return {t, 0.f, 0.f};
  if (!Exact) {
    const float inv = k * reciprocal(s);
    return {t, -inv, inv * rest};
  }
  return {t, -k / s, k * (rest / s)};
}
// factor * e for the powers of a vector.
__device__ __forceinline__ uint4 scaled(float, const f32x2 (&e)[2], float factor) {
  float x[4];
#pragma unroll
  for (int i = 0; i < 2; ++i) unpack2(mul2(e[i], pack2(factor, factor)), x[2 * i], x[2 * i + 1]);
  return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
__device__ __forceinline__ uint4 scaled(__nv_bfloat16, const f32x2 (&e)[4], float factor) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a, b;
    unpack2(mul2(e[i], pack2(factor, factor)), a, b);
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    w[i] = *reinterpret_cast<const uint32_t *>(&p);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// A vector of the gradient (`same`: the address is aligned for it).
template <typename T>
__device__ __forceinline__ void store_vec(T *to, bool same, const uint4 &g) {
  if (same) {
    *reinterpret_cast<uint4 *>(to) = g;
    return;
  }
#pragma unroll
  for (int i = 0; i < Vec<T>::n / 2; ++i) {
    float a, b;
    pair_of(T(), g, i, a, b);
    to[2 * i] = from_float<T>(a);
    to[2 * i + 1] = from_float<T>(b);
  }
}

// ---- policy loss

struct PolicyArgs {
  const void *logits;
  void *grad;  // may be null
  long long ld, ld_grad;
  int rows, n_classes;
  const int *actions;
  const float *old_logp, *ref_logp, *advantage, *weight;
  float *logp, *row_loss;
  float *loss;  // partitions of one row: the same values again; else null
  Coef c;
  float scale, low, high, kl;
};
__device__ __forceinline__ void put_row(const PolicyArgs &a, long long row, float logp, float loss) {
  if (a.logp) a.logp[row] = logp;
  a.row_loss[row] = loss;
  if (a.loss) a.loss[row] = loss;
}

// A row's own numbers.
struct Sample {
  int label;
  float old_logp, ref_logp, advantage, weight;
  bool live;
};
__device__ __forceinline__ Sample sample_of(const PolicyArgs &a, int row) {
  Sample s;
  s.label = a.actions[row];
  s.weight = a.weight ? a.weight[row] : 1.f;
  s.old_logp = a.old_logp[row];
  s.advantage = a.advantage[row];
  s.ref_logp = a.ref_logp ? a.ref_logp[row] : 0.f;
  s.live = s.label >= 0 && s.label < a.n_classes && s.weight != 0.f;
  return s;
}

// e^d - 1 - d, and e^d - 1 in `q`, for d up to 88.  The difference of the two would keep few digits of a small d (at 1e-4 it was
// off by 4e-4 of itself, at 1e-6 by a tenth): d^2 / 2 + ... + d^11 / 11! up to 1, within 1e-6 either way.
__device__ __forceinline__ float exp_minus_line(float d, float &q) {
  constexpr float c[] = {1.f / 39916800.f, 1.f / 3628800.f, 1.f / 362880.f, 1.f / 40320.f, 1.f / 5040.f,
                         1.f / 720.f,      1.f / 120.f,     1.f / 24.f,     1.f / 6.f,     0.5f};
  float v = c[0];
#pragma unroll
  for (int i = 1; i < 10; ++i) v = fmaf(d, v, c[i]);
  v = d * d * v;
  q = d + v;
  if (!(fabsf(d) < 1.f)) {
    q = expf(d) - 1.f;
    v = q - d;
  }
  return v;
}

// 2^92, and its logarithm in two parts.
constexpr float kFar = 0x1p92f, kFarLog = 0x1.fe28040p+5f, kFarLogLo = 0x1.d0f668p-20f;
// Where the ratio or e^d leaves the range of fp32 (delta or d above 88): both divided by 2^92, which comes back with the weight,
// so that what is finite after the advantage, the weight and kl_coef stays finite (as far as e^150), and an advantage of
// 0 takes the ratio out.  Returns the slope with the weight.
__device__ __forceinline__ float far_terms(const PolicyArgs &a, const Sample &y, const Pair &delta, const Pair &below_ref,
                                           float &loss) {
  const float d = -(below_ref.hi + below_ref.lo);
  const bool far_ratio = delta.hi > 80.f, far_kl = a.ref_logp && d > 80.f;
  const float down = far_ratio ? 1.f / kFar : 1.f, up = y.weight * (far_ratio ? kFar : 1.f);
  const float ratio = far_ratio ? expf(delta.hi - kFarLog) * (1.f + (delta.lo - kFarLogLo)) : expf(delta.hi) * (1.f + delta.lo);
  const float free_ = y.advantage == 0.f && delta.hi < INFINITY ? 0.f : ratio * y.advantage;
  const float held = fminf(fmaxf(ratio, a.low * down), a.high * down) * y.advantage;
  float value = -fminf(free_, held), slope = free_ <= held ? -free_ : 0.f;
  if (free_ != free_) value = slope = free_;
  loss = up * value;
  slope *= up;
  if (a.ref_logp) {
    float q, v;
    if (far_kl)  // (d itself is nothing beside e^d)
      v = q = expf(-below_ref.hi - kFarLog) * (1.f - (below_ref.lo + kFarLogLo));
    else
      v = exp_minus_line(d, q);
    const float kl = y.weight * a.kl * (far_kl ? kFar : 1.f);
    loss = fmaf(kl, v, loss);
    slope = fmaf(-kl, q, slope);
  }
  return slope;
}

// Loss of a live row, its log p, and the factor k of its gradient k (onehot - p).
__device__ __forceinline__ float policy_terms(const PolicyArgs &a, const Pair &lp, const Sample &y, float &logp,
                                              float &loss) {
  const Pair delta = minus(lp, y.old_logp), below_ref = minus(lp, y.ref_logp);
  const float d = -(below_ref.hi + below_ref.lo);
  logp = lp.hi + lp.lo;
  if (__builtin_expect(fmaxf(delta.hi, a.ref_logp ? d : 0.f) > 88.f, 0)) return far_terms(a, y, delta, below_ref, loss) * a.scale;
  const float ratio = expf(delta.hi) * (1.f + delta.lo);
  const float free_ = ratio * y.advantage, held = fminf(fmaxf(ratio, a.low), a.high) * y.advantage;
  float value = -fminf(free_, held), slope = free_ <= held ? -free_ : 0.f;
  if (free_ != free_) value = slope = free_;
  if (a.ref_logp) {
    float q;
    value = fmaf(a.kl, exp_minus_line(d, q), value);
    slope = fmaf(-a.kl, q, slope);
  }
  loss = y.weight * value;
  return y.weight * slope * a.scale;
}

// ---- any row, by subtracting the largest logit first: x - max is finite (or -infinity) for every finite maximum.
// `id` of `n` threads, a warp (part == nullptr) or a block (part: one value per warp, in shared memory).

template <typename F>
__device__ __forceinline__ void for_classes(int n_classes, int label, int id, int n, F f) {
  for (unsigned v = id; v < (unsigned)n_classes; v += n)
    if ((int)v != label) f((int)v);
}
__device__ __forceinline__ float team_max(float m, float *part) {
  m = warp_max(m);
  if (!part) return m;
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
  __syncthreads();
  for (int w = 0; w < (int)(blockDim.x >> 5); ++w) m = fmaxf(m, part[w]);
  return m;
}
__device__ __forceinline__ float team_sum(float s, float *part) {
  s = warp_sum(s);
  if (!part) return s;
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
  __syncthreads();
  s = 0.f;
  for (int w = 0; w < (int)(blockDim.x >> 5); ++w) s += part[w];
  return s;
}
__device__ __forceinline__ float slow_power(float below, float c, float c_lo) {
  return exp2_fast(fmaf(below, c, below * c_lo));
}
struct SlowRow {
  float top, e_y, rest, far;  // far: see label_logp
  Pair d;
  bool nothing;  // all logits -infinity
  __device__ __forceinline__ Pair logp() const { return label_logp(d, e_y, rest, d.hi == 0.f ? rest : rest + e_y, far); }
};
template <typename T>
__device__ __noinline__ SlowRow slow_stats(const T *row, int n_classes, int label, float c, float c_lo, float scale, int id,
                                           int n, float *part) {
  SlowRow r;
  const float x_y = to_float(row[label]);
  float m = x_y;
  bool nan = m != m;
  for_classes(n_classes, label, id, n, [&](int v) {
    const float x = to_float(row[v]);
    m = fmaxf(m, x);
    nan |= x != x;
  });
  r.top = team_max(m, part);
  nan = team_sum(nan ? 1.f : 0.f, part) > 0.f;
  r.nothing = r.top == kNegInf && !nan;
  if (r.nothing) return r;
  float s = nan ? NAN : 0.f;
  for_classes(n_classes, label, id, n, [&](int v) { s += slow_power(to_float(row[v]) - r.top, c, c_lo); });
  r.rest = team_sum(s, part);
  const Pair diff = two_sum(x_y, -r.top);
  const float p = c * diff.hi;
  r.d = {p, fmaf(c, diff.hi, -p) + (c * diff.lo + c_lo * diff.hi)};
  if (!(fabsf(p) <= 1e30f)) r.d = {c * (x_y - r.top), 0.f};
  r.e_y = exp2_fast(r.d.hi);
  const float below = x_y - r.top;
  r.far = fabsf(below) < INFINITY ? scale * below : fmaf(scale, x_y, -scale * r.top);
  return r;
}
template <typename T>
__device__ __noinline__ void slow_gradient(const T *row, T *grad, int n_classes, int label, float c, float c_lo, float top,
                                           float neg, float at_label, bool live, int id, int n) {
  for_classes(n_classes, label, id, n, [&](int v) {
    grad[v] = from_float<T>(live ? neg * slow_power(to_float(row[v]) - top, c, c_lo) : 0.f);
  });
  if (id == 0 && label >= 0 && label < n_classes) grad[label] = from_float<T>(live ? at_label : 0.f);
}
template <typename T>
__device__ __forceinline__ void slow_policy_row(const PolicyArgs &a, int r, const Sample &y, int id, int n, float *part) {
  const T *row = static_cast<const T *>(a.logits) + (size_t)r * a.ld;
  const SlowRow s = slow_stats(row, a.n_classes, y.label, a.c.hi, a.c.lo, a.c.scale, id, n, part);
  float logp = 0.f, loss = 0.f, k = 0.f;
  if (!s.nothing) k = policy_terms(a, s.logp(), y, logp, loss);
  if (id == 0) put_row(a, r, logp, loss);
  if (part) __syncthreads(); else __syncwarp();  // everybody has read the label's logit
  const float sum = s.rest + s.e_y;
  if (a.grad)
    slow_gradient(row, static_cast<T *>(a.grad) + (size_t)r * a.ld_grad, a.n_classes, y.label, a.c.hi, a.c.lo, s.top,
                  -k / sum, k * (s.rest / sum), k != 0.f, id, n);
}

// ---- one row for a team of threads (one warp, or a block), kHeld vectors per thread and round

constexpr int kHeld = 8;
template <typename T, int Threads, int Held = kHeld>
struct Team {
  static constexpr int N = Vec<T>::n, kRound = Threads * Held;
  const T *row;
  Layout<T> at;
  int tid, label, vec, rounds;
  int first_round;  // vectors of round 0: the short one, so that the last, which may be held, is a whole one
  bool label_mine;  // this thread has the label's vector, or the label among its loose elements

  __device__ __forceinline__ Team(const T *r, int n_classes, int label_, int tid_)
      : row(r), at(r, n_classes), tid(tid_), label(label_) {
    rounds = max(1, (int)((unsigned)(at.vecs + kRound - 1) / kRound));
    // (a multiple of 8 vectors, 128 bytes, so that the later rounds start where a line does if the row does)
    first_round = min(at.vecs, (at.vecs - (rounds - 1) * kRound + 7) & ~7);
    vec = at.vec_of(label);
    label_mine = vec >= 0 ? (vec - begin_of(round_of(vec))) % Threads == tid : at.loose_of(label) == tid;
  }
  __device__ __forceinline__ int begin_of(int k) const { return k == 0 ? 0 : first_round + (k - 1) * kRound; }
  __device__ __forceinline__ int round_of(int v) const { return v < first_round ? 0 : 1 + (v - first_round) / kRound; }
  // Vectors of round k from this thread's first one on.
  __device__ __forceinline__ int left_in(int k) const { return (k == 0 ? first_round : min(kRound, at.vecs - begin_of(k))) - tid; }
  // Round k, -infinity behind the row's end.
  __device__ __forceinline__ void read(int k, uint4 (&q)[Held]) const {
    const int left = left_in(k);
    const uint4 *const from = reinterpret_cast<const uint4 *>(row + at.head) + tid + begin_of(k);
    if (left > kRound - Threads) {
#pragma unroll
      for (int j = 0; j < Held; ++j) q[j] = from[j * Threads];
    } else {
#pragma unroll
      for (int j = 0; j < Held; ++j) {
        q[j] = make_uint4(Vec<T>::neg_inf, Vec<T>::neg_inf, Vec<T>::neg_inf, Vec<T>::neg_inf);
        if (j * Threads < left) q[j] = from[j * Threads];
      }
    }
  }
  // This thread's loose element; -infinity for none and for the label.
  __device__ __forceinline__ float read_loose() const {
    return tid < at.loose && (vec >= 0 || !label_mine) ? to_float(row[at.loose_at(tid)]) : kNegInf;
  }
  // This thread's sum over the row without the label; the last round stays in `q`.
  __device__ __forceinline__ Sum sum(const Coef &c, float loose, uint4 (&q)[Held]) const {
    Sum s{shift_of(loose, c), 0.f};
    s.s = no_infinity(exp2_fast(c.power(loose, -s.t)));
    for (int k = 0; k < rounds; ++k) {
      read(k, q);
      if (label_mine && vec >= 0 && round_of(vec) == k)
        drop_element<T, Held>(q, (vec - begin_of(k)) / Threads, (unsigned)(label - at.head) % N);
      const float t = fmaxf(s.t, shift_of(max_of(T(), q), c));
      s = {t, no_infinity(s.s * exp2_fast(s.t - t) + held_sum<T, Held>(q, 0.f, c, t))};
    }
    return s;
  }
  // The row's gradient, the youngest round first; `held`: that round is still in `q`.
  __device__ __forceinline__ void write(T *grad, const Gradient &g, const Coef &c, float loose, uint4 (&q)[Held], bool held) const {
    const bool same = same_alignment(row, grad), zero = g.zero();
    constexpr bool kFine = sizeof(T) == 4;  // (bf16: what the second part of c changes within a row is lost in the rounding)
    const float factor = kFine ? g.factor : g.factor * c.lacking(g.t);
    T *const dst = grad + at.head + (size_t)tid * N;
    for (int k = rounds - 1; k >= 0; --k) {
      const int left = left_in(k);
      T *const to = dst + (size_t)begin_of(k) * N;
      if (!zero && !(held && k == rounds - 1)) read(k, q);
#pragma unroll
      for (int j = 0; j < Held; ++j) {
        if (j * Threads < left) {
          uint4 w = make_uint4(0, 0, 0, 0);
          if (!zero) {
            pin(q[j]);  // (unpacked again rather than kept unpacked)
            f32x2 e[N / 2];
            exp_vec<T, kFine>(q[j], c, -g.t, e);
            w = scaled(T(), e, factor);
          }
          store_vec(to + j * Threads * N, same, w);
        }
      }
    }
    if (tid < at.loose) grad[at.loose_at(tid)] = from_float<T>(zero ? 0.f : g.factor * exp2_fast(c.power(loose, -g.t)));
    // the label's own place, by the thread that wrote it (a thread's stores stay in order)
    if (!zero && label_mine) grad[label] = from_float<T>(g.at_label);
  }
};

// Short rows: G lanes of a warp hold one row of up to G NV vectors, so a warp works on 32 / G rows with the same
// instructions (at 256 bf16 classes: 8 rows of 4 lanes).  Up to 32 powers per lane stay in registers for the gradient,
// of more the logits do.  What bounds it is the instructions for the label, the loss and the KL term, 300 per warp
// whatever the rows' length, and latency: 204800 rows of 256 bf16 logits 44.5 us (48 from cold inputs); 4 rows of 8 lanes with their powers
// kept 49.7 us; the same with the loss of a thread block's 16 rows worked out together, a quarter fewer instructions,
// 53.5 us; two rows per team, 64 powers kept and fewer warps, 58-71 us; a whole warp for every row 76 us.
constexpr int kShortWarps = 4;
template <typename T, int G, int NV>
struct ShortRow {
  static constexpr int N = Vec<T>::n, kLoose = (2 * N - 2 + G - 1) / G;
  const T *row;
  Layout<T> at;
  int id, label, vec;
  bool label_mine;  // this lane has the label's vector, or the label among its loose elements
  uint4 q[NV];
  float loose[kLoose];

  // `wanted`: the logits are read (else all of them are -infinity).  `label` may be none: -1.
  __device__ __forceinline__ ShortRow(const T *r, int n_classes, int label_, int id_, bool wanted)
      : row(r), at(r, n_classes), id(id_), label(label_), vec(at.vec_of(label_)) {
    const uint4 *const from = reinterpret_cast<const uint4 *>(row + at.head) + id;
    const int left = wanted ? at.vecs - id : 0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      q[j] = make_uint4(Vec<T>::neg_inf, Vec<T>::neg_inf, Vec<T>::neg_inf, Vec<T>::neg_inf);
      if (j * G < left) q[j] = from[j * G];
    }
    const int loose_label = at.loose_of(label);
#pragma unroll
    for (int j = 0; j < kLoose; ++j) {
      const int i = id + j * G;
      loose[j] = wanted && i < at.loose && !(vec < 0 && i == loose_label) ? to_float(row[at.loose_at(i)]) : kNegInf;
    }
    label_mine = label >= 0 && (vec >= 0 ? vec % G : loose_label % G) == id;
  }
  // Takes the label out (it is not among the loose elements) and returns the largest of the other logits.
  __device__ __forceinline__ float drop_label_and_max() {
    if (label_mine && vec >= 0) drop_element<T, NV>(q, vec / G, (unsigned)(label - at.head) % N);
    float m = max_of(T(), q);
#pragma unroll
    for (int j = 0; j < kLoose; ++j) m = fmaxf(m, loose[j]);
    if (G == 32) return warp_max(m);
#pragma unroll
    for (int o = G / 2; o > 0; o /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    return m;
  }
  // The team's sum of 2^(c x - t), of which this lane has added up `sum` over its vectors and its first loose element.
  __device__ __forceinline__ float team_sum_of(float sum, const Coef &c, float t) const {
#pragma unroll
    for (int j = 1; j < kLoose; ++j) sum += exp2_fast(c.power(loose[j], -t));
#pragma unroll
    for (int o = G / 2; o > 0; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    return no_infinity(sum);
  }
  // The row's gradient factor * 2^(c x - t), at_label for the label; Keep: the powers are in `e`.
  template <bool Keep>
  __device__ __forceinline__ void write(T *grad, const Coef &c, float t, float factor, float at_label,
                                        f32x2 (&e)[Keep ? NV : 1][N / 2], bool zero) {
    T *const dst = grad + at.head + id * N;
    const bool same = same_alignment(row, static_cast<const T *>(grad));
    constexpr bool kFine = Keep || sizeof(T) == 4;
    const float vec_factor = kFine ? factor : factor * c.lacking(t);
    const bool none = factor == 0.f;  // (the powers may be infinite where all but the label is masked)
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (j * G < at.vecs - id) {
        uint4 w = make_uint4(0, 0, 0, 0);
        if (!none) {
          if constexpr (!Keep) {
            pin(q[j]);  // (unpacked again rather than kept unpacked)
            exp_vec<T, kFine>(q[j], c, -t, e[0]);
          }
          w = scaled(T(), e[Keep ? j : 0], vec_factor);
        }
        store_vec(dst + j * G * N, same, w);
      }
    }
#pragma unroll
    for (int j = 0; j < kLoose; ++j)
      if (id + j * G < at.loose)
        grad[at.loose_at(id + j * G)] = from_float<T>(none ? 0.f : factor * exp2_fast(c.power(loose[j], -t)));
    // the label's own place, by the lane that wrote it (a thread's stores stay in order)
    if (!zero && label_mine) grad[label] = from_float<T>(at_label);
  }
};

template <typename T, int G, int NV>
__global__ void __launch_bounds__(kShortWarps * 32, NV <= 8 ? 8 : NV <= 10 ? 6 : 5)
policy_short_kernel(const PolicyArgs a) {
  pdl_sync();
  constexpr int N = Vec<T>::n, kRows = 32 / G;
  const int lane = threadIdx.x & 31, id = lane % G;
  const long long first = ((long long)blockIdx.x * kShortWarps + (threadIdx.x >> 5)) * kRows;
  if (first >= a.rows) return;  // (the whole warp)
  const long long r = first + lane / G;
  const Coef c = a.c;
  Sample y = {};
  y.label = -1;
  if (r < a.rows) y = sample_of(a, (int)r);
  const T *row = static_cast<const T *>(a.logits) + r * a.ld;
  ShortRow<T, G, NV> team(row, a.n_classes, y.live ? y.label : -1, id, y.live);
  const float x_y = y.live ? to_float(row[y.label]) : kNegInf;
  const float t = shift_of(team.drop_label_and_max(), c), first_power = exp2_fast(c.power(team.loose[0], -t));
  constexpr bool kKeep = NV * N <= 32;
  f32x2 e[kKeep ? NV : 1][N / 2];
  float sum;
  if constexpr (kKeep)
    sum = held_sum<T, NV>(team.q, first_power, c, t, e);
  else
    sum = held_sum<T, NV>(team.q, first_power, c, t);
  sum = team.team_sum_of(sum, c, t);
  float logp = 0.f, loss = 0.f;
  Gradient g{0.f, 0.f, 0.f};
  const Row stat({t, sum}, x_y, c);
  const bool slow = y.live && stat.slow();
  if (y.live && !slow)
    g = gradient_of<!kKeep && sizeof(T) == 2>(policy_terms(a, stat.logp(x_y, c), y, logp, loss), stat.t, stat.rest, stat.e_y);
  if (r < a.rows && id == 0 && !slow) put_row(a, r, logp, loss);
  __syncwarp();  // every lane has read its row's label
  if (a.grad && r < a.rows && !slow) {
    const bool zero = g.zero();
    const float factor = zero ? 0.f : g.factor * exp2_fast(t - g.t);  // the powers are relative to the others' maximum
    team.template write<kKeep>(static_cast<T *>(a.grad) + r * a.ld_grad, c, t, factor, g.at_label, e, zero);
  }
  unsigned slow_lanes = __ballot_sync(0xffffffffu, slow && id == 0);
  for (; slow_lanes; slow_lanes &= slow_lanes - 1) {  // (the whole warp, row by row)
    const int z = (int)first + (__ffs(slow_lanes) - 1) / G;
    slow_policy_row<T>(a, z, sample_of(a, z), lane, 32, nullptr);
  }
}

// Longer rows: one thread block each.  The last round of a row stays in registers until the gradient, the others are
// read again, which L2 still holds, the youngest first.  Many blocks that know nothing of each other keep the memory
// busier than one that works ahead: 8192 rows of 32000 bf16 logits, a quarter of them left out, 155-166 us; the whole row
// in the registers of 512 threads 174-181 us, the same with the powers kept (32 per thread) and the next rows copied
// into shared memory 246 us, a persistent block with bulk copies three rows ahead and a warp of its own for what
// happens once per row 177 us, clusters of blocks that hold longer rows together 224 us against 140 us (1999 rows of
// 50021 fp32 logits).
template <typename T, int Threads>
__global__ void __launch_bounds__(Threads, 1024 / Threads) policy_row_kernel(const PolicyArgs a) {
  pdl_sync();
  __shared__ __align__(8) Sum part[Threads / 32];
  __shared__ float slow_part[Threads / 32];
  __shared__ Gradient out;
  __shared__ int out_slow;
  const int r = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int label = a.actions[r];
  const float weight = a.weight ? a.weight[r] : 1.f;  // (asked for beside the label, not after it)
  const bool live = label >= 0 && label < a.n_classes && weight != 0.f;
  const T *row = static_cast<const T *>(a.logits) + (size_t)r * a.ld;
  const Team<T, Threads> team(row, a.n_classes, label, tid);
  float logp = 0.f, loss = 0.f, loose = kNegInf;
  Gradient g{0.f, 0.f, 0.f};
  uint4 q[kHeld];
  if (live) {  // (the whole block)
    Sample y;
    float x_y = 0.f;
    if (warp == 0) {
      y = sample_of(a, r);
      x_y = to_float(row[label]);
    }
    loose = team.read_loose();
    Sum s = warp_join(team.sum(a.c, loose, q));
    if (lane == 0) part[warp] = s;
    __syncthreads();
    if (warp == 0) {
      s = {kFloor, 0.f};
      if (lane < Threads / 32) s = part[lane];
      const Row stat(warp_join(s), x_y, a.c);
      if (!stat.slow()) g = gradient_of<true>(policy_terms(a, stat.logp(x_y, a.c), y, logp, loss), stat.t, stat.rest, stat.e_y);
      if (lane == 0) {
        out = g;
        out_slow = stat.slow();
      }
    }
    __syncthreads();
    g = out;
    if (out_slow) {  // (the whole block)
      slow_policy_row<T>(a, r, sample_of(a, r), tid, Threads, slow_part);
      return;
    }
  }
  if (tid == 0) put_row(a, r, logp, loss);
  if (a.grad) team.write(static_cast<T *>(a.grad) + (size_t)r * a.ld_grad, g, a.c, loose, q, true);
}

// Sums of row_loss over the partitions, in fp64 and a fixed order: one thread block each, or a cluster of eight where a
// partition takes a block more than one round (204800 rows in one partition take 3 us longer than in 50; with one block
// 19 us).
constexpr int kSumThreads = 1024, kSumLoads = 8;
template <int Blocks>
__global__ void __cluster_dims__(Blocks, 1, 1) __launch_bounds__(kSumThreads)
partition_sum_kernel(const float *row_loss, int rows, long long each, float *loss) {
  pdl_sync();
  __shared__ double part[kSumThreads / 32], total[Blocks];
  const auto cluster = cooperative_groups::this_cluster();
  const int rank = blockIdx.x % Blocks, mine = blockIdx.x / Blocks;
  if (Blocks > 1) cluster.sync();  // the other blocks' shared memory is there
  const long long first = mine * each, last = min((long long)rows, first + each);
  constexpr int kRound = kSumThreads * kSumLoads;
  double s = 0.0;
  for (long long r = first + rank * kRound + threadIdx.x; r < last; r += Blocks * kRound) {
    float x[kSumLoads];
#pragma unroll
    for (int i = 0; i < kSumLoads; ++i) x[i] = r + i * kSumThreads < last ? row_loss[r + i * kSumThreads] : 0.f;
#pragma unroll
    for (int i = 0; i < kSumLoads; ++i) s += (double)x[i];
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = s;
  __syncthreads();
  if (threadIdx.x < 32) {
    s = part[threadIdx.x];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (Blocks > 1 && threadIdx.x == 0) *cluster.map_shared_rank(&total[rank], 0) = s;
  }
  if (Blocks > 1) {
    cluster.sync();
    if (rank > 0) return;
    s = 0.0;
    for (int i = 0; i < Blocks; ++i) s += total[i];
  }
  if (threadIdx.x == 0) loss[mine] = (float)s;
}

// ---- preference loss: statistics of every row, then pairs, then gradients
//
// A gradient needs its whole pair's sum, so logits are read twice, and three launches are what this costs: 16 pairs of
// 256 tokens over 32000 classes (bf16) 199 us, 1.29 GB at 6.5 TB/s.  One launch that orders statistics and gradients of
// groups of pairs so that the second read finds L2 (items drawn from a counter, a flag per pair) took 232 us, and 421
// instead of 225 us at 8000 classes: a row-sized item is too short for its draw, look-up, fence and wait.

struct alignas(16) Stat {  // of a row, what its gradient needs
  float t, rest, e_y;       // slow: t is the largest logit
  int live;                 // 0: left out, 1, 2: slow
};
// What a pair reads and writes of its rows lies apart, so that a warp does so in whole lines (4 pairs of 41666 rows, one
// block each: 56 us of pair_kernel when it was part of Stat).
constexpr size_t kStatBytes = 32;  // a row's share of the workspace: Stat, log p, the factor of its gradient
constexpr double kLeftOut = INFINITY;  // log p of a row that does not count (no other is above zero)

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
  double *logp;
  float *k;  // factors of the gradients, written for each pair
  Coef c;
  double scale, beta, smooth;
};

__device__ __forceinline__ int row_bound(const PreferenceArgs &a, int s) {
  const long long b = a.begin[s];
  return b < 0 ? 0 : b > a.rows ? a.rows : (int)b;
}

__device__ __forceinline__ void put_stat(const PreferenceArgs &a, long long r, double logp, const Stat &s) {
  a.stat[r] = s;
  a.logp[r] = logp;
}
template <typename T>
__device__ __forceinline__ void slow_stat_row(const PreferenceArgs &a, long long r, const T *row, int label, int id, int n,
                                              float *part) {
  const SlowRow z = slow_stats(row, a.n_classes, label, a.c.hi, a.c.lo, a.c.scale, id, n, part);
  if (id != 0) return;
  if (z.nothing) {
    put_stat(a, r, kLeftOut, Stat{});
  } else {
    const Pair lp = z.logp();
    put_stat(a, r, (double)lp.hi + (double)lp.lo, Stat{z.top, z.rest, z.e_y, 2});
  }
}

// Statistics keep nothing: rounds of four vectors in 32 registers, so that an SM holds all its 2048 threads (16 pairs of
// 1024 tokens over 8000 classes: 200 us in all, with eight vectors and 1024 threads 219 us).
constexpr int kStatHeld = 4;
// Rows per thread block of the two kernels below: teams of 32 share a block of four.
template <int Threads>
constexpr int kTeams = Threads == 32 ? 4 : 1;

template <typename T, int Threads>
__global__ void __launch_bounds__(Threads * kTeams<Threads>, 2048 / (Threads * kTeams<Threads>))
row_stat_kernel(const PreferenceArgs a) {
  pdl_sync();
  constexpr bool kWarp = Threads == 32;
  __shared__ __align__(8) Sum part[Threads / 32];
  __shared__ float slow_part[Threads / 32];
  __shared__ int out_slow;
  const int tid = threadIdx.x % Threads, warp = tid >> 5, lane = tid & 31;
  const int r = blockIdx.x * kTeams<Threads> + threadIdx.x / Threads;
  const int label = r >= 0 && r < a.rows ? a.labels[r] : -1;          // (asked for beside the offsets, not after them)
  if (r < row_bound(a, 0) || r >= row_bound(a, 2 * a.pairs)) return;  // (the whole team)
  if (label < 0 || label >= a.n_classes) {
    if (tid == 0) put_stat(a, r, kLeftOut, Stat{});
    return;
  }
  const T *row = static_cast<const T *>(a.logits) + (size_t)r * a.ld;
  const Team<T, Threads, kStatHeld> team(row, a.n_classes, label, tid);
  const float x_y = to_float(row[label]);
  uint4 q[kStatHeld];
  Sum s = warp_join(team.sum(a.c, team.read_loose(), q));
  bool slow = false;
  if (!kWarp) {
    if (lane == 0) part[warp] = s;
    __syncthreads();
    s = {kFloor, 0.f};
    if (warp == 0) {
      if (lane < Threads / 32) s = part[lane];
      s = warp_join(s);
    }
  }
  if (warp == 0) {
    const Row stat(s, x_y, a.c);
    slow = stat.slow();
    if (!slow && lane == 0) {
      const Pair lp = stat.logp(x_y, a.c);
      put_stat(a, r, (double)lp.hi + (double)lp.lo, Stat{stat.t, stat.rest, stat.e_y, 1});
    }
  }
  if (!kWarp) {
    if (tid == 0) out_slow = slow;
    __syncthreads();
    slow = out_slow;
  }
  if (slow) {  // (the whole team)
    slow_stat_row(a, r, row, label, tid, Threads, kWarp ? nullptr : slow_part);
  }
}

// The same for short rows, teams of lanes as in policy_short_kernel (666656 rows of 300 bf16 classes, the whole call with the
// gradients below: 265 us, with a warp for every row 723 us).
template <typename T, int G, int NV>
__global__ void __launch_bounds__(kShortWarps * 32, 8) short_stat_kernel(const PreferenceArgs a) {
  pdl_sync();
  constexpr int kRows = 32 / G;
  const int lane = threadIdx.x & 31, id = lane % G;
  const long long first = ((long long)blockIdx.x * kShortWarps + (threadIdx.x >> 5)) * kRows, r = first + lane / G;
  int label = r < a.rows ? a.labels[r] : -1;
  const bool covered = r >= row_bound(a, 0) && r < row_bound(a, 2 * a.pairs);  // (and so r < rows)
  if (!covered || label >= a.n_classes) label = -1;
  const bool live = label >= 0;
  const Coef c = a.c;
  const T *row = static_cast<const T *>(a.logits) + r * a.ld;
  ShortRow<T, G, NV> team(row, a.n_classes, live ? label : -1, id, live);
  const float x_y = live ? to_float(row[label]) : kNegInf;
  const float t = shift_of(team.drop_label_and_max(), c);
  const float sum = team.team_sum_of(held_sum<T, NV>(team.q, exp2_fast(c.power(team.loose[0], -t)), c, t), c, t);
  const Row stat({t, sum}, x_y, c);
  const bool slow = live && stat.slow();
  const Pair lp = stat.logp(x_y, c);
  if (id == 0 && covered && !slow)
    put_stat(a, r, live ? (double)lp.hi + (double)lp.lo : kLeftOut, live ? Stat{stat.t, stat.rest, stat.e_y, 1} : Stat{});
  unsigned slow_lanes = __ballot_sync(0xffffffffu, slow && id == 0);
  for (; slow_lanes; slow_lanes &= slow_lanes - 1) {  // (the whole warp, row by row)
    const int from = __ffs(slow_lanes) - 1;
    const long long z = first + from / G;
    slow_stat_row(a, z, static_cast<const T *>(a.logits) + z * a.ld, __shfl_sync(0xffffffffu, label, from), lane, 32, nullptr);
  }
}

__device__ __forceinline__ double log_sigmoid(double x) { return fmin(x, 0.0) - log1p(exp(-fabs(x))); }
__device__ __forceinline__ double sigmoid(double x) {
  const double e = exp(-fabs(x));
  return (x >= 0.0 ? 1.0 : e) / (1.0 + e);
}

// share * x, also where x is infinite and has no share.
__device__ __forceinline__ double part_of(double share, double x) { return share == 0.0 && isinf(x) ? 0.0 : share * x; }

constexpr int kPairThreads = 512;
// One thread block per pair.  (Rows count in 32 bits without a sign: the last ones of 2^31 - 1 and a stride fit.)
__global__ void __launch_bounds__(kPairThreads) pair_kernel(const PreferenceArgs a) {
  pdl_sync();
  __shared__ double sum[2][kPairThreads / 32];
  __shared__ int count[2][kPairThreads / 32];
  const int q = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int first[2], last[2];
  double lp[2], n[2];
  const double ref[2] = {(double)a.ref_logp[2 * q], (double)a.ref_logp[2 * q + 1]};
  const double w = a.pair_weight ? (double)a.pair_weight[q] : 1.0;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    first[h] = row_bound(a, 2 * q + h);
    last[h] = row_bound(a, 2 * q + h + 1);
    double s = 0.0;
    int c = 0;
#pragma unroll 4
    for (unsigned r = (unsigned)first[h] + threadIdx.x; r < (unsigned)last[h]; r += kPairThreads) {
      const double logp = a.logp[r];
      if (logp != kLeftOut) { s += logp; ++c; }
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
    for (int w = 0; w < kPairThreads / 32; ++w) { s += sum[h][w]; c += count[h][w]; }
    n[h] = a.length_mean && c > 1 ? (double)c : 1.0;
    lp[h] = s / n[h];
  }
  // offsets that do not ascend, or lead to rows outside the first and the last offset, which have no statistics
  const bool bad = a.begin[2 * q] > a.begin[2 * q + 1] || a.begin[2 * q + 1] > a.begin[2 * q + 2] ||
                   first[0] < row_bound(a, 0) || last[1] > row_bound(a, 2 * a.pairs);
  if (bad) lp[0] = lp[1] = NAN;
  const double x = a.beta * ((lp[0] - ref[0]) - (lp[1] - ref[1]));
  const bool none = w == 0.0 && !bad;  // whatever its sequences hold
  const double slope = none ? 0.0 : a.beta * w * a.scale * (a.smooth * sigmoid(x) - (1.0 - a.smooth) * sigmoid(-x));
  if (threadIdx.x == 0) {
    a.seq_logp[2 * q] = (float)lp[0];
    a.seq_logp[2 * q + 1] = (float)lp[1];
    a.pair_loss[q] = none ? 0.f : (float)(-w * (part_of(1.0 - a.smooth, log_sigmoid(x)) + part_of(a.smooth, log_sigmoid(-x))));
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float k = (float)((h ? -slope : slope) / n[h]);
    for (unsigned r = (unsigned)first[h] + threadIdx.x; r < (unsigned)last[h]; r += kPairThreads) a.k[r] = k;
  }
}

// The last rows come first: they are what the statistics have left in L2.
template <typename T, int Threads>
__global__ void __launch_bounds__(Threads * kTeams<Threads>, 1024 / (Threads * kTeams<Threads>))
row_gradient_kernel(const PreferenceArgs a) {
  pdl_sync();
  const int tid = threadIdx.x % Threads;
  const int r = a.rows - 1 - (int)(blockIdx.x * kTeams<Threads> + threadIdx.x / Threads);
  if (r < 0) return;
  const Stat st = a.stat[r];  // (asked for beside the offsets)
  const float factor = a.k[r];
  const int label = a.labels[r];
  if (r < row_bound(a, 0) || r >= row_bound(a, 2 * a.pairs)) return;
  const T *row = static_cast<const T *>(a.logits) + (size_t)r * a.ld;
  T *grad = static_cast<T *>(a.grad) + (size_t)r * a.ld_grad;
  const float k = st.live ? factor : 0.f, s = st.rest + st.e_y;
  if (st.live == 2) {
    slow_gradient(row, grad, a.n_classes, label, a.c.hi, a.c.lo, st.t, -k / s, k * (st.rest / s), k != 0.f, tid, Threads);
    return;
  }
  const Team<T, Threads> team(row, a.n_classes, st.live ? label : -1, tid);
  uint4 q[kHeld];
  team.write(grad, gradient_of<true>(k, st.t, st.rest, st.e_y), a.c, st.live ? team.read_loose() : 0.f, q, false);
}

template <typename T, int G, int NV>
__global__ void __launch_bounds__(kShortWarps * 32, 8) short_gradient_kernel(const PreferenceArgs a) {
  pdl_sync();
  constexpr int kRows = 32 / G;
  const int lane = threadIdx.x & 31, id = lane % G;
  // (the last rows first, here too)
  const long long last = a.rows - 1 - ((long long)blockIdx.x * kShortWarps + (threadIdx.x >> 5)) * kRows, r = last - lane / G;
  Stat st = {};
  float k = 0.f;
  int label = -1;
  if (r >= 0) {
    st = a.stat[r];
    k = a.k[r];
    label = a.labels[r];
  }
  const bool covered = r >= row_bound(a, 0) && r < row_bound(a, 2 * a.pairs), slow = covered && st.live == 2;
  if (!covered || !st.live) label = -1;
  const Gradient g = gradient_of<true>(label >= 0 ? k : 0.f, st.t, st.rest, st.e_y);
  if (covered && !slow) {
    const T *row = static_cast<const T *>(a.logits) + r * a.ld;
    ShortRow<T, G, NV> team(row, a.n_classes, label, id, !g.zero());
    f32x2 e[1][Vec<T>::n / 2];
    team.template write<false>(static_cast<T *>(a.grad) + r * a.ld_grad, a.c, g.t, g.factor, g.at_label, e, g.zero());
  }
  unsigned slow_lanes = __ballot_sync(0xffffffffu, slow && id == 0);
  for (; slow_lanes; slow_lanes &= slow_lanes - 1) {  // (the whole warp, row by row)
    const long long z = last - (__ffs(slow_lanes) - 1) / G;
    const Stat x = a.stat[z];
    const float kz = a.k[z], s = x.rest + x.e_y;
    slow_gradient(static_cast<const T *>(a.logits) + z * a.ld, static_cast<T *>(a.grad) + z * a.ld_grad, a.n_classes,
                  a.labels[z], a.c.hi, a.c.lo, x.t, -kz / s, kz * (x.rest / s), kz != 0.f, lane, 32);
  }
}

template <typename T, int G, int NV>
cudaError_t launch_short(const PolicyArgs &a, cudaStream_t stream) {
  constexpr int rows = kShortWarps * (32 / G);
  return launch_k(policy_short_kernel<T, G, NV>, (unsigned)((a.rows - 1ll) / rows + 1), kShortWarps * 32, 0, stream, a);
}

// Threads for a longer row.  A row keeps its threads for as many reads, one after the other, as it has rounds, and about as
// long again for its sums, its loss and its gradient: the fewest (rounds + 1) * threads keep most rows on the way, as far
// as rows of three rounds (what is read again costs L2's time), fewer rounds if equal.  Measured for 200 million bf16
// logits, with 32 / 64 / 96 / 128 / 160 / 192 / 256 / 512 threads: classes 4200: 157 / 200 / 197 / 224 / 276 / 317 / 386 / 745 us,
// 8192: 162 / 140 / 164 / 146 / 172 / 193 / 225 / 416, 17000: 182 / 162 / 145 / 153 / 151 / 164 / 184 / 237,
// 33000: 219 / 189 / 175 / 166 / 159 / 149 / 155 / 205, 131072: 364 / 222 / 234 / 218 / 196 / 194 / 180 / 164.
inline int rounds_of(int slots, int threads) { return (slots - 1) / (threads * kHeld) + 1; }
template <int Last>
int row_threads(int) { return Last; }
template <int First, int Second, int... More>
int row_threads(int slots) {
  const int other = row_threads<Second, More...>(slots), r = rounds_of(slots, First), r_other = rounds_of(slots, other);
  return r <= 3 && (r + 1) * First < (r_other + 1) * other ? First : other;
}
template <typename T, int First, int... More>
cudaError_t launch_row_kernel(const PolicyArgs &a, int threads, cudaStream_t stream) {
  if constexpr (sizeof...(More) > 0) {
    if (threads != First) return launch_row_kernel<T, More...>(a, threads, stream);
  }
  return launch_k(policy_row_kernel<T, First>, a.rows, First, 0, stream, a);
}
template <typename T, int... Threads>
cudaError_t launch_rows(const PolicyArgs &a, int slots, cudaStream_t stream) {
  return launch_row_kernel<T, Threads...>(a, row_threads<Threads...>(slots), stream);
}

// Which kernel serves rows of a length: the fewest lanes that hold it in at most 8 vectors each (6 where these do; one or
// two where the row has not more, 400000 rows of 10 bf16 logits 23 us against 46 with four), then a warp with up to 12,
// then blocks.  Eight vectors against four on twice the lanes, same rows: 200000 x 1000 bf16 146 against 168 us; six
// against eight: 128000 x 1500 150 against 175 us; 16 per lane against a block of one warp in two rounds: 50000 x 4000
// 156 against 140 us, but 12 against that: 66666 x 3000 152 against 160 us.
template <typename T>
cudaError_t launch_policy(const PolicyArgs &a, cudaStream_t stream) {
  const int slots = a.n_classes / Vec<T>::n;  // whole vectors of a row, at most
  if (slots <= 2) return launch_short<T, 2, 1>(a, stream);
  if (slots <= 4) return launch_short<T, 4, 1>(a, stream);
  if (slots <= 8) return launch_short<T, 4, 2>(a, stream);
  if (slots <= 16) return launch_short<T, 2, 8>(a, stream);
  if (slots <= 24) return launch_short<T, 4, 6>(a, stream);
  if (slots <= 32) return launch_short<T, 4, 8>(a, stream);
  if (slots <= 48) return launch_short<T, 8, 6>(a, stream);
  if (slots <= 64) return launch_short<T, 8, 8>(a, stream);
  if (slots <= 96) return launch_short<T, 16, 6>(a, stream);
  if (slots <= 128) return launch_short<T, 16, 8>(a, stream);
  if (slots <= 192) return launch_short<T, 32, 6>(a, stream);
  if (slots <= 256) return launch_short<T, 32, 8>(a, stream);
  if (slots <= 320) return launch_short<T, 32, 10>(a, stream);
  if (slots <= 384) return launch_short<T, 32, 12>(a, stream);
  // (fp32 rows above 240 KB: those of two blocks on every SM would fill L2 before they are read again; 100000 classes 158
  // against 173 us, but 50021 157 against 146, and 131072 bf16, with twice the powers per byte, 166 against 162)
  constexpr int kWhole = 15 * 1024;
  if (sizeof(T) == 4 && slots > kWhole) return launch_k(policy_row_kernel<T, 1024>, a.rows, 1024, 0, stream, a);
  return launch_rows<T, 32, 64, 96, 128, 160, 192, 256, 320, 512>(a, slots, stream);
}

inline cudaError_t launch_pairs(const PreferenceArgs &a, cudaStream_t stream) {
  return launch_k(pair_kernel, a.pairs, kPairThreads, 0, stream, a);
}
template <typename T, int Threads>
cudaError_t launch_preference_rows(const PreferenceArgs &a, cudaStream_t stream) {
  constexpr int rows = kTeams<Threads>, block = Threads * rows;
  const unsigned grid = (unsigned)(((long long)a.rows + rows - 1) / rows);
  cudaError_t e = cudaSuccess;
  if (grid > 0) e = launch_k(row_stat_kernel<T, Threads>, grid, block, 0, stream, a);
  if (e == cudaSuccess) e = launch_pairs(a, stream);
  if (e == cudaSuccess && grid > 0 && a.grad) e = launch_k(row_gradient_kernel<T, Threads>, grid, block, 0, stream, a);
  return e;
}
template <typename T, int G, int NV>
cudaError_t launch_preference_short(const PreferenceArgs &a, cudaStream_t stream) {
  constexpr int rows = kShortWarps * (32 / G), block = kShortWarps * 32;
  const unsigned grid = (unsigned)(((long long)a.rows + rows - 1) / rows);
  cudaError_t e = cudaSuccess;
  if (grid > 0) e = launch_k(short_stat_kernel<T, G, NV>, grid, block, 0, stream, a);
  if (e == cudaSuccess) e = launch_pairs(a, stream);
  if (e == cudaSuccess && grid > 0 && a.grad) e = launch_k(short_gradient_kernel<T, G, NV>, grid, block, 0, stream, a);
  return e;
}

// Lanes with up to 8 vectors each, then the smallest block that has a row in two and a half rounds of 8 (200 million bf16
// logits, with 32 / 64 / 96 / 128 / 192 / 256 / 512 threads: classes 4200: 181 / 186 / 195 / 225 / 269 / 340 / 653 us,
// 17000: 178 / 165 / 160 / 159 / 157 / 169 / 225, 40000: 226 / 166 / 159 / 156 / 150 / 146 / 154).
template <typename T>
cudaError_t launch_preference(const PreferenceArgs &a, cudaStream_t stream) {
  const int slots = a.n_classes / Vec<T>::n;
  if (slots <= 8) return launch_preference_short<T, 4, 2>(a, stream);
  if (slots <= 16) return launch_preference_short<T, 2, 8>(a, stream);
  if (slots <= 32) return launch_preference_short<T, 4, 8>(a, stream);
  if (slots <= 64) return launch_preference_short<T, 8, 8>(a, stream);
  if (slots <= 128) return launch_preference_short<T, 16, 8>(a, stream);
  if (slots <= 256) return launch_preference_short<T, 32, 8>(a, stream);
  constexpr int kPerThread = kHeld * 5 / 2;
  if (slots <= 32 * kPerThread) return launch_preference_rows<T, 32>(a, stream);
  if (slots <= 64 * kPerThread) return launch_preference_rows<T, 64>(a, stream);
  if (slots <= 96 * kPerThread) return launch_preference_rows<T, 96>(a, stream);
  if (slots <= 128 * kPerThread) return launch_preference_rows<T, 128>(a, stream);
  if (slots <= 192 * kPerThread) return launch_preference_rows<T, 192>(a, stream);
  if (slots <= 256 * kPerThread) return launch_preference_rows<T, 256>(a, stream);
  return launch_preference_rows<T, 512>(a, stream);
}

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Whether a gradient shares elements with the logits in another way than element by element.  Rows of one stride may
// interleave (two halves of a wider matrix).
bool overlap(long long rows, int n_classes, size_t e, const void *logits, long long ld, const void *grad, long long ld_grad) {
  if (rows == 0 || (grad == logits && (ld == ld_grad || rows == 1))) return false;
  const uintptr_t x = reinterpret_cast<uintptr_t>(logits), g = reinterpret_cast<uintptr_t>(grad);
  const uintptr_t x_end = x + ((rows - 1) * ld + n_classes) * e, g_end = g + ((rows - 1) * ld_grad + n_classes) * e;
  if (x_end <= g || g_end <= x) return false;
  if (ld != ld_grad) return true;
  const uintptr_t stride = (uintptr_t)ld * e, row = n_classes * e, off = (g > x ? g - x : x - g) % stride;
  return off < row || off + row > stride;
}

// Bytes of an argument (none: a null pointer).
struct Span {
  uintptr_t first, last;
  Span(const void *p, size_t bytes) : first(reinterpret_cast<uintptr_t>(p)), last(p ? first + bytes : first) {}
};
Span matrix_span(const void *p, long long rows, int n_classes, long long ld, size_t e) {
  return Span(p, rows > 0 ? (size_t)((rows - 1) * ld + n_classes) * e : 0);
}
bool apart(const Span &a, const Span &b) { return a.last <= b.first || b.last <= a.first || a.first == a.last || b.first == b.last; }
bool apart(const Span &a, std::initializer_list<Span> others) {
  for (const Span &b : others)
    if (!apart(a, b)) return false;
  return true;
}
// An output that may take an input's place, number for number: whoever writes a row's (or a pair's) has read it by then.
bool apart_or_same(const Span &a, std::initializer_list<Span> others) {
  for (const Span &b : others)
    if (!apart(a, b) && a.first != b.first) return false;
  return true;
}

// What both entry points ask of the logits and their gradient.
bool logits_ok(long long rows, int n_classes, int dtype, double scale, const void *logits, long long ld, const void *grad,
               long long ld_grad) {
  if (rows < 0 || rows > 0x7fffffffll || n_classes < 1 || (dtype != NGC_F32 && dtype != NGC_BF16)) return false;
  if (!(scale > 0.0) || !std::isfinite(scale) || !((float)(scale * 1.4426950408889634) > 0.f) ||
      !std::isfinite((float)(scale * 1.4426950408889634)))
    return false;
  const size_t e = dtype == NGC_F32 ? 4 : 2;
  const long long far = (1ll << 44) / (rows + 1);  // (no buffer reaches further; offsets stay far below 63 bits)
  if (ld < n_classes || ld > far || (rows > 0 && !logits) || !aligned(logits, e)) return false;
  if (grad && (ld_grad < n_classes || ld_grad > far || !aligned(grad, e))) return false;
  return !grad || !overlap(rows, n_classes, e, logits, ld, grad, ld_grad);
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
  if (!(cfg->clip_low >= 0.0 && cfg->clip_low <= 1.0) || !(cfg->clip_high >= 0.0) || !std::isfinite((float)cfg->clip_high) ||
      !(cfg->kl_coef >= 0.0) || !std::isfinite((float)cfg->kl_coef) || cfg->rows_per_partition < 1)
    return NGC_ERR_INVALID;
  if (cfg->rows == 0) return NGC_OK;
  if (!actions || !old_logp || !advantage || !row_loss) return NGC_ERR_INVALID;
  for (const void *p : {(const void *)actions, (const void *)old_logp, (const void *)ref_logp, (const void *)advantage,
                        (const void *)weight, (const void *)logp, (const void *)row_loss, (const void *)loss})
    if (!aligned(p, 4)) return NGC_ERR_INVALID;
  const size_t e = cfg->dtype == NGC_F32 ? 4 : 2, vec = (size_t)cfg->rows * 4;
  const bool single = cfg->rows_per_partition == 1;
  const Span x = matrix_span(logits, cfg->rows, cfg->n_classes, ld, e), g = matrix_span(dlogits, cfg->rows, cfg->n_classes, ld_grad, e);
  const Span in[] = {{old_logp, vec}, {ref_logp, vec}, {advantage, vec}, {weight, vec}}, act(actions, vec);
  const Span lp(logp, vec), row(row_loss, vec), sum(loss, ((size_t)((cfg->rows - 1) / cfg->rows_per_partition) + 1) * 4);
  if (!apart(g, {act, in[0], in[1], in[2], in[3], lp, row, sum}) || !apart(x, {lp, row, sum}) || !apart(act, {lp, row}) ||
      !apart(lp, {row, sum}) || !(single ? apart_or_same(row, {sum}) : apart(row, sum)))
    return NGC_ERR_INVALID;
  for (const Span &out : {lp, row})
    if (!apart_or_same(out, {in[0], in[1], in[2], in[3]})) return NGC_ERR_INVALID;
  // (sums over more than one row are written when every row has been read)
  if (single && (!apart(sum, act) || !apart_or_same(sum, {in[0], in[1], in[2], in[3]}))) return NGC_ERR_INVALID;
  PolicyArgs a;
  a.logits = logits; a.grad = dlogits; a.ld = ld; a.ld_grad = ld_grad;
  a.rows = (int)cfg->rows; a.n_classes = cfg->n_classes;
  a.actions = actions; a.old_logp = old_logp; a.ref_logp = cfg->kl_coef > 0.0 ? ref_logp : nullptr;
  a.advantage = advantage; a.weight = weight; a.logp = logp; a.row_loss = row_loss;
  a.loss = single ? loss : nullptr;
  a.c = coef_of(cfg->scale); a.scale = (float)cfg->scale;
  a.low = (float)(1.0 - cfg->clip_low); a.high = (float)(1.0 + cfg->clip_high); a.kl = (float)cfg->kl_coef;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t rc = cfg->dtype == NGC_F32 ? launch_policy<float>(a, stream) : launch_policy<__nv_bfloat16>(a, stream);
  if (rc != cudaSuccess) return NGC_ERR_CUDA;
  if (loss && !a.loss) {
    const long long each = cfg->rows_per_partition, parts = (a.rows - 1) / each + 1;
    constexpr int kBlocks = 8;
    const bool wide = each > kSumThreads * kSumLoads && a.rows > kSumThreads * kSumLoads;  // (parts * kBlocks < 2^31 then)
    const cudaError_t e2 = wide ? launch_k(partition_sum_kernel<kBlocks>, (unsigned)parts * kBlocks, kSumThreads, 0, stream,
                                           (const float *)row_loss, a.rows, each, loss)
                                : launch_k(partition_sum_kernel<1>, (unsigned)parts, kSumThreads, 0, stream,
                                           (const float *)row_loss, a.rows, each, loss);
    if (e2 != cudaSuccess) return NGC_ERR_CUDA;
  }
  return NGC_OK;
}

size_t ngc_preference_workspace_bytes(int64_t rows, int32_t pairs) {
  (void)pairs;
  return rows < 0 ? 0 : ((size_t)rows + 1) * ngc::kStatBytes;
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
  const size_t e = cfg->dtype == NGC_F32 ? 4 : 2, per_pair = (size_t)cfg->pairs * 4;
  const Span x = matrix_span(logits, cfg->rows, cfg->n_classes, ld, e), g = matrix_span(dlogits, cfg->rows, cfg->n_classes, ld_grad, e);
  const Span lab(labels, (size_t)cfg->rows * 4), begin(seq_begin, ((size_t)cfg->pairs * 2 + 1) * 8);
  const Span ref(ref_logp, per_pair * 2), w(pair_weight, per_pair), seq(seq_logp, per_pair * 2), out(pair_loss, per_pair);
  const Span ws(workspace, ngc_preference_workspace_bytes(cfg->rows, cfg->pairs));
  if (!apart(ws, {x, g, lab, begin, ref, w, seq, out}) || !apart(g, {lab, begin, ref, w, seq, out}) ||
      !apart(seq, {x, lab, begin, w, out}) || !apart(out, {x, lab, begin, ref}) || !apart_or_same(seq, {ref}) ||
      !apart_or_same(out, {w}))
    return NGC_ERR_INVALID;
  PreferenceArgs a;
  a.logits = logits; a.grad = dlogits; a.ld = ld; a.ld_grad = ld_grad;
  a.rows = (int)cfg->rows; a.pairs = cfg->pairs; a.n_classes = cfg->n_classes; a.length_mean = cfg->length_mean != 0;
  a.labels = labels; a.begin = reinterpret_cast<const long long *>(seq_begin);
  a.ref_logp = ref_logp; a.pair_weight = pair_weight; a.seq_logp = seq_logp; a.pair_loss = pair_loss;
  a.stat = static_cast<Stat *>(workspace);
  a.logp = reinterpret_cast<double *>(a.stat + a.rows);
  a.k = reinterpret_cast<float *>(a.logp + a.rows);
  a.c = coef_of(cfg->scale);
  a.scale = cfg->scale; a.beta = cfg->beta; a.smooth = cfg->label_smoothing;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t rc = cfg->dtype == NGC_F32 ? launch_preference<float>(a, stream) : launch_preference<__nv_bfloat16>(a, stream);
  if (rc != cudaSuccess) return NGC_ERR_CUDA;
  return NGC_OK;
}

}  // extern "C"

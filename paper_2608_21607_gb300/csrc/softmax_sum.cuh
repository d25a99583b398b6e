// Sums of powers for the softmax of a row, shared by the kernels that take
// log-probabilities: exponents, a running maximum and sum, and their merging.
//
// For values x, temperature tau, c = log2(e) / tau and a value m near the largest
// x, a sum is kept as (m, S) with S = sum 2^(c x - ref(m)).
#pragma once

#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

namespace nmd {

constexpr double kLn2 = 0.69314718055994530942;
constexpr double kLog2e = 1.4426950408889634074;

// 2^x by the SFU (results below 2^-126 become 0, which no sum of
// probabilities can tell from the exact value)
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// the larger value, NaN if one is
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

// Pairs of fp32 values (fp32x2 instructions: one issue slot for two)
typedef unsigned long long pair_t;
__device__ __forceinline__ pair_t pair_of(float a, float b) {
  pair_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 halves(pair_t p) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(p));
  return r;
}
__device__ __forceinline__ pair_t add2(pair_t a, pair_t b) {
  pair_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ pair_t mul2(pair_t a, pair_t b) {
  pair_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ pair_t fma2(pair_t a, pair_t b, pair_t c) {
  pair_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}

// c = log2(e) / tau as hi + lo, hi of 12 bits, so that a 16-bit x times hi less
// an integer is exact and the exponent is rounded once, without a leaning that
// the sum over a long sequence would show.  lo > 0: both products of -inf are
// -inf.  `whole` is c in one fp32 value.
struct Scale {
  float hi, lo, whole;
};
// 2^(c (x - m))
__device__ __forceinline__ float power(float x, float m, Scale c) {
  const float d = x - m;
  return ex2(fmaf(d, c.hi, d * c.lo));
}
__device__ __forceinline__ pair_t exponent2(pair_t x, float m, Scale c) {
  const pair_t d = add2(x, pair_of(-m, -m));
  return fma2(d, pair_of(c.hi, c.hi), mul2(d, pair_of(c.lo, c.lo)));
}
__device__ __forceinline__ pair_t power2(pair_t x, float m, Scale c) {
  const float2 e = halves(exponent2(x, m, c));
  return pair_of(ex2(e.x), ex2(e.y));
}
inline float2 two_floats(double v) {
  float2 t;
  t.x = (float)v;
  t.y = (float)(v - (double)t.x);
  return t;
}
// c of a temperature; false if it is not a positive number of ordinary size
inline bool scale_of(double temperature, Scale* s) {
  if (!(temperature > 0.0)) return false;
  const double c = kLog2e / temperature;
  if (!(c >= 1e-30) || !(c <= 1e30)) return false;
  int e = 0;
  const double f = frexp(c, &e);   // in [1/2, 1)
  double head = floor(f * 4096.0);
  if (head == f * 4096.0) head -= 1.0;   // hi is below c, so that lo > 0
  s->hi = (float)ldexp(head, e - 12);
  s->lo = (float)(c - (double)s->hi);
  s->whole = (float)c;
  return true;
}

// (m, S) of a set of elements: a value near their maximum (NaN if one is; -inf
// of none) and the sum of 2^(c x - ref), where ref is the integer ceil(c m) if
// that is within +-1024, and c m otherwise.  An integer reference makes every
// rescaling exact.
struct __align__(8) Stat {
  float m, S;
};
__device__ __forceinline__ bool is_near(float m, Scale c) { return fabsf(m * c.hi) <= 1024.f; }
__device__ __forceinline__ float ref_of(float m, Scale c) { return ceilf(m * c.hi); }
// ref - c m: what the reference is above the maximum
__device__ __forceinline__ float above(float m, Scale c) {
  return is_near(m, c) ? fmaf(-m, c.lo, fmaf(-m, c.hi, ref_of(m, c))) : 0.f;
}
// 2^(reference of m - reference of to), m <= to
__device__ __forceinline__ float rescale(float m, float to, Scale c) {
  if (is_near(m, c) && is_near(to, c)) {   // a power of two, put together from its bits
    const int e = (int)(ref_of(m, c) - ref_of(to, c));
    return e < -126 ? 0.f : __int_as_float((e + 127) << 23);
  }
  if (m == to) return 1.f;
  const float d = m - to;
  return ex2(fmaf(d, c.hi, d * c.lo) + (above(m, c) - above(to, c)));
}
// log p = (x - m) / tau - ln S - ln2 above(m) as hi + lo, for 1 / tau = it.x + it.y:
// its distance from a reference is much smaller than log p itself, and would show
// the roundings of one fp32 value.  (In fp64 it cost the policy loss 3 %.)
struct LogProb {
  float hi, lo;
  __device__ __forceinline__ float value() const { return hi + lo; }
  __device__ __forceinline__ float less(float reference) const { return (hi - reference) + lo; }
};
__device__ __forceinline__ LogProb log_prob(float x, Stat st, float over, float2 it) {
  int k = 0;
  float f = frexpf(st.S, &k);   // S = f 2^k, f near 1
  if (f < 0.7f) {
    f *= 2.f;
    --k;
  }
  constexpr float ln2_lo = (float)(kLn2 - (double)(float)kLn2);
  const float d = x - st.m, t = d - x, kf = (float)k;
  const float d_lo = (x - (d - t)) - (st.m + t);   // what the difference rounds away
  const float p = d * it.x, p_lo = fmaf(d, it.x, -p) + fmaf(d, it.y, d_lo * it.x);
  const float q = kf * (float)kLn2, q_lo = fmaf(kf, (float)kLn2, -q) + kf * ln2_lo;
  LogProb o;
  o.hi = p - q;
  const float u = o.hi - p;
  o.lo = (p - (o.hi - u)) - (q + u) + (p_lo - q_lo) - fmaf(over, (float)kLn2, log1pf(f - 1.f));
  if (!(fabsf(o.hi) < INFINITY)) o.lo = st.S > 0.f ? 0.f : NAN;   // (no sum: no distribution)
  // No probability is above 1: roundings that say so, above all of a target's score
  // that was not formed like those in the sum, would make log(1 - p) no number.
  if (o.hi + o.lo > 0.f) o.hi = o.lo = 0.f;
  return o;
}
// Merges over groups of `width` lanes (a power of two); every lane of a group
// gets the same result.
template <int width>
__device__ __forceinline__ Stat merge_lanes(Stat st, Scale c) {
  float m = st.m;
#pragma unroll
  for (int o = width / 2; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
  float S = st.S * rescale(st.m, m, c);
#pragma unroll
  for (int o = width / 2; o > 0; o >>= 1) S += __shfl_xor_sync(0xffffffffu, S, o);
  return {m, S};
}

// A running pair.  The reference is the maximum of the first elements and stays
// until a group of elements exceeds it by much (its sum passes kHigh), so that
// the usual group costs a product, a correction, an exponential and an addition
// per element and no comparison.  The SFU's exponential is low by 5e-8 on
// average for arguments below -1 and high by 3.5e-8 for those above 1 (measured
// over many arguments), which the sum over a long sequence would show; so one
// half of the elements is taken 2^kLift larger and the other half 2^kSink
// smaller, and their sums are set right by these powers, exactly.  kLift brings the
// elements that make up a sum above 1: 2^16 those of a long row.  A short row is made
// up by elements near its maximum, and its few roundings do not average; there the
// exponent's own, at 2^-20 for a lift of 16, is the largest (rows of up to 256 columns:
// 1.0e-7 off in the root mean square, 7.8e-8 with a lift of 4).
struct RunningSum {
  static constexpr float kHigh = 4096.f, kSink = 2.f;
  Stat s{-INFINITY, 0.f};
  float r = 0.f;
  bool usual = false;   // the reference is an integer

  // The sum of a group of 2 H values against the (integer) reference; x is used
  // up.  All products, then all exponentials, then the sums: enough of each under
  // way to cover their latencies.
  template <int H, int kLift = 16>
  __device__ __forceinline__ float group_sum(pair_t (&x)[H], Scale c) const {
    const pair_t hi = pair_of(c.hi, c.hi), lo = pair_of(c.lo, c.lo), k0 = pair_of(-r - kSink, (float)kLift - r);
#pragma unroll
    for (int i = 0; i < H; ++i) x[i] = fma2(x[i], lo, fma2(x[i], hi, k0));
#pragma unroll
    for (int i = 0; i < H; ++i) {
      const float2 e = halves(x[i]);
      x[i] = pair_of(ex2(e.x), ex2(e.y));
    }
#pragma unroll
    for (int d = H / 2; d > 0; d /= 2)
#pragma unroll
      for (int i = 0; i < d; ++i) x[i] = add2(x[i], x[i + d]);
    const float2 t = halves(x[0]);
    return fmaf(t.y, 1.f / (1 << kLift), t.x * (float)(1 << (int)kSink));
  }
  // takes m (at least s.m, or NaN) as the value near the maximum
  __device__ __forceinline__ void raise(float m, Scale c) {
    if (m == s.m) return;
    s.S *= rescale(s.m, m, c);
    s.m = m;
    r = ref_of(m, c);
    usual = is_near(m, c);
  }
};

}  // namespace nmd

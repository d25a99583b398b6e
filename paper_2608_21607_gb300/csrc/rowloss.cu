// Losses over the rows of a logits matrix, with the gradient of the logits:
// the log-probability of one column per row, the paired preference loss and
// the clipped policy loss (formulas in include/nmd.h).
//
// For row t with logits x_tv, temperature tau, c = log2(e) / tau and the row's
// maximum m,
//   e_tv = 2^(c (x_tv - m)),  S = sum_v e_tv,  p_tv = e_tv / S,
//   log p_ty = (x_ty - m) / tau - ln S,
//   d loss / d x_tv = g_t (1[v = y_t] - p_tv) / tau.
// (The difference is taken before the product: c m alone would pass fp32's
// range where a row is masked with the type's lowest value.)  m and S come
// from one pass with a running maximum: a thread keeps its own (m, S),
// rescales S when a group of vectors raises m, and the threads' pairs are
// merged in a fixed order.  A row's sum of powers is fp32, sums over the rows of a
// sequence or batch are fp64; the only rounding to fewer bits is that of the gradient
// to the logits' type, once, when it is stored.
//
// Everything here is bound by HBM: a row is read once (twice where the
// gradient's coefficient depends on other rows) and its gradient written once.
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include "nmd_internal.cuh"
#include "softmax_sum.cuh"
#include "tc_pipe.cuh"
#include "tc_ptx.cuh"

namespace nmd {
namespace {

// 16-byte vectors of the three element types: N values, the largest of them (NaN
// if one is), pairs of them
template <class T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ uint4 none() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }   // -inf
  static __device__ __forceinline__ pair_t pair(const uint4& v, int i) {
    return i == 0 ? pair_of(__uint_as_float(v.x), __uint_as_float(v.y))
                  : pair_of(__uint_as_float(v.z), __uint_as_float(v.w));
  }
  static __device__ __forceinline__ float top(const uint4& v) {
    return max_nan(max_nan(__uint_as_float(v.x), __uint_as_float(v.y)),
                   max_nan(__uint_as_float(v.z), __uint_as_float(v.w)));
  }
  static __device__ __forceinline__ uint4 pack(const pair_t (&f)[2]) {
    const float2 a = halves(f[0]), b = halves(f[1]);
    return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
  }
  static __device__ __forceinline__ float get(float x) { return x; }
  static __device__ __forceinline__ float put(float x) { return x; }
};
__device__ __forceinline__ uint32_t word(const uint4& v, int i) {
  return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
}
template <>
struct Vec<bf16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ uint4 none() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }   // -inf
  static __device__ __forceinline__ pair_t pair(const uint4& v, int i) {
    const uint32_t w = word(v, i);
    return pair_of(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  }
  static __device__ __forceinline__ float top(const uint4& v) {
    const __nv_bfloat162* h = (const __nv_bfloat162*)&v;
    const float2 f = __bfloat1622float2(__hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3])));
    return max_nan(f.x, f.y);
  }
  static __device__ __forceinline__ uint4 pack(const pair_t (&f)[4]) {
    uint4 w;
    __nv_bfloat162* h = (__nv_bfloat162*)&w;
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __float22bfloat162_rn(halves(f[i]));
    return w;
  }
  static __device__ __forceinline__ float get(bf16 x) { return __bfloat162float(x); }
  static __device__ __forceinline__ bf16 put(float x) { return __float2bfloat16_rn(x); }
};
template <>
struct Vec<__half> {
  static constexpr int N = 8;
  static __device__ __forceinline__ uint4 none() { return make_uint4(0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u, 0xfc00fc00u); }   // -inf
  static __device__ __forceinline__ pair_t pair(const uint4& v, int i) {
    const uint32_t w = word(v, i);
    const float2 f = __half22float2(*(const __half2*)&w);
    return pair_of(f.x, f.y);
  }
  static __device__ __forceinline__ float top(const uint4& v) {
    const __half2* h = (const __half2*)&v;
    const float2 f = __half22float2(__hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3])));
    return max_nan(f.x, f.y);
  }
  static __device__ __forceinline__ uint4 pack(const pair_t (&f)[4]) {
    uint4 w;
    __half2* h = (__half2*)&w;
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __float22half2_rn(halves(f[i]));
    return w;
  }
  static __device__ __forceinline__ float get(__half x) { return __half2float(x); }
  static __device__ __forceinline__ __half put(float x) { return __float2half_rn(x); }
};

// A running pair over a thread's vectors.
template <class T, int LIFT = 16>
struct Running : RunningSum {
  // four vectors: get(0) to get(3), asked for again where the group is not a usual one
  template <class G>
  __device__ __forceinline__ void add(G get, Scale c) {
    constexpr int P = Vec<T>::N / 2, H = 4 * P;
    for (;;) {
      if (usual) {
        pair_t x[H];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint4 v = get(k);
#pragma unroll
          for (int i = 0; i < P; ++i) x[k * P + i] = Vec<T>::pair(v, i);
        }
        const float group = this->template group_sum<H, LIFT>(x, c);
        if (group < kHigh) {
          s.S += group;
          return;
        }
      }
      // the first group, one with larger values, or one with NaN or infinities
      float m = s.m;
#pragma unroll 1
      for (int k = 0; k < 4; ++k) m = max_nan(m, Vec<T>::top(get(k)));
      raise(m, c);
      if (usual) continue;
      // huge, infinite or no numbers; only -inf so far: the sum is 0 and stays 0
      const float z = s.m == -INFINITY ? 0.f : s.m;
      pair_t sum = pair_of(0.f, 0.f);
#pragma unroll 1
      for (int k = 0; k < 4; ++k) {
        const uint4 v = get(k);
#pragma unroll
        for (int i = 0; i < P; ++i) sum = add2(sum, power2(Vec<T>::pair(v, i), z, c));
      }
      const float2 t = halves(sum);
      s.S += t.x + t.y;
      return;
    }
  }
  // one value
  __device__ __forceinline__ void add(float x, Scale c) {
    raise(max_nan(s.m, x), c);
    if (usual) s.S += ex2(fmaf(x, c.hi, -r) + x * c.lo);
    else s.S += power(x, s.m == -INFINITY ? 0.f : s.m, c);
  }
};

struct Policy {
  const float* old;      // T: log-probabilities under the policy that produced the tokens
  const float* ref;      // T, or nullptr (the preference loss has it too)
  const float* adv;      // T
  const float* weight;   // T: each row's share of the loss; nullptr: the row kernel takes it itself
  float lo, hi, kl;      // 1 - clip_low, 1 + clip_high, KL coefficient
  float* terms;          // 3 T: weighted loss, KL, cut-off terms
  const int64_t* offsets;   // S + 1, or nullptr
  int64_t S;
  float* stats;          // 3: the sums of the terms
};

struct Rows {
  const void* x;
  int64_t T, V, ld;
  const int64_t* y;
  Scale c;
  float2 inv_temp;       // 1 / tau as the sum of two
  float* logps;          // T
  Stat* stats;           // T (the statistics pass writes, the gradient pass reads) or nullptr
  float* coef;           // T: g_t; zeroed by the statistics pass
  float* gap;            // T: log-probability less the reference's
  void* grad;            // T x V with row stride gld, or nullptr
  int64_t gld;
  int64_t each;          // vectors of a row that one CTA of its cluster takes
  int same_phase;        // rows of x and grad start at the same offset from a 16-byte boundary
  unsigned* done;        // a count that starts at zero: finished CTAs, or rows
  Policy p;
};

// where the 16-byte vectors of a row lie: `head` elements, `nvec` vectors, `tail` elements
struct Span {
  int head, tail;
  int64_t nvec;
};
template <class T>
__device__ __forceinline__ Span span_of(const T* row, int64_t V) {
  Span s;
  const int off = (int)((uintptr_t)row & 15);
  const int64_t h = off ? (16 - off) / (int)sizeof(T) : 0;
  s.head = (int)(h < V ? h : V);
  s.nvec = (V - s.head) / Vec<T>::N;
  s.tail = (int)(V - s.head - s.nvec * Vec<T>::N);
  return s;
}

// Fixed-order sum over one CTA of up to 1024 threads; every thread gets it.
__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = (threadIdx.x & 31) < blockDim.x / 32 ? red[threadIdx.x & 31] : 0.0;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// Whether this CTA is the last of the grid to come here; what the others wrote before is then visible.
__device__ __forceinline__ bool last_cta(unsigned* done) {
  __shared__ int last;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(done, 1u) == gridDim.x - 1;
  __syncthreads();
  if (last) __threadfence();
  return last != 0;
}

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// border k of the sequences, held within the rows whatever the array says
__device__ __forceinline__ int64_t border(const int64_t* offsets, int64_t k, int64_t T) {
  const int64_t o = offsets[k];
  return o < 0 ? 0 : (o > T ? T : o);
}

// A row's share of the policy loss, by one warp: 1 / (live rows), or 1 /
// (sequences x live rows of its sequence); 0 for a row outside every sequence.
__device__ __forceinline__ float weight_of(const int64_t* y, const int64_t* offsets, int64_t T, int64_t S, int64_t t) {
  const int lane = threadIdx.x & 31;
  int64_t from = 0, to = T;
  double sequences = 1.0;
  if (offsets != nullptr) {
    bool mine = false;
    for (int64_t k = lane; k < S; k += 32) {
      const int64_t a = border(offsets, k, T), b = border(offsets, k + 1, T);
      if (a <= t && t < b) {
        mine = true;
        from = a;
        to = b;
      }
    }
    const unsigned m = __ballot_sync(0xffffffffu, mine);
    if (m == 0) return 0.f;
    from = __shfl_sync(0xffffffffu, from, __ffs(m) - 1);
    to = __shfl_sync(0xffffffffu, to, __ffs(m) - 1);
    sequences = (double)S;
  }
  int n = 0;
#pragma unroll 8
  for (int64_t i = from + lane; i < to; i += 32) n += y[i] >= 0;
  n = __reduce_add_sync(0xffffffffu, n);
  return (float)(1.0 / (sequences * (double)max(n, 1)));
}

// A row's gradient: d_v = down 2^(c (x_v - m)) + up [v = y].  16-bit gradients
// take the factor |down| into the exponent, where its rounding (2^-14 at most)
// is far below theirs.
struct Slope {
  float m, down, up, k, sign;
  bool zero, fold;
};
template <class T>
__device__ __forceinline__ Slope slope_of(bool live, float coef, Stat st, float2 inv_temp, Scale c) {
  Slope d;
  d.zero = !live || coef == 0.f;   // left out, cut off, in no sequence: the logits are not needed
  d.m = st.m;
  d.up = coef * inv_temp.x;
  d.down = -d.up / st.S;
  const float l = log2f(fabsf(d.down));
  d.k = fmaf(-st.m, c.whole, l);
  d.sign = d.down < 0.f ? -1.f : 1.f;
  d.fold = sizeof(T) == 2 && is_near(st.m, c) && fabsf(l) < 1024.f;
  return d;
}
// One element of it.
template <class T>
__device__ __forceinline__ float slope_at(T x, const Slope& s, Scale c, bool target) {
  return fmaf(s.down, power(Vec<T>::get(x), s.m, c), target ? s.up : 0.f);
}
// K vectors of it, read `apart` and written `stride` vectors apart.
template <class T, bool FOLD, bool ALIGNED, int K>
__device__ __forceinline__ void write_vectors(const uint4* v, int apart, int stride, T* g, const Slope& s, Scale c) {
  constexpr int N = Vec<T>::N, H = N / 2;
  uint4 w[K];
#pragma unroll
  for (int q = 0; q < K; ++q) w[q] = v[q * apart];
  const pair_t mul = FOLD ? pair_of(s.sign, s.sign) : pair_of(s.down, s.down);
  const pair_t cc = pair_of(c.whole, c.whole), kk = pair_of(s.k, s.k);
  // all products, then all exponentials, ...: enough of each under way to cover their latencies
  pair_t d[K][H];
#pragma unroll
  for (int q = 0; q < K; ++q)
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const pair_t x = Vec<T>::pair(w[q], h);
      d[q][h] = FOLD ? fma2(x, cc, kk) : exponent2(x, s.m, c);
    }
#pragma unroll
  for (int q = 0; q < K; ++q)
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const float2 e = halves(d[q][h]);
      d[q][h] = pair_of(ex2(e.x), ex2(e.y));
    }
#pragma unroll
  for (int q = 0; q < K; ++q) {
#pragma unroll
    for (int h = 0; h < H; ++h) d[q][h] = mul2(d[q][h], mul);
    const uint4 r = Vec<T>::pack(d[q]);
    if (ALIGNED) {
      __stcs((uint4*)g + q * stride, r);
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k) g[(int64_t)q * stride * N + k] = ((const T*)&r)[k];
    }
  }
}
template <class T, bool FOLD, bool ALIGNED>
__device__ __forceinline__ void write_run(const uint4* v, int apart, int n, int tid, int stride, T* g, const Slope& s,
                                          Scale c) {
  constexpr int N = Vec<T>::N, K = ALIGNED ? 4 : 1;
  int i = tid;
  for (; i + (K - 1) * stride < n; i += K * stride, v += K * apart)
    write_vectors<T, FOLD, ALIGNED, K>(v, apart, stride, g + (int64_t)i * N, s, c);
  if (K > 1)
    for (; i < n; i += stride, v += apart)
      write_vectors<T, FOLD, ALIGNED, 1>(v, apart, stride, g + (int64_t)i * N, s, c);
}
// n vectors of a gradient row from g on, by `stride` threads.  v: this thread's
// first vector, its next ones `apart` further each.  `target`: the target's
// place among the elements, or anything outside of them.
template <class T>
__device__ __forceinline__ void write_slope(const uint4* v, int n, int tid, int stride, T* g, const Slope& s, Scale c,
                                            int64_t target, bool aligned, int apart) {
  constexpr int N = Vec<T>::N;
  if (s.zero) {
    const uint4 w = make_uint4(0, 0, 0, 0);
    if (aligned)
      for (int i = tid; i < n; i += stride) __stcs((uint4*)g + i, w);
    else
      for (int64_t i = tid; i < (int64_t)n * N; i += stride) g[i] = Vec<T>::put(0.f);
    return;
  }
  if (!aligned) write_run<T, false, false>(v, apart, n, tid, stride, g, s, c);
  else if (sizeof(T) == 2 && s.fold) write_run<T, sizeof(T) == 2, true>(v, apart, n, tid, stride, g, s, c);
  else write_run<T, false, true>(v, apart, n, tid, stride, g, s, c);
  // the thread that wrote the target's vector puts its value right
  if (target >= 0 && target < (int64_t)n * N) {
    const int i = (int)(target / N);
    if (i % stride == tid) {
      const T* e = (const T*)(v + (int64_t)(i / stride) * apart);
      g[target] = Vec<T>::put(slope_at(e[target % N], s, c, true));
    }
  }
}

enum { kStats = 0, kPolicy = 1 };

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// What a row's single values make of its statistics.
struct RowOut {
  float lp, term, kl, cut, coef, gap;   // gap: lp less the reference's
};
template <int MODE, class W>
__device__ __forceinline__ RowOut row_out(const Rows& a, bool live, float xy, float adv, float old, float ref, W weight,
                                          Stat& st) {
  RowOut o{0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (!live) return o;
  if (st.m == INFINITY) st.m = NAN;   // no distribution
  const float over = above(st.m, a.c);
  const LogProb lp = log_prob(xy, st, over, a.inv_temp);
  o.lp = lp.value();
  st.S *= ex2(over);   // from here on against the maximum itself, as the gradient takes it
  o.gap = lp.less(ref);
  if (MODE == kPolicy) {
    const Policy& p = a.p;
    const float d = lp.less(old), ratio = expf(d);
    const float bound = fminf(fmaxf(ratio, p.lo), p.hi);
    const bool off = (adv > 0.f && ratio > p.hi) || (adv < 0.f && ratio < p.lo);
    // without an advantage there is no term, also where exp(d) passes fp32's range
    const float ra = adv == 0.f && d < INFINITY ? 0.f : ratio * adv, ba = bound * adv;
    o.term = -(ra < ba || ra != ra ? ra : ba);
    o.coef = off ? 0.f : -ra;
    if (p.ref != nullptr) {
      const float q = expm1f(-o.gap);
      o.kl = q + o.gap;
      if (p.kl != 0.f) {
        o.term += p.kl * o.kl;
        o.coef -= p.kl * q;
      }
    }
    const float w = weight();
    // a row outside every sequence takes no part, whatever it holds (0 x inf is no number)
    o.term = w != 0.f ? o.term * w : 0.f;
    o.kl = w != 0.f ? o.kl * w : 0.f;
    o.coef = w != 0.f ? o.coef * w : 0.f;
    o.cut = off ? w : 0.f;
  }
  return o;
}
template <int MODE>
__device__ __forceinline__ void write_row(const Rows& a, int64_t t, const RowOut& o, const Stat& st) {
  a.logps[t] = o.lp;
  if (MODE == kStats && a.stats != nullptr) {
    a.stats[t] = st;
    a.gap[t] = o.gap;
    a.coef[t] = 0.f;
    if (t == 0) *a.done = 0;
  }
  if (MODE == kPolicy) {
    a.p.terms[t] = o.term;
    a.p.terms[a.T + t] = o.kl;
    a.p.terms[2 * a.T + t] = o.cut;
  }
}

// The sums of the rows' terms, in their order, by the warp (GROUP 32) or CTA that
// finished the last row.
template <int GROUP>
__device__ __noinline__ void sum_terms(const Rows& a, double* red) {
  __threadfence();
  const int tid = GROUP == 32 ? threadIdx.x & 31 : threadIdx.x, step = GROUP == 32 ? 32 : blockDim.x;
  double s[3] = {0.0, 0.0, 0.0};
#pragma unroll 4
  for (int64_t i = tid; i < a.T; i += step)
#pragma unroll
    for (int k = 0; k < 3; ++k) s[k] += (double)__ldcg(a.p.terms + k * a.T + i);
#pragma unroll
  for (int k = 0; k < 3; ++k) s[k] = warp_sum(s[k]);
  if (GROUP != 32) {   // red: 3 x 16 warps
    if ((tid & 31) == 0)
      for (int k = 0; k < 3; ++k) red[k * 16 + tid / 32] = s[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) s[k] = warp_sum((tid & 31) < step / 32 ? red[k * 16 + (tid & 31)] : 0.0);
  }
  if (tid == 0)
    for (int k = 0; k < 3; ++k) a.p.stats[k] = (float)s[k];
}

__device__ __forceinline__ void copy_async(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int left>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(left) : "memory"); }

// Log-probabilities, and for the policy loss everything of a row: one warp per
// row (WARP), or one CTA or cluster of CTAs, each with one run of its vectors.
// A thread's vectors come through slots of its own in shared memory, DEPTH
// groups of four ahead, so that the loads under way take no registers.  For a
// policy row's gradient (KEEP) all groups stay there, and the row is read once.
// Bound by HBM: 4001 rows of 50,001 fp16 columns, a fifth of them left out,
// take 52.3 us, 6.1 TB/s or 0.90 of a plain copy's rate; one row of 139,255
// columns (a cluster of eight) 4.8 us, which is the launch and two barriers.
template <class T, bool WARP, int MODE, int DEPTH, bool KEEP>
__global__ void __launch_bounds__(512, 2) row_kernel(const __grid_constant__ Rows a) {
  constexpr int N = Vec<T>::N;
  extern __shared__ uint4 slots[];
  __shared__ Stat red[16], peers[8];
  __shared__ Slope shared_slope;
  __shared__ int shared_last;
  __shared__ double dred[MODE == kPolicy && !WARP ? 48 : 1];
  __shared__ float shared_share;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (MODE == kStats) asm volatile("griddepcontrol.launch_dependents;");
  unsigned csize = 1, rank = 0;
  if (!WARP) {
    asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(csize));
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    if (csize > 1) cluster_arrive();   // waited for before a peer's shared memory is written
  }
  const int64_t t = WARP ? (int64_t)blockIdx.x * (blockDim.x / 32) + warp : blockIdx.x / csize;
  if (WARP && t >= a.T) return;
  const int tid = WARP ? lane : threadIdx.x, nthr = WARP ? 32 : blockDim.x;

  const int64_t y = a.y[t];
  const bool live = y >= 0;
  const T* x = (const T*)a.x + t * a.ld;
  const Span sp = span_of(x, a.V);
  // this CTA's vectors: [0, n) from xv, the first of them vector v0 of the row
  const int64_t v0 = min(sp.nvec, rank * a.each);
  const int n = (int)min(a.each, sp.nvec - v0);
  const uint4* xv = (const uint4*)(x + sp.head) + v0;
  // the elements before and after the vectors: at most one per thread of the first CTA
  const int64_t scalar = rank != 0 ? -1 : tid < sp.head ? tid
                         : tid - sp.head < sp.tail ? sp.head + sp.nvec * N + tid - sp.head : -1;
  // slot i of a thread is slots[i blockDim + thread]
  const uint4* mine = slots + threadIdx.x;
  // the row's single values, under way with the vectors; a target past the
  // last column has no log-probability: NaN, so that the mistake shows
  float xy = NAN, adv = 0.f, old = 0.f, ref = 0.f;
  T xs = Vec<T>::put(0.f);
  // a small policy batch: no kernel before this one has taken the weights, and
  // none after it will add up the terms
  const bool alone = MODE == kPolicy && a.p.weight == nullptr;
  float share = 0.f;
  Stat st{-INFINITY, 0.f};
  if (live) {
    int ahead = tid;   // next vector to be loaded
    auto load = [&](int slot) {
#pragma unroll
      for (int q = 0; q < 4; ++q, ahead += nthr)
        if (ahead < n) copy_async(tc::smem_u32(mine + (slot * 4 + q) * blockDim.x), xv + ahead);
      copy_commit();
    };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) load(d);
    if (scalar >= 0) xs = x[scalar];
    if (y < a.V) xy = Vec<T>::get(x[y]);
    if (a.p.ref != nullptr) ref = a.p.ref[t];
    if (MODE == kPolicy) {
      adv = a.p.adv[t];
      old = a.p.old[t];
      if (alone && WARP) share = weight_of(a.y, a.p.offsets, a.T, a.p.S, t);
      if (alone && !WARP && warp == (int)blockDim.x / 32 - 1) {   // (the first warp has the rest to do)
        share = weight_of(a.y, a.p.offsets, a.T, a.p.S, t);
        if (lane == 0) shared_share = share;
      }
    }
    Running<T, WARP ? 4 : 16> run;
    int d = 0;
    for (int i = tid; i < n; i += 4 * nthr) {
      copy_wait<DEPTH - 1>();
      if (i + 3 * nthr < n)
        run.add([&](int q) { return mine[(d * 4 + q) * blockDim.x]; }, a.c);
      else   // -inf past the end of the run
        run.add([&](int q) { return i + q * nthr < n ? mine[(d * 4 + q) * blockDim.x] : Vec<T>::none(); }, a.c);
      if (KEEP) {
        copy_commit();
        ++d;
      } else {
        load(d);
        if (++d == DEPTH) d = 0;
      }
    }
    if (scalar >= 0) run.add(Vec<T>::get(xs), a.c);
    st = merge_lanes<32>(run.s, a.c);
  }
  auto weight = [&] {
    if (alone) return WARP ? share : shared_share;
    asm volatile("griddepcontrol.wait;" ::: "memory");   // the weights are the previous kernel's
    return a.p.weight[t];
  };
  // Rows left out have not waited.  Where all are, the grid would be over before the
  // weights' kernel, which still writes to a workspace that the caller may reuse.
  auto finish = [] { asm volatile("griddepcontrol.wait;" ::: "memory"); };
  bool last = false;   // the batch's last row
  Slope d;
  if constexpr (WARP) {
    const RowOut o = row_out<MODE>(a, live, xy, adv, old, ref, weight, st);
    if (lane == 0) {
      write_row<MODE>(a, t, o, st);
      if (alone) {
        __threadfence();
        last = atomicAdd(a.done, 1u) == (unsigned)a.T - 1;
      }
    }
    last = __shfl_sync(0xffffffffu, last, 0);
    if (last) sum_terms<32>(a, nullptr);
    if (MODE == kStats) return;
    if (a.grad == nullptr) {
      finish();
      return;
    }
    d = slope_of<T>(live, o.coef, st, a.inv_temp, a.c);
  } else {
    if (lane == 0) red[warp] = st;
    __syncthreads();
    if (warp == 0) st = merge_lanes<16>(lane < (int)(blockDim.x / 32) ? red[lane] : Stat{-INFINITY, 0.f}, a.c);
    if (csize > 1) {   // every CTA writes its pair to all of them
      cluster_wait();
      if (threadIdx.x < csize) {
        uint32_t to;
        asm("mapa.shared::cluster.u32 %0, %1, %2;"
            : "=r"(to)
            : "r"((uint32_t)__cvta_generic_to_shared(peers + rank)), "r"(threadIdx.x));
        asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(st.m), "f"(st.S) : "memory");
      }
      __syncwarp();
      cluster_arrive();
      cluster_wait();
      if (warp == 0) st = merge_lanes<8>(lane < (int)csize ? peers[lane] : Stat{-INFINITY, 0.f}, a.c);
    }
    if (warp == 0) {
      const RowOut o = row_out<MODE>(a, live, xy, adv, old, ref, weight, st);
      if (threadIdx.x == 0) {
        shared_last = 0;
        if (rank == 0) {
          write_row<MODE>(a, t, o, st);
          if (alone) {
            __threadfence();
            shared_last = atomicAdd(a.done, 1u) == (unsigned)a.T - 1;
          }
        }
        if (MODE == kPolicy) shared_slope = slope_of<T>(live, o.coef, st, a.inv_temp, a.c);
      }
    }
    if (MODE == kStats) return;
    __syncthreads();
    if (shared_last) sum_terms<0>(a, dred);
    if (a.grad == nullptr) {
      finish();
      return;
    }
    d = shared_slope;
  }
  T* g = (T*)a.grad + t * a.gld;
  const int64_t target = y - sp.head - v0 * N;
  if (KEEP)   // (a thread writes the vectors that it holds)
    write_slope<T>(mine, n, tid, nthr, g + sp.head + v0 * N, d, a.c, target, a.same_phase, blockDim.x);
  else
    write_slope<T>(xv + tid, n, tid, nthr, g + sp.head + v0 * N, d, a.c, target, a.same_phase, nthr);
  if (scalar >= 0) g[scalar] = Vec<T>::put(d.zero ? 0.f : slope_at(xs, d, a.c, scalar == y));
  if (MODE == kPolicy) finish();
}

// The policy loss with its gradient for batches that fill the GPU: one
// persistent CTA per SM (each cluster takes every so many rows), whose warps
// share the work of a row so that no part of it waits for another row's:
//   producer   (1 warp)  keeps the next vectors coming into a ring of
//                        shared-memory slots by bulk copies
//   summing    (8 warps) the row's maximum and sum
//   scalar     (1 warp)  merges the warps' and the cluster's pairs, takes the
//                        row's terms and its slope
//   writing    (8 warps) the gradient from the slots, which it then frees
// The ring has to hold a CTA's whole run of a row.
// Bound by HBM and the ring's turnover: 4096 rows of 139,255 bf16 columns, a
// tenth of them left out, take 395 us with the two small kernels beside it, 5.5
// TB/s or 0.81 of a plain copy's rate (rows kept in registers: 586 us; two CTAs
// per SM with half the ring each: 743 us; 12 + 12 warps spill).
constexpr int kSlotVec = 1024, kSlots = 13;          // 16 KB each
constexpr int kGroup = 256, kGroupWarps = kGroup / 32;
constexpr int kScalarWarp = 2 * kGroupWarps, kProducerWarp = kScalarWarp + 1;
constexpr int kStreamThreads = (kProducerWarp + 1) * 32;
constexpr int kSlopes = 4;                           // rows between the scalar and the writing warps
constexpr size_t kRingBytes = (size_t)kSlots * kSlotVec * 16;

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}
// The test of a phase that other CTAs of the cluster complete: what they sent is seen
// after an acquire of the cluster's scope (the plain test acquires within the CTA).
__device__ __forceinline__ bool try_wait_cluster(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// Bounded wait (2 s); false once any wait of this CTA has run out.
template <bool CLUSTER = false>
__device__ __forceinline__ bool ring_wait(uint32_t bar, uint32_t parity, volatile int* stop) {
  auto done = [&] { return CLUSTER ? try_wait_cluster(bar, parity) : tc::mbar_try_wait(bar, parity); };
  if (done()) return true;
  const uint64_t t0 = tc::globaltimer_ns();
  while (!done()) {
    if (*stop) return false;
    if (tc::globaltimer_ns() - t0 > tc::kTimeoutNs) {
      *stop = 1;
      return false;
    }
  }
  return true;
}

template <class T>
__global__ void __launch_bounds__(kStreamThreads, 1) policy_stream_kernel(const __grid_constant__ Rows a) {
  constexpr int N = Vec<T>::N;
  extern __shared__ __align__(128) uint4 ring[];
  __shared__ __align__(8) uint64_t bars[2 * kSlots + 4 + 2 * kSlopes + 2];
  __shared__ Stat red[2][kGroupWarps], peers[2][8];
  __shared__ Slope slopes[kSlopes];
  __shared__ int stop_flag;
  volatile int* stop = &stop_flag;
  const uint32_t b_full = tc::smem_u32(bars), b_empty = b_full + 8 * kSlots;   // slots
  const uint32_t b_sum = b_empty + 8 * kSlots, b_sumfree = b_sum + 16;         // pairs of the summing warps
  const uint32_t b_slope = b_sumfree + 16, b_slopefree = b_slope + 8 * kSlopes;
  const uint32_t b_peers = b_slopefree + 8 * kSlopes;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned csize, rank;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(csize));
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  if (threadIdx.x == 0) {
    for (int i = 0; i < kSlots; ++i) {
      tc::mbar_init(b_full + 8 * i, 1);
      tc::mbar_init(b_empty + 8 * i, kGroupWarps);
    }
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(b_sum + 8 * i, kGroupWarps);
      tc::mbar_init(b_sumfree + 8 * i, 1);
      tc::mbar_init(b_peers + 8 * i, 1);
    }
    for (int i = 0; i < kSlopes; ++i) {
      tc::mbar_init(b_slope + 8 * i, 1);
      tc::mbar_init(b_slopefree + 8 * i, kGroupWarps);
    }
    stop_flag = 0;
    tc::fence_mbar_init();
  }
  __syncthreads();
  if (csize > 1) {   // a peer's barriers exist before anything is sent to them
    cluster_arrive();
    cluster_wait();
  }
  const int64_t t0 = blockIdx.x / csize, step = gridDim.x / csize;
  int slot = 0;
  uint32_t phase = 0;          // of the slot's next use
  uint32_t k = 0;              // live rows so far
  int64_t next = t0 < a.T ? a.y[t0] : -1;
  auto advance = [&] {
    if (++slot == kSlots) {
      slot = 0;
      phase ^= 1u;
    }
  };
  const bool sums = warp < kGroupWarps, writes = warp >= kGroupWarps && warp < 2 * kGroupWarps;
  int64_t issued = 0;
  if (warp == kScalarWarp) asm volatile("griddepcontrol.wait;" ::: "memory");   // the weights are the previous kernel's
  for (int64_t t = t0; t < a.T; t += step) {
    const int64_t y = next;
    if (t + step < a.T) next = a.y[t + step];
    const bool live = y >= 0;
    const T* x = (const T*)a.x + t * a.ld;
    const Span sp = span_of(x, a.V);
    // this CTA's run of the row, and the elements outside of the vectors (the first CTA's)
    const int64_t v0 = min(sp.nvec, rank * a.each);
    const int n = (int)min(a.each, sp.nvec - v0);
    const uint4* xv = (const uint4*)(x + sp.head) + v0;
    const int tid = threadIdx.x & (kGroup - 1);
    const int64_t scalar = rank != 0 ? -1 : tid < sp.head ? tid
                           : tid - sp.head < sp.tail ? sp.head + sp.nvec * N + tid - sp.head : -1;
    bool ok = true;
    if (sums) {
      if (!live) continue;
      Running<T> run;
      const float xs = scalar >= 0 ? Vec<T>::get(x[scalar]) : -INFINITY;
      for (int c = 0; c < n; c += kSlotVec) {
        if (!(ok = ring_wait(b_full + 8 * slot, phase, stop))) break;
        const uint4* v = ring + slot * kSlotVec + tid;
        const int left = n - c - tid;
        if (n - c >= kSlotVec) run.add([&](int q) { return v[q * kGroup]; }, a.c);
        else run.add([&](int q) { return left > q * kGroup ? v[q * kGroup] : Vec<T>::none(); }, a.c);   // -inf past its end
        advance();
      }
      if (scalar >= 0) run.add(xs, a.c);
      const Stat st = merge_lanes<32>(run.s, a.c);
      ok = ok && ring_wait(b_sumfree + 8 * (k & 1), ((k >> 1) & 1u) ^ 1u, stop);
      if (!__all_sync(0xffffffffu, ok)) break;
      if (lane == 0) {
        red[k & 1][warp] = st;
        tc::mbar_arrive(b_sum + 8 * (k & 1));
      }
    } else if (writes) {
      T* g = (T*)a.grad + t * a.gld;
      Slope d{};
      d.zero = true;
      T xs = Vec<T>::put(0.f);
      if (live) {
        if (scalar >= 0) xs = x[scalar];
        ok = ring_wait(b_slope + 8 * (k % kSlopes), (k / kSlopes) & 1u, stop);
        if (!__all_sync(0xffffffffu, ok)) break;
        d = slopes[k % kSlopes];
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(b_slopefree + 8 * (k % kSlopes));
        for (int c = 0; c < n; c += kSlotVec) {
          // A lane whose wait ran out stays with its warp, which meets below, to the row's end;
          // what it writes there counts for nothing.  A vote instead: 398.5
          // us for the case above, 395.9 without.
          ok = ring_wait(b_full + 8 * slot, phase, stop) && ok;
          const int64_t col = sp.head + (v0 + c) * N;
          write_slope<T>(ring + slot * kSlotVec + tid, min(kSlotVec, n - c), tid, kGroup, g + col, d, a.c, y - col,
                         a.same_phase, kGroup);
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(b_empty + 8 * slot);
          advance();
        }
        if (!__all_sync(0xffffffffu, ok)) break;
      } else {
        write_slope<T>(nullptr, n, tid, kGroup, g + sp.head + v0 * N, d, a.c, -1, a.same_phase, kGroup);
      }
      if (scalar >= 0) g[scalar] = Vec<T>::put(d.zero ? 0.f : slope_at(xs, d, a.c, scalar == y));
    } else if (warp == kScalarWarp) {
      float xy = NAN, adv = 0.f, old = 0.f, ref = 0.f, w = 0.f;
      Stat st{0.f, 1.f};
      bool room = true;   // for this row's slope
      if (live) {
        if (y < a.V) xy = Vec<T>::get(x[y]);
        adv = a.p.adv[t];
        old = a.p.old[t];
        w = a.p.weight[t];
        if (a.p.ref != nullptr) ref = a.p.ref[t];
        ok = __all_sync(0xffffffffu, ring_wait(b_sum + 8 * (k & 1), (k >> 1) & 1u, stop));
        st = merge_lanes<8>(lane < kGroupWarps ? red[k & 1][lane] : Stat{-INFINITY, 0.f}, a.c);
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(b_sumfree + 8 * (k & 1));
        if (!ok) st.m = st.S = NAN;   // a wait ran out: no result
        if (csize > 1) {              // every CTA sends its pair to all of them
          const uint32_t bar = b_peers + 8 * (k & 1);
          if (lane == 0) tc::mbar_expect_tx(bar, csize * (uint32_t)sizeof(Stat));
          __syncwarp();
          st.m = __shfl_sync(0xffffffffu, st.m, 0);
          st.S = __shfl_sync(0xffffffffu, st.S, 0);
          if (lane < (int)csize) {
            uint32_t to, tobar;
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(tc::smem_u32(&peers[k & 1][rank])), "r"(lane));
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(tobar) : "r"(bar), "r"(lane));
            asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(to),
                         "f"(st.m), "f"(st.S), "r"(tobar)
                         : "memory");
          }
          ok = __all_sync(0xffffffffu, ring_wait<true>(bar, (k >> 1) & 1u, stop)) && ok;
          st = merge_lanes<8>(lane < (int)csize ? peers[k & 1][lane] : Stat{-INFINITY, 0.f}, a.c);
          if (!ok) st.m = st.S = NAN;
        }
        room = __all_sync(0xffffffffu, ring_wait(b_slopefree + 8 * (k % kSlopes), ((k / kSlopes) & 1u) ^ 1u, stop));
      }
      const RowOut o = row_out<kPolicy>(a, live, xy, adv, old, ref, [&] { return w; }, st);
      if (lane == 0) {
        if (rank == 0) write_row<kPolicy>(a, t, o, st);
        if (live && room) {
          slopes[k % kSlopes] = slope_of<T>(live, o.coef, st, a.inv_temp, a.c);
          tc::mbar_arrive(b_slope + 8 * (k % kSlopes));
        }
      }
      __syncwarp();
    } else if (lane == 0) {
      if (!live) continue;
      for (int c = 0; c < n; c += kSlotVec) {
        if (!(ok = ring_wait(b_empty + 8 * slot, phase ^ 1u, stop))) break;
        const uint32_t bytes = min(kSlotVec, n - c) * 16u;
        tc::mbar_expect_tx(b_full + 8 * slot, bytes);
        bulk_load(tc::smem_u32(ring + slot * kSlotVec), xv + c, bytes, b_full + 8 * slot);
        ++issued;
        advance();
      }
      if (!ok) break;
    } else {
      break;   // the producer warp's other lanes
    }
    if (live) ++k;
  }
  if (warp == kProducerWarp && lane == 0 && *stop)   // the copies in flight end before shared memory goes away
    for (int64_t q = issued > kSlots ? issued - kSlots : 0; q < issued; ++q) {
      const uint64_t from = tc::globaltimer_ns();
      while (!tc::mbar_try_wait(b_full + 8 * (int)(q % kSlots), (uint32_t)((q / kSlots) & 1)) &&
             tc::globaltimer_ns() - from < 100000000ull) {
      }
    }
  asm volatile("griddepcontrol.wait;" ::: "memory");   // rows left out have not waited
  __syncwarp();
  if (csize > 1) {   // no CTA's shared memory goes away while a peer may write to it
    cluster_arrive();
    cluster_wait();
  } else {
    __syncthreads();
  }
  if (*stop) {   // some rows have no gradient, whatever their terms: the loss says so
    if (threadIdx.x < 3) a.p.terms[threadIdx.x * a.T + t0] = NAN;
    if (csize > 1) {   // (a CTA whose wait ran out has not waited for what peers had sent it)
      const uint64_t from = tc::globaltimer_ns();
      while (tc::globaltimer_ns() - from < 100000ull) {
      }
    }
  }
}

// The sums of the policy rows' terms, in their order; a few microseconds of
// latency after the rows (batches of more than 1024 rows only).
__global__ void __launch_bounds__(1024) terms_kernel(const float* terms, int64_t T, float* stats) {
  __shared__ double red[32];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const float* v = terms + blockIdx.x * T;
  double s = 0.0;
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < T; i += blockDim.x) s += (double)v[i];
  s = block_sum(s, red);
  if (threadIdx.x == 0) stats[blockIdx.x] = (float)s;
}

struct Pairs {
  const int64_t* offsets;   // 2 P + 1
  int64_t P;
  double inv_pairs, beta, smoothing;
  int average;
  float *ratios, *margins;  // 2 P, P
  double* loss_of;          // P
  float* loss;
};

// The mean of the pairs' losses, by one CTA.
__device__ __forceinline__ void mean_loss(const Pairs& q, double* red) {
  double s = 0.0;
#pragma unroll 4
  for (int64_t i = threadIdx.x; i < q.P; i += blockDim.x) s += __ldcg(q.loss_of + i);
  s = block_sum(s, red);
  if (threadIdx.x == 0) *q.loss = (float)(s * q.inv_pairs);
}

// The sums of the log ratios of pair rows [at0, at1) and [at1, at2) and their
// numbers of live rows, by a warp or a CTA; every thread gets them.
template <int GROUP>
__device__ __forceinline__ void pair_sums(const Rows& a, const int64_t (&at)[3], double (&sum)[2], int (&n)[2],
                                          double (*red)[32], int (*count_of)[8]) {
  sum[0] = sum[1] = 0.0;
  n[0] = n[1] = 0;
  // both sequences together, so that their loads and sums overlap
#pragma unroll 4
  for (int64_t t = at[0] + threadIdx.x % GROUP; t < at[2]; t += GROUP) {
    const int64_t yt = a.y[t];
    const float d = a.gap[t];
    const bool live = yt >= 0, second = t >= at[1];
    sum[0] += live && !second ? (double)d : 0.0;
    sum[1] += live && second ? (double)d : 0.0;
    n[0] += live && !second;
    n[1] += live && second;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const double s0 = __shfl_xor_sync(0xffffffffu, sum[0], o), s1 = __shfl_xor_sync(0xffffffffu, sum[1], o);
    sum[0] += s0;
    sum[1] += s1;
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) n[k] = __reduce_add_sync(0xffffffffu, n[k]);
  if (GROUP != 32) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __syncthreads();
    if (lane == 0) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        red[k][warp] = sum[k];
        count_of[k][warp] = n[k];
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      sum[k] = 0.0;
      n[k] = 0;
      for (int w = 0; w < 8; ++w) {
        sum[k] += red[k][w];
        n[k] += count_of[k][w];
      }
    }
  }
}

// What a pair makes of them: with `write` its outputs; the coefficient of the
// rows of each sequence.
__device__ __forceinline__ float2 pair_out(const Pairs& q, int64_t p, const double (&sum)[2], const int (&n)[2],
                                           bool write) {
  double share[2] = {1.0, 1.0};
  if (q.average) {
#pragma unroll
    for (int k = 0; k < 2; ++k) share[k] = 1.0 / (double)max(n[k], 1);
  }
  const double ratio[2] = {sum[0] * share[0], sum[1] * share[1]};
  const double h = q.beta * (ratio[0] - ratio[1]);
  const float hf = (float)h;
  if (write) {
    // -log sigma(h) = max(-h, 0) + log(1 + e^-|h|), in fp32 from here on
    const float l = log1pf(expf(-fabsf(hf)));
    const double down = (double)(fmaxf(-hf, 0.f) + l), up = (double)(fmaxf(hf, 0.f) + l);
    q.ratios[2 * p] = (float)ratio[0];
    q.ratios[2 * p + 1] = (float)ratio[1];
    q.margins[p] = hf;
    q.loss_of[p] = q.smoothing > 0.0 ? (1.0 - q.smoothing) * down + q.smoothing * up : down;   // no 0 x inf
  }
  const double gain = q.beta * (q.smoothing - (double)(1.f / (1.f + expf(hf)))) * q.inv_pairs;
  return {(float)(gain * share[0]), (float)(-gain * share[1])};
}

// One warp (GROUP 32) or one CTA (GROUP 256) per pair: the two sequences' sums
// of log ratios, the margin, the pair's loss and the coefficient of each of its
// rows.  Latency is all there is to it, so long sequences get a CTA (16 pairs of
// 8191 rows: 216 us a call against 239 us by warps).  Without a gradient the CTA
// that finishes last takes the mean of the losses.
template <int GROUP>
__global__ void __launch_bounds__(256) pair_kernel(const __grid_constant__ Rows a, const __grid_constant__ Pairs q) {
  __shared__ double red[2][32];
  __shared__ int count_of[2][8];
  constexpr int per = 256 / GROUP;   // pairs at a time per CTA
  const int tid = threadIdx.x % GROUP;
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  for (int64_t p = (int64_t)blockIdx.x * per + threadIdx.x / GROUP; p < q.P; p += (int64_t)gridDim.x * per) {
    int64_t at[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) at[k] = border(q.offsets, 2 * p + k, a.T);
    double sum[2];
    int n[2];
    pair_sums<GROUP>(a, at, sum, n, red, count_of);
    const float2 g = pair_out(q, p, sum, n, tid == 0);
    if (a.grad != nullptr)
      for (int64_t t = at[0] + tid; t < at[2]; t += GROUP) a.coef[t] = a.y[t] < 0 ? 0.f : t < at[1] ? g.x : g.y;
  }
  if (a.grad == nullptr && last_cta(a.done)) mean_loss(q, red[0]);
}

// The coefficient of row t by one warp, and with `write`, where t is the first
// row of its pair, the pair's outputs.
__device__ __noinline__ float coef_of(const Rows& a, const Pairs& q, int64_t t, bool write) {
  const int lane = threadIdx.x & 31;
  unsigned in = 0;
  int64_t p0 = 0;
  for (; p0 < q.P; p0 += 32) {
    const int64_t p = p0 + lane;
    in = __ballot_sync(0xffffffffu, p < q.P && border(q.offsets, 2 * p, a.T) <= t && t < border(q.offsets, 2 * p + 2, a.T));
    if (in) break;
  }
  if (!in) return 0.f;   // outside of the sequences
  const int64_t p = p0 + __ffs(in) - 1;
  int64_t at[3];
#pragma unroll
  for (int k = 0; k < 3; ++k) at[k] = border(q.offsets, 2 * p + k, a.T);
  double sum[2];
  int n[2];
  pair_sums<32>(a, at, sum, n, nullptr, nullptr);
  const float2 g = pair_out(q, p, sum, n, write && t == at[0] && lane == 0);
  return t < at[1] ? g.x : g.y;
}

// The gradient rows from the statistics and coefficients of earlier kernels:
// one warp per row, or `pieces` CTAs per row of 4 vectors per thread.  The rows
// are taken from the last to the first: the statistics pass read those last,
// and part of them is still in L2.  Bound by HBM: with the statistics pass and
// the pairs between them 2048 rows of 139,255 bf16 columns take 267 us, 6.4 TB/s
// over the three passes or 0.94 of a plain copy's rate.  The first CTA takes the
// mean of the losses along, which nothing has to wait for.  ALONE (small
// batches): no kernel has dealt with the pairs; each row takes its coefficient
// from its pair's log ratios itself, and the last CTA takes the mean.
template <class T, bool WARP, bool ALONE>
__global__ void __launch_bounds__(256)
    grad_kernel(const __grid_constant__ Rows a, const __grid_constant__ Pairs q, unsigned pieces) {
  constexpr int N = Vec<T>::N, K = 4;
  __shared__ double red[32];
  __shared__ float row_coef;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (!ALONE && blockIdx.x == 0) mean_loss(q, red);
  const int64_t rows = WARP ? 8 : 1;
  const int64_t t = a.T - 1 - (WARP ? (int64_t)blockIdx.x * rows + (threadIdx.x >> 5) : blockIdx.x / pieces);
  const unsigned piece = WARP ? 0 : blockIdx.x % pieces;
  float coef = 0.f;
  if (ALONE) {
    if (blockIdx.x == 0) {   // pairs without rows
      const double sum[2] = {0.0, 0.0};
      const int n[2] = {0, 0};
      for (int64_t p = threadIdx.x; p < q.P; p += blockDim.x)
        if (border(q.offsets, 2 * p + 2, a.T) <= border(q.offsets, 2 * p, a.T)) pair_out(q, p, sum, n, true);
    }
    if (t >= 0 && (WARP || threadIdx.x < 32)) coef = coef_of(a, q, t, piece == 0);
    if (!WARP) {
      if (threadIdx.x == 0) row_coef = coef;
      __syncthreads();
      coef = row_coef;
    }
  } else if (t >= 0) {
    coef = a.coef[t];
  }
  if (t >= 0) {
    const int64_t y = a.y[t];
    const Stat st = a.stats[t];
    const T* x = (const T*)a.x + t * a.ld;
    T* g = (T*)a.grad + t * a.gld;
    const Span sp = span_of(x, a.V);
    const uint4* xv = (const uint4*)(x + sp.head);
    const Slope d = slope_of<T>(y >= 0, coef, st, a.inv_temp, a.c);
    const int tid = WARP ? threadIdx.x & 31 : threadIdx.x, nthr = WARP ? 32 : blockDim.x;
    const int64_t first = (int64_t)piece * K * nthr;
    const int n = (int)(WARP ? sp.nvec : min((int64_t)K * nthr, sp.nvec - first));
    const int64_t col = sp.head + first * N;
    write_slope<T>(xv + first + tid, n, tid, nthr, g + col, d, a.c, y - col, a.same_phase, nthr);
    if (piece == 0) {
      const int64_t scalar = tid < sp.head ? tid
                             : tid - sp.head < sp.tail ? sp.head + sp.nvec * N + tid - sp.head : -1;
      if (scalar >= 0) g[scalar] = Vec<T>::put(d.zero ? 0.f : slope_at(x[scalar], d, a.c, scalar == y));
    }
  }
  if (ALONE) {
    if (last_cta(a.done)) mean_loss(q, red);
  }
}

// Each row's share of the policy loss: 1 / (live rows), or 1 / (sequences x
// live rows of its sequence); 0 for rows outside every sequence.  One CTA: the
// rows' sums run beside it (4096 rows: hidden).
__global__ void __launch_bounds__(1024)
    weight_kernel(const int64_t* y, const int64_t* offsets, int64_t T, int64_t S, float* weight) {
  __shared__ double red[32];
  // the rows' statistics do not need the weights, and the logits are older than this kernel
  asm volatile("griddepcontrol.launch_dependents;");
  if (offsets == nullptr) {
    int64_t count = 0;
#pragma unroll 8
    for (int64_t t = threadIdx.x; t < T; t += blockDim.x) count += y[t] >= 0;
    const double n = block_sum((double)count, red);
    const float w = (float)(1.0 / fmax(n, 1.0));
    for (int64_t t = threadIdx.x; t < T; t += blockDim.x) weight[t] = w;
    return;
  }
  for (int64_t t = threadIdx.x; t < T; t += blockDim.x) weight[t] = 0.f;
  __syncthreads();
  const int lane = threadIdx.x & 31;
  for (int64_t k = threadIdx.x >> 5; k < S; k += blockDim.x / 32) {
    const int64_t a = border(offsets, k, T), b = border(offsets, k + 1, T);
    int64_t n = 0;
    for (int64_t t = a + lane; t < b; t += 32) n += y[t] >= 0;
    const double live = warp_sum((double)n);
    const float w = (float)(1.0 / ((double)S * fmax(live, 1.0)));
    for (int64_t t = a + lane; t < b; t += 32) weight[t] = w;
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
int num_sms() {
  static std::atomic<int> sms[kMaxDevices];
  return per_device(sms, [] {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
      return 0;
    return n;
  });
}

// Launches `kernel`; with `overlap` it may start before the kernel ahead of it
// in the stream has finished (it waits for that one itself, where it needs it).
template <class... P, class... A>
cudaError_t launch(void (*kernel)(P...), int64_t grid, int block, size_t smem, unsigned cluster, bool overlap,
                   cudaStream_t s, const A&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3((unsigned)block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2]{};
  int n = 0;
  if (cluster > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = cluster;
    attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
    ++n;
  }
  if (overlap) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n].val.programmaticStreamSerializationAllowed = 1;
    ++n;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

constexpr int kMaxKeep = 220 * 1024;   // shared memory of a run that is kept

// The same with up to kMaxKeep of dynamic shared memory.
template <class... P, class... A>
cudaError_t launch_row(void (*kernel)(P...), size_t smem, int64_t grid, int block, unsigned cluster, bool overlap,
                       cudaStream_t s, const A&... args) {
  if (smem > 40 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxKeep);
    if (e != cudaSuccess) return e;
  }
  return launch(kernel, grid, block, smem, cluster, overlap, s, args...);
}

// The statistics pass, or a policy batch without its gradient.
template <class T, int MODE>
cudaError_t launch_sums(Rows a, int64_t nvec, int sms, cudaStream_t s) {
  const bool late = MODE == kPolicy && a.p.weight != nullptr;   // the weights' kernel is ahead of it
  // A warp per row of up to 8192 16-bit columns where there are rows enough (at
  // V = 4096: 61 us against 113 us for 48,828 rows by CTAs of 128 threads).
  if (nvec <= 256 || (nvec <= 1024 && a.T >= 16 * sms))
    return launch_row(row_kernel<T, true, MODE, 2, false>, 32 * 1024, (a.T + 7) / 8, 256, 1, late, s, a);
  // A CTA per row, and clusters of up to eight where there are too few to fill the SMs
  int64_t cs = 1;
  while (cs < 8 && a.T * cs < 2 * sms && nvec >= cs * 2 * 256) cs *= 2;
  int block = nvec > 8192 && a.T >= 8 * sms ? 256 : 128;   // (V = 139,255, 4096 rows: 166 us against 172 us)
  if (a.T * cs < 2 * sms) {
    block = 512;
    while (block > 64 && (nvec + cs - 1) / cs < block) block /= 2;
  }
  a.each = (nvec + cs - 1) / cs;
  return launch_row(row_kernel<T, false, MODE, 2, false>, (size_t)block * 128, a.T * cs, block, (unsigned)cs, late, s, a);
}

// CTAs of a streaming cluster of rows of `nvec` vectors: one or two where their
// runs are at most nine of the ring's thirteen slots, else four or more, with
// runs of at most nine slots, or six of fp32, which is written as fast as it comes
// (V = 200,005, 2000 rows of bf16: 314 us by three CTAs, 286 by four; V =
// 139,255, 2000 rows of fp32: 359 us by four, 335 by six).
constexpr int64_t kMostCluster = 6;
int64_t stream_cluster(int64_t nvec, int es) {
  for (int64_t cs = 1; cs <= 2; ++cs)
    if (nvec <= cs * 9 * kSlotVec) return cs;
  for (int64_t cs = 4; cs < kMostCluster; ++cs)
    if (nvec <= cs * (es == 4 ? 6 : 9) * kSlotVec) return cs;
  return kMostCluster;
}
// whether a policy batch with its gradient streams: long rows, which six CTAs hold
// in twelve slots each, in batches that fill the GPU
bool streams(int64_t nvec, int es, int64_t T, int sms) {
  return nvec > 3072 && nvec <= kMostCluster * (kSlots - 1) * kSlotVec && T * stream_cluster(nvec, es) >= 4 * sms;
}

// A policy batch with its gradient.
template <class T>
cudaError_t launch_policy(Rows a, int64_t nvec, int sms, cudaStream_t s) {
  const bool late = a.p.weight != nullptr;   // the weights' kernel is ahead of it
  // a warp per row of up to 4096 16-bit columns (V = 4096, 48,828 rows: 195 us against 234 us by CTAs)
  if (nvec <= 256 || (nvec <= 513 && a.T >= 16 * sms)) {
    const int groups = (int)((nvec + 127) / 128);
    if (groups <= 2)
      return launch_row(row_kernel<T, true, kPolicy, 2, true>, groups * 16384, (a.T + 7) / 8, 256, 1, late, s, a);
    return launch_row(row_kernel<T, true, kPolicy, 8, true>, groups * 16384, (a.T + 7) / 8, 256, 1, late, s, a);
  }
  // Long rows in batches that fill the GPU: the streaming kernel (V = 32768, 6103
  // rows of bf16: 158 us against 161 us by clusters of row_kernel; V = 139255: 163
  // us against 171 us; V = 16384: 198 us against 153 us).
  int64_t cs = stream_cluster(nvec, sizeof(T));
  if (streams(nvec, sizeof(T), a.T, sms)) {
    static std::atomic<int> ready[kMaxDevices], room[kMostCluster + 1][kMaxDevices];
    if (!per_device(ready, [] {
          return cudaFuncSetAttribute(policy_stream_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                      (int)kRingBytes) == cudaSuccess ? 1 : 0;
        }))
      return cudaErrorInvalidValue;
    // as many clusters as run at the same time
    const int clusters = per_device(room[cs], [&] {
      cudaLaunchConfig_t cfg{};
      cudaLaunchAttribute at{};
      at.id = cudaLaunchAttributeClusterDimension;
      at.val.clusterDim.x = (unsigned)cs;
      at.val.clusterDim.y = at.val.clusterDim.z = 1;
      cfg.gridDim = dim3((unsigned)(sms / cs * cs));
      cfg.blockDim = dim3(kStreamThreads);
      cfg.dynamicSmemBytes = kRingBytes;
      cfg.attrs = &at;
      cfg.numAttrs = 1;
      int n = 0;
      return cudaOccupancyMaxActiveClusters(&n, policy_stream_kernel<T>, &cfg) == cudaSuccess ? n : 0;
    });
    if (clusters == 0) return cudaErrorInvalidValue;
    a.each = (nvec + cs - 1) / cs;
    return launch(policy_stream_kernel<T>, std::min<int64_t>(a.T, clusters) * cs, kStreamThreads, kRingBytes,
                  (unsigned)cs, late, s, a);
  }
  // A CTA per row, or a cluster with runs of 32 KB, or where the rows are too few to fill the SMs
  cs = nvec * 16 <= 48 * 1024 ? 1 : std::min<int64_t>(8, (nvec * 16 + 32767) / 32768);
  int block = 128;
  while (cs < 8 && a.T * cs < 2 * sms && nvec >= cs * 2 * 256) cs = std::min<int64_t>(8, cs * 2);
  if (a.T * cs < 2 * sms) {
    block = 512;
    while (block > 64 && (nvec + cs - 1) / cs < block) block /= 2;
  }
  a.each = (nvec + cs - 1) / cs;
  while (block < 512 && a.each > 32 * block) block *= 2;   // up to eight groups per thread are kept
  const int64_t groups = (a.each + 4 * block - 1) / (4 * block);
  const size_t smem = (size_t)block * 64 * groups;
  if (groups <= 2)
    return launch_row(row_kernel<T, false, kPolicy, 2, true>, smem, a.T * cs, block, (unsigned)cs, late, s, a);
  if (groups <= 8 && smem <= kMaxKeep)
    return launch_row(row_kernel<T, false, kPolicy, 8, true>, smem, a.T * cs, block, (unsigned)cs, late, s, a);
  // too long to be kept: read again
  return launch_row(row_kernel<T, false, kPolicy, 2, false>, (size_t)block * 128, a.T * cs, block, (unsigned)cs, late,
                    s, a);
}

template <class T, int MODE>
nmd_status launch_rows_t(Rows a, cudaStream_t s) {
  const int sms = num_sms();
  if (sms == 0) return NMD_ERR_CUDA;
  const int64_t nvec = a.V / Vec<T>::N + 1;
  a.each = nvec;
  cudaError_t e;
  if constexpr (MODE == kPolicy) e = a.grad ? launch_policy<T>(a, nvec, sms, s) : launch_sums<T, MODE>(a, nvec, sms, s);
  else e = launch_sums<T, MODE>(a, nvec, sms, s);
  return e == cudaSuccess ? NMD_OK : NMD_ERR_CUDA;
}

template <int MODE>
nmd_status launch_rows(int dtype, const Rows& a, cudaStream_t s) {
  switch (dtype) {
    case NMD_DT_FP32: return launch_rows_t<float, MODE>(a, s);
    case NMD_DT_BF16: return launch_rows_t<bf16, MODE>(a, s);
    default: return launch_rows_t<__half, MODE>(a, s);
  }
}

// CTAs of the gradient pass: `pieces` per row, or one for 8 rows (0 pieces)
unsigned grad_pieces(int64_t nvec, int64_t T, int sms) {
  return nvec <= 256 || (nvec <= 1024 && T >= 16 * sms) ? 0 : (unsigned)((nvec + 4 * 256 - 1) / (4 * 256));
}
// Whether the gradient pass deals with the pairs too: in small batches of short
// sequences, where all its CTAs run at the same time and each looks through few
// pairs and rows.  Such calls wait for the host, and a launch less is worth more
// than the row's own search (4 pairs, 160 rows of 4096 fp32 columns: 29 us a call
// against 36, of which the device works 12.0 against 10.6).
bool grad_alone(int64_t nvec, int64_t T, int64_t P, int sms) {
  const int64_t pieces = grad_pieces(nvec, T, sms);
  return T <= 1024 && P <= 128 && T <= 128 * P && (pieces ? T * pieces : (T + 7) / 8) <= 8 * sms;
}

template <class T>
nmd_status launch_grad_t(const Rows& a, const Pairs& q, bool alone, cudaStream_t s) {
  const int64_t nvec = a.V / Vec<T>::N;
  const int sms = num_sms();
  if (sms == 0) return NMD_ERR_CUDA;
  const unsigned pieces = grad_pieces(nvec, a.T, sms);
  cudaError_t e;
  if (pieces == 0)
    e = launch(alone ? grad_kernel<T, true, true> : grad_kernel<T, true, false>, (a.T + 7) / 8, 256, 0, 1, true, s, a, q,
               1u);
  else
    e = launch(alone ? grad_kernel<T, false, true> : grad_kernel<T, false, false>, a.T * pieces, 256, 0, 1, true, s, a, q,
               pieces);
  return e == cudaSuccess ? NMD_OK : NMD_ERR_CUDA;
}

nmd_status launch_grad(int dtype, const Rows& a, const Pairs& q, bool alone, cudaStream_t s) {
  switch (dtype) {
    case NMD_DT_FP32: return launch_grad_t<float>(a, q, alone, s);
    case NMD_DT_BF16: return launch_grad_t<bf16>(a, q, alone, s);
    default: return launch_grad_t<__half>(a, q, alone, s);
  }
}

int dtype_bytes(int dtype) { return dtype == NMD_DT_FP32 ? 4 : 2; }

constexpr int64_t kMaxRows = int64_t(1) << 27;   // rows x 8 CTAs within a grid

// Checks what the three losses share and fills the common arguments.
nmd_status fill(const void* x, int32_t dtype, int64_t T, int64_t V, int64_t ld, const int64_t* y, double temperature,
                float* logps, void* grad, int64_t gld, Rows* a) {
  if (dtype < NMD_DT_FP32 || dtype > NMD_DT_FP16 || T < 0 || T > kMaxRows || V < 1 || V >= (int64_t(1) << 31) ||
      ld < 0)
    return NMD_ERR_INVALID;
  Scale scale;
  if (!scale_of(temperature, &scale)) return NMD_ERR_INVALID;
  if (T > 0 && (!x || !y || !logps)) return NMD_ERR_INVALID;
  const int es = dtype_bytes(dtype);
  if (((uintptr_t)x | (uintptr_t)grad) & (uintptr_t)(es - 1)) return NMD_ERR_INVALID;
  *a = Rows{};
  a->x = x;
  a->T = T;
  a->V = V;
  a->ld = ld;
  a->y = y;
  a->c = scale;
  a->inv_temp = two_floats(1.0 / temperature);
  a->logps = logps;
  if (grad) {
    if (T > 0 && gld < V) return NMD_ERR_INVALID;
    if (T > 0) {   // the gradient may not overlap the logits
      const uintptr_t x0 = (uintptr_t)x, x1 = x0 + (size_t)((T - 1) * ld + V) * es;
      const uintptr_t g0 = (uintptr_t)grad, g1 = g0 + (size_t)((T - 1) * gld + V) * es;
      if (x0 < g1 && g0 < x1) return NMD_ERR_INVALID;
    }
    a->grad = grad;
    a->gld = gld;
    a->same_phase = ((uintptr_t)x & 15) == ((uintptr_t)grad & 15) && (T <= 1 || ((ld - gld) * es) % 16 == 0);
  }
  return NMD_OK;
}

bool policy_streams(int dtype, const Rows& a) {
  return a.grad != nullptr && streams(a.V * dtype_bytes(dtype) / 16 + 1, dtype_bytes(dtype), a.T, num_sms());
}

size_t align256(size_t v) { return (v + 255) & ~size_t(255); }

}  // namespace
}  // namespace nmd

using namespace nmd;

extern "C" {

nmd_status nmd_token_logprobs(const void* d_logits, int32_t dtype, int64_t T, int64_t V, int64_t ld,
                              const int64_t* d_targets, double temperature, float* d_logps, void* stream) {
  Rows a;
  const nmd_status st = fill(d_logits, dtype, T, V, ld, d_targets, temperature, d_logps, nullptr, 0, &a);
  if (st != NMD_OK || T == 0) return st;
  return launch_rows<kStats>(dtype, a, (cudaStream_t)stream);
}

nmd_status nmd_preference_workspace_bytes(int64_t T, int64_t P, size_t* bytes) {
  if (T < 0 || T > kMaxRows || P < 1 || P > kMaxRows || !bytes) return NMD_ERR_INVALID;
  *bytes = align256((size_t)T * sizeof(Stat)) + 2 * align256((size_t)T * sizeof(float)) +
           align256((size_t)P * sizeof(double)) + 256;
  return NMD_OK;
}

nmd_status nmd_preference_loss(const void* d_logits, int32_t dtype, int64_t T, int64_t V, int64_t ld,
                               const int64_t* d_targets, const int64_t* d_offsets, int64_t P,
                               const float* d_reference, double beta, double smoothing, int32_t average,
                               double temperature, float* d_loss, float* d_logps, float* d_ratios, float* d_margins,
                               void* d_grad, int64_t grad_ld, void* d_workspace, size_t ws_bytes, void* stream) {
  Rows a;
  nmd_status st = fill(d_logits, dtype, T, V, ld, d_targets, temperature, d_logps, d_grad, grad_ld, &a);
  if (st != NMD_OK) return st;
  size_t need = 0;
  if ((st = nmd_preference_workspace_bytes(T, P, &need)) != NMD_OK) return st;
  if (!d_offsets || (T > 0 && !d_reference) || !d_loss || !d_ratios || !d_margins || !std::isfinite(beta) ||
      !(smoothing >= 0.0 && smoothing < 1.0))
    return NMD_ERR_INVALID;
  if (!d_workspace || ws_bytes < need || ((uintptr_t)d_workspace & 255u)) return NMD_ERR_WORKSPACE;
  cudaStream_t s = (cudaStream_t)stream;
  char* w = (char*)d_workspace;
  a.stats = (Stat*)w;
  w += align256((size_t)T * sizeof(Stat));
  a.coef = (float*)w;
  w += align256((size_t)T * sizeof(float));
  a.gap = (float*)w;
  w += align256((size_t)T * sizeof(float));
  a.p.ref = d_reference;
  const Pairs q{d_offsets, P, 1.0 / (double)P, beta, smoothing, (int)average, d_ratios, d_margins, (double*)w, d_loss};
  a.done = (unsigned*)(w + align256((size_t)P * sizeof(double)));
  if (T > 0) {
    if ((st = launch_rows<kStats>(dtype, a, s)) != NMD_OK) return st;   // zeroes the count too
  } else {
    a.grad = nullptr;   // no rows: no gradient pass
    if (cudaMemsetAsync(a.done, 0, sizeof(unsigned), s) != cudaSuccess) return NMD_ERR_CUDA;
  }
  const bool alone = a.grad && grad_alone(V * dtype_bytes(dtype) / 16, T, P, num_sms());
  if (alone) return launch_grad(dtype, a, q, true, s);
  const bool large = T > 128 * P;   // long sequences
  const int64_t grid = std::min<int64_t>(large ? P : (P + 7) / 8, 1024);
  if (launch(large ? pair_kernel<256> : pair_kernel<32>, grid, 256, 0, 1, true, s, a, q) != cudaSuccess)
    return NMD_ERR_CUDA;
  return a.grad ? launch_grad(dtype, a, q, false, s) : NMD_OK;
}

nmd_status nmd_policy_workspace_bytes(int64_t T, size_t* bytes) {
  if (T < 0 || T > kMaxRows || !bytes) return NMD_ERR_INVALID;
  *bytes = align256((size_t)T * sizeof(float)) + align256((size_t)T * 3 * sizeof(float)) + 256;
  return NMD_OK;
}

nmd_status nmd_policy_loss(const void* d_logits, int32_t dtype, int64_t T, int64_t V, int64_t ld,
                           const int64_t* d_targets, const float* d_old, const float* d_reference,
                           const float* d_advantages, const int64_t* d_offsets, int64_t S, double clip_low,
                           double clip_high, double kl_coef, double temperature, float* d_stats, float* d_logps,
                           void* d_grad, int64_t grad_ld, void* d_workspace, size_t ws_bytes, void* stream) {
  Rows a;
  nmd_status st = fill(d_logits, dtype, T, V, ld, d_targets, temperature, d_logps, d_grad, grad_ld, &a);
  if (st != NMD_OK) return st;
  size_t need = 0;
  if ((st = nmd_policy_workspace_bytes(T, &need)) != NMD_OK) return st;
  if ((T > 0 && (!d_old || !d_advantages || (!d_reference && kl_coef != 0.0))) || !d_stats ||
      (d_offsets && (S < 1 || S > kMaxRows)) || !(clip_low >= 0.0 && clip_low <= 1.0) ||
      !(clip_high >= 0.0 && std::isfinite(clip_high)) || !(kl_coef >= 0.0 && std::isfinite(kl_coef)))
    return NMD_ERR_INVALID;
  cudaStream_t s = (cudaStream_t)stream;
  if (T == 0) return cudaMemsetAsync(d_stats, 0, 3 * sizeof(float), s) == cudaSuccess ? NMD_OK : NMD_ERR_CUDA;
  if (!d_workspace || ws_bytes < need || ((uintptr_t)d_workspace & 255u)) return NMD_ERR_WORKSPACE;
  char* w = (char*)d_workspace;
  float* weight = (float*)w;
  w += align256((size_t)T * sizeof(float));
  // up to 1024 rows one kernel does it all (and a cleared count): a launch costs more than the rows' counting
  const bool alone = T <= 1024 && !policy_streams(dtype, a);
  a.p = Policy{d_old, d_reference, d_advantages, alone ? nullptr : weight, (float)(1.0 - clip_low),
               (float)(1.0 + clip_high), (float)kl_coef, (float*)w, d_offsets, S, d_stats};
  a.done = (unsigned*)(w + align256((size_t)T * 3 * sizeof(float)));
  if (alone) {
    if (cudaMemsetAsync(a.done, 0, sizeof(unsigned), s) != cudaSuccess) return NMD_ERR_CUDA;
    return launch_rows<kPolicy>(dtype, a, s);
  }
  weight_kernel<<<1, 1024, 0, s>>>(d_targets, d_offsets, T, S, weight);
  if (cudaGetLastError() != cudaSuccess) return NMD_ERR_CUDA;
  if ((st = launch_rows<kPolicy>(dtype, a, s)) != NMD_OK) return st;
  return launch(terms_kernel, 3, 1024, 0, 0, true, s, (const float*)a.p.terms, T, d_stats) == cudaSuccess
             ? NMD_OK : NMD_ERR_CUDA;
}

}  // extern "C"

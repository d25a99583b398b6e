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
// merged by (m1, S1) + (m2, S2) = (m, S1 2^(c (m1 - m)) + S2 2^(c (m2 - m)))
// in a fixed order.  All sums are fp32; the only rounding to fewer bits is that of
// the gradient to the logits' type, once, when it is stored.
//
// Everything here is bound by HBM: a row is read once (twice where the
// gradient's coefficient depends on other rows) and its gradient written once.
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include "nmd_internal.cuh"

namespace nmd {
namespace {

namespace cg = cooperative_groups;

constexpr double kLog2e = 1.4426950408889634074;

// 2^x by the SFU (relative error about 2^-22; results below 2^-126 become 0,
// which no sum of probabilities can tell from the exact value)
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 16-byte vectors of the three element types
template <class T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[4]) {
    f[0] = __uint_as_float(v.x);
    f[1] = __uint_as_float(v.y);
    f[2] = __uint_as_float(v.z);
    f[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
  static __device__ __forceinline__ float get(float x) { return x; }
  static __device__ __forceinline__ float put(float x) { return x; }
};
template <>
struct Vec<bf16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *(const uint32_t*)&h;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ float get(bf16 x) { return __bfloat162float(x); }
  static __device__ __forceinline__ bf16 put(float x) { return __float2bfloat16_rn(x); }
};
template <>
struct Vec<__half> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 g = __half22float2(*(const __half2*)&w[i]);
      f[2 * i] = g.x;
      f[2 * i + 1] = g.y;
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2 h = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *(const uint32_t*)&h;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ float get(__half x) { return __half2float(x); }
  static __device__ __forceinline__ __half put(float x) { return __float2half_rn(x); }
};

// (m, S) of a set of elements: the maximum and the sum of 2^(c (x - m))
struct Stat {
  float m, S;
};
// -inf until a finite element has been seen: the sum is 0 and stays 0
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ Stat merge(const Stat& a, const Stat& b, float c) {
  const float m = fmaxf(a.m, b.m), z = base_of(m);
  return {m, a.S * ex2((a.m - z) * c) + b.S * ex2((b.m - z) * c)};
}
// adds the values f[0..N) to the pair
template <int N>
__device__ __forceinline__ void add(Stat& s, const float (&f)[N], float c) {
  float m = f[0];
#pragma unroll
  for (int i = 1; i < N; ++i) m = fmaxf(m, f[i]);
  if (m > s.m) {
    s.S *= ex2((s.m - m) * c);
    s.m = m;
  }
  const float z = base_of(s.m);
  float t = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) t += ex2((f[i] - z) * c);
  s.S += t;
}

struct Policy {
  const float* old;      // T: log-probabilities under the policy that produced the tokens
  const float* ref;      // T, or nullptr
  const float* adv;      // T
  const float* weight;   // T: each row's share of the loss
  float lo, hi, kl;      // 1 - clip_low, 1 + clip_high, KL coefficient
  float* terms;          // 3 T: weighted loss, KL, cut-off terms
};

struct Rows {
  const void* x;
  int64_t T, V, ld;
  const int64_t* y;
  float c, inv_temp;
  float* logps;          // T
  Stat* stats;           // T (the statistics pass writes, the gradient pass reads) or nullptr
  float* coef;           // T: g_t; zeroed by the statistics pass
  void* grad;            // T x V with row stride gld, or nullptr
  int64_t gld;
  int same_phase;        // rows of x and grad start at the same offset from a 16-byte boundary
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

enum { kStats = 0, kPolicy = 1, kGrad = 2 };

// One group of threads per row: a warp (GROUP 32), or a CTA or cluster of
// CTAs (GROUP 0; the cluster shares one row).
template <class T, int GROUP, int MODE>
__global__ void __launch_bounds__(512) row_kernel(const Rows a) {
  constexpr int N = Vec<T>::N;
  __shared__ Stat red[16];
  __shared__ Stat cred;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t t;
  int64_t tid, nthr;
  unsigned csize = 1;
  if constexpr (GROUP == 32) {
    t = (int64_t)blockIdx.x * (blockDim.x / 32) + warp;
    if (t >= a.T) return;
    tid = lane;
    nthr = 32;
  } else {
    csize = cg::this_cluster().num_blocks();
    t = blockIdx.x / csize;
    tid = (int64_t)(blockIdx.x % csize) * blockDim.x + threadIdx.x;
    nthr = (int64_t)csize * blockDim.x;
  }
  const int64_t y = a.y[t];
  const T* x = (const T*)a.x + t * a.ld;
  T* g = (T*)a.grad + t * a.gld;
  const Span sp = span_of(x, a.V);
  const uint4* xv = (const uint4*)(x + sp.head);
  // the row's scalar elements: at most one per thread
  const int64_t scalar = tid < sp.head ? tid : (tid - sp.head < sp.tail ? sp.head + sp.nvec * N + tid - sp.head : -1);

  Stat st{-INFINITY, 0.f};
  float coef = 0.f;
  const bool live = y >= 0;
  if (MODE == kStats && tid == 0 && a.coef != nullptr) a.coef[t] = 0.f;
  if (MODE != kGrad && live) {
    constexpr int U = 32 / N;   // vectors in flight per thread
    int64_t i = tid;
    for (; i + (U - 1) * nthr < sp.nvec; i += U * nthr) {
      uint4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = xv[i + u * nthr];
      float f[U * N];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float h[N];
        Vec<T>::unpack(v[u], h);
#pragma unroll
        for (int k = 0; k < N; ++k) f[u * N + k] = h[k];
      }
      add(st, f, a.c);
    }
    for (; i < sp.nvec; i += nthr) {
      float f[N];
      Vec<T>::unpack(xv[i], f);
      add(st, f, a.c);
    }
    if (scalar >= 0) {
      float f[1] = {Vec<T>::get(x[scalar])};
      add(st, f, a.c);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const Stat other{__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.S, o)};
      st = merge(st, other, a.c);
    }
    if constexpr (GROUP != 32) {
      if (lane == 0) red[warp] = st;
      __syncthreads();
      st = lane < (int)(blockDim.x / 32) ? red[lane] : Stat{-INFINITY, 0.f};
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) {
        const Stat other{__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.S, o)};
        st = merge(st, other, a.c);
      }
      st.m = __shfl_sync(0xffffffffu, st.m, 0);
      st.S = __shfl_sync(0xffffffffu, st.S, 0);
      if (csize > 1) {
        cg::cluster_group cl = cg::this_cluster();
        if (threadIdx.x == 0) cred = st;
        cl.sync();
        st = lane < (int)csize ? *cl.map_shared_rank(&cred, lane) : Stat{-INFINITY, 0.f};
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) {
          const Stat other{__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.S, o)};
          st = merge(st, other, a.c);
        }
        st.m = __shfl_sync(0xffffffffu, st.m, 0);
        st.S = __shfl_sync(0xffffffffu, st.S, 0);
        cl.sync();   // the peers' copies stay until everybody has read them
      }
    }
  }
  if (MODE != kGrad) {
    float lp = 0.f;
    if (live) {
      // a target past the last column has no log-probability: NaN, so that the mistake shows
      lp = y < a.V ? (Vec<T>::get(x[y]) - st.m) * a.inv_temp - logf(st.S) : NAN;
    }
    if (tid == 0) {
      a.logps[t] = lp;
      if (a.stats != nullptr) a.stats[t] = st;
    }
    if (MODE == kPolicy) {
      float term = 0.f, kl = 0.f, cut = 0.f;
      if (live) {
        const Policy& p = a.p;
        const float w = p.weight[t], adv = p.adv[t];
        const float ratio = expf(lp - p.old[t]);
        const float bound = fminf(fmaxf(ratio, p.lo), p.hi);
        const bool off = (adv > 0.f && ratio > p.hi) || (adv < 0.f && ratio < p.lo);
        const float ra = ratio * adv, ba = bound * adv;
        term = -(ra < ba || ra != ra ? ra : ba);
        coef = off ? 0.f : -ra;
        if (p.ref != nullptr) {
          const float gap = p.ref[t] - lp;
          const float q = expm1f(gap);
          kl = q - gap;
          if (p.kl != 0.f) {
            term += p.kl * kl;
            coef -= p.kl * q;
          }
        }
        term *= w;
        kl *= w;
        coef *= w;
        cut = off ? w : 0.f;
      }
      if (tid == 0) {
        a.p.terms[t] = term;
        a.p.terms[a.T + t] = kl;
        a.p.terms[2 * a.T + t] = cut;
      }
    }
  } else {
    if (live) {
      coef = a.coef[t];
      st = a.stats[t];
    }
  }
  if (MODE == kStats || a.grad == nullptr) return;

  // the gradient row; a zero coefficient (a row left out or cut off) needs no logits
  const bool zero = !live || coef == 0.f;
  const float up = coef * a.inv_temp, down = -up / st.S, m = st.m;
  for (int64_t i = tid; i < sp.nvec; i += nthr) {
    float d[N];
    if (zero) {
#pragma unroll
      for (int k = 0; k < N; ++k) d[k] = 0.f;
    } else {
      float f[N];
      Vec<T>::unpack(xv[i], f);
      const int64_t at = y - (sp.head + i * N);
#pragma unroll
      for (int k = 0; k < N; ++k) d[k] = fmaf(down, ex2((f[k] - m) * a.c), k == at ? up : 0.f);
    }
    T* to = g + sp.head + i * N;
    if (a.same_phase) {
      *(uint4*)to = Vec<T>::pack(d);
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k) to[k] = Vec<T>::put(d[k]);
    }
  }
  if (scalar >= 0) {
    const float d = zero ? 0.f : fmaf(down, ex2((Vec<T>::get(x[scalar]) - m) * a.c), scalar == y ? up : 0.f);
    g[scalar] = Vec<T>::put(d);
  }
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

// One warp per pair: the two sequences' sums of log ratios, the margin, the
// pair's loss and the coefficient of each of its rows.
__global__ void __launch_bounds__(256)
    pair_kernel(const int64_t* y, const float* logps, const float* ref, const int64_t* offsets, int64_t T, int64_t P,
                double beta, double smoothing, int average, float* ratios, float* margins, double* pair_loss,
                float* coef) {
  const int64_t p = (int64_t)blockIdx.x * (blockDim.x / 32) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (p >= P) return;
  double ratio[2], share[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int64_t a = border(offsets, 2 * p + k, T), b = border(offsets, 2 * p + k + 1, T);
    double sum = 0.0, count = 0.0;
    for (int64_t t = a + lane; t < b; t += 32)
      if (y[t] >= 0) {
        sum += (double)logps[t] - (double)ref[t];
        count += 1.0;
      }
    sum = warp_sum(sum);
    count = warp_sum(count);
    share[k] = average && count > 1.0 ? 1.0 / count : 1.0;
    ratio[k] = sum * share[k];
  }
  const double h = beta * (ratio[0] - ratio[1]);
  // -log sigma(h) = max(-h, 0) + log(1 + e^-|h|)
  const double l = log1p(exp(-fabs(h)));
  const double down = fmax(-h, 0.0) + l, up = fmax(h, 0.0) + l;
  if (lane == 0) {
    ratios[2 * p] = (float)ratio[0];
    ratios[2 * p + 1] = (float)ratio[1];
    margins[p] = (float)h;
    pair_loss[p] = smoothing > 0.0 ? (1.0 - smoothing) * down + smoothing * up : down;   // no 0 x inf
  }
  if (coef == nullptr) return;
  const double slope = beta * (smoothing - 1.0 / (1.0 + exp(h))) / (double)P;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int64_t a = border(offsets, 2 * p + k, T), b = border(offsets, 2 * p + k + 1, T);
    const float g = (float)((k ? -slope : slope) * share[k]);
    for (int64_t t = a + lane; t < b; t += 32) coef[t] = y[t] >= 0 ? g : 0.f;
  }
}

// out[k] = scale sum_i v[k n + i], k < gridDim.x
template <class T>
__global__ void __launch_bounds__(1024) sum_kernel(const T* v, int64_t n, double scale, float* out) {
  __shared__ double red[32];
  v += (int64_t)blockIdx.x * n;
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += blockDim.x) s += (double)v[i];
  s = block_sum(s, red);
  if (threadIdx.x == 0) out[blockIdx.x] = (float)(s * scale);
}

// Each row's share of the policy loss: 1 / (live rows), or 1 / (sequences x
// live rows of its sequence); 0 for rows outside every sequence.
__global__ void __launch_bounds__(1024)
    weight_kernel(const int64_t* y, const int64_t* offsets, int64_t T, int64_t S, float* weight) {
  __shared__ double red[32];
  if (offsets == nullptr) {
    double n = 0.0;
    for (int64_t t = threadIdx.x; t < T; t += blockDim.x) n += y[t] >= 0 ? 1.0 : 0.0;
    n = block_sum(n, red);
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

template <class T, int MODE>
nmd_status launch_rows_t(const Rows& a, cudaStream_t s) {
  if (a.T == 0) return NMD_OK;
  const int sms = num_sms();
  if (sms == 0) return NMD_ERR_CUDA;
  cudaError_t e;
  if (a.V <= 1024) {   // a warp per row
    row_kernel<T, 32, MODE><<<(unsigned)((a.T + 7) / 8), 256, 0, s>>>(a);
    e = cudaGetLastError();
  } else {
    // a CTA per row, or a cluster where there are too few rows to fill the
    // SMs and each CTA still gets two vectors per thread
    unsigned cs = 1;
    while (cs < 8 && a.T * cs < 2 * sms && a.V >= (int64_t)cs * 4 * 512 * Vec<T>::N) cs *= 2;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(a.T * cs));
    cfg.blockDim = dim3(512);
    cfg.stream = s;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = cs;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, row_kernel<T, 0, MODE>, a);
  }
  return e == cudaSuccess ? NMD_OK : NMD_ERR_CUDA;
}

template <int MODE>
nmd_status launch_rows(int dtype, const Rows& a, cudaStream_t s) {
  switch (dtype) {
    case NMD_DT_FP32: return launch_rows_t<float, MODE>(a, s);
    case NMD_DT_BF16: return launch_rows_t<bf16, MODE>(a, s);
    case NMD_DT_FP16: return launch_rows_t<__half, MODE>(a, s);
  }
  return NMD_ERR_INVALID;
}

int dtype_bytes(int dtype) { return dtype == NMD_DT_FP32 ? 4 : 2; }

constexpr int64_t kMaxRows = int64_t(1) << 27;   // rows x 8 CTAs within a grid

// Checks what the three losses share and fills the common arguments.
nmd_status fill(const void* x, int32_t dtype, int64_t T, int64_t V, int64_t ld, const int64_t* y, double temperature,
                float* logps, void* grad, int64_t gld, Rows* a) {
  if (dtype < NMD_DT_FP32 || dtype > NMD_DT_FP16 || T < 0 || T > kMaxRows || V < 1 || V >= (int64_t(1) << 31) ||
      ld < 0 || !(temperature > 0.0) || !std::isfinite(temperature))
    return NMD_ERR_INVALID;
  const float c = (float)(kLog2e / temperature), it = (float)(1.0 / temperature);
  if (!(c > 0.f) || !std::isfinite(c) || !std::isfinite(it)) return NMD_ERR_INVALID;
  if (T > 0 && (!x || !y || !logps)) return NMD_ERR_INVALID;
  const int es = dtype_bytes(dtype);
  if (((uintptr_t)x | (uintptr_t)grad) & (uintptr_t)(es - 1)) return NMD_ERR_INVALID;
  *a = Rows{};
  a->x = x;
  a->T = T;
  a->V = V;
  a->ld = ld;
  a->y = y;
  a->c = c;
  a->inv_temp = it;
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

size_t align256(size_t v) { return (v + 255) & ~size_t(255); }

}  // namespace
}  // namespace nmd

using namespace nmd;

extern "C" {

nmd_status nmd_token_logprobs(const void* d_logits, int32_t dtype, int64_t T, int64_t V, int64_t ld,
                              const int64_t* d_targets, double temperature, float* d_logps, void* stream) {
  Rows a;
  const nmd_status st = fill(d_logits, dtype, T, V, ld, d_targets, temperature, d_logps, nullptr, 0, &a);
  if (st != NMD_OK) return st;
  return launch_rows<kStats>(dtype, a, (cudaStream_t)stream);
}

nmd_status nmd_preference_workspace_bytes(int64_t T, int64_t P, size_t* bytes) {
  if (T < 0 || T > kMaxRows || P < 1 || P > kMaxRows || !bytes) return NMD_ERR_INVALID;
  *bytes = align256((size_t)T * sizeof(Stat)) + align256((size_t)T * sizeof(float)) + align256((size_t)P * sizeof(double));
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
  a.coef = (float*)(w + align256((size_t)T * sizeof(Stat)));
  double* pair_loss = (double*)(w + align256((size_t)T * sizeof(Stat)) + align256((size_t)T * sizeof(float)));
  if ((st = launch_rows<kStats>(dtype, a, s)) != NMD_OK) return st;
  pair_kernel<<<(unsigned)((P + 7) / 8), 256, 0, s>>>(d_targets, d_logps, d_reference, d_offsets, T, P, beta,
                                                      smoothing, average, d_ratios, d_margins, pair_loss,
                                                      d_grad ? a.coef : nullptr);
  sum_kernel<double><<<1, 1024, 0, s>>>(pair_loss, P, 1.0 / (double)P, d_loss);
  if (cudaGetLastError() != cudaSuccess) return NMD_ERR_CUDA;
  return d_grad ? launch_rows<kGrad>(dtype, a, s) : NMD_OK;
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
  if (!d_workspace || ws_bytes < need || ((uintptr_t)d_workspace & 255u)) return NMD_ERR_WORKSPACE;
  cudaStream_t s = (cudaStream_t)stream;
  char* w = (char*)d_workspace;
  float* weight = (float*)w;
  a.p = Policy{d_old, d_reference, d_advantages, weight, (float)(1.0 - clip_low), (float)(1.0 + clip_high),
               (float)kl_coef, (float*)(w + align256((size_t)T * sizeof(float)))};
  weight_kernel<<<1, 1024, 0, s>>>(d_targets, d_offsets, T, S, weight);
  if (cudaGetLastError() != cudaSuccess) return NMD_ERR_CUDA;
  if ((st = launch_rows<kPolicy>(dtype, a, s)) != NMD_OK) return st;
  sum_kernel<float><<<3, 1024, 0, s>>>(a.p.terms, T, 1.0, d_stats);
  return cudaGetLastError() == cudaSuccess ? NMD_OK : NMD_ERR_CUDA;
}

}  // extern "C"

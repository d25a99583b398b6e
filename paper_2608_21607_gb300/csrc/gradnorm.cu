// The global norm of a list of gradients and the gradients scaled to a
// largest norm:  norm = sqrt(sum_i sum_j g_ij^2),
//                out_ij = g_ij min(1, max_norm / norm).
//
// Two passes over the list, both bound by HBM: one reads every element for
// the norm, one reads it again and writes it scaled.  The scale stays on the
// device: every CTA of the second pass adds up the first pass's partial sums
// itself, in the same fixed order, so that no third launch and no counter is
// needed.  The list travels in the kernel's parameters (up to kTable tensors
// per launch), so that nothing is copied to the device first.
//
// Squares are summed in fp32 by each thread, in fp64 from there on.  So that
// no square leaves fp32's range, a vector of elements whose largest
// magnitude is above 2^56 or below 2^-50 is scaled by 2^-80 or 2^80 and summed
// apart; the three sums are put together in fp64, and norms over all of
// fp32's range come out right.
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include "nmd_internal.cuh"

namespace nmd {
namespace {

constexpr int kThreads = 256;
constexpr int kChunkBytes = 32768;     // one CTA's piece of a tensor at a time
constexpr int kMaxCtas = 2048;         // CTAs of the norm pass over all launches

template <int K>
struct Table {
  int count;
  int64_t chunks;            // of all entries
  const void* in[K];
  void* out[K];
  int64_t n[K];              // elements
  int64_t first[K];          // first chunk
  int dtype[K];
};

struct Sums {
  double mid, big, small;
};

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(bf16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float as_float(__half x) { return __half2float(x); }
__device__ __forceinline__ void from_float(float v, float* x) { *x = v; }
__device__ __forceinline__ void from_float(float v, bf16* x) { *x = __float2bfloat16_rn(v); }
__device__ __forceinline__ void from_float(float v, __half* x) { *x = __float2half_rn(v); }

// the squares of N values into one of the three sums
template <int N>
__device__ __forceinline__ void add_squares(const float (&f)[N], float (&acc)[3]) {
  float m = 0.f;
#pragma unroll
  for (int k = 0; k < N; ++k) m = fmaxf(m, fabsf(f[k]));
  const int which = m > 0x1p56f ? 1 : (m < 0x1p-50f ? 2 : 0);
  const float sc = which == 0 ? 1.f : (which == 1 ? 0x1p-80f : 0x1p80f);
  float t = 0.f;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const float v = f[k] * sc;
    t = fmaf(v, v, t);
  }
  acc[0] += which == 0 ? t : 0.f;
  acc[1] += which == 1 ? t : 0.f;
  acc[2] += which == 2 ? t : 0.f;
}

// Elements [e0, e1) of a tensor, walked by one CTA: f(i, N) is called with
// the first element of each 16-byte vector (N of them) and of each single
// element before and after them (1)
template <class T, class F>
__device__ __forceinline__ void walk(const T* x, int64_t e0, int64_t e1, F f) {
  constexpr int N = 16 / sizeof(T);
  const int off = (int)((uintptr_t)(x + e0) & 15);
  const int64_t n = e1 - e0;
  const int64_t h = off ? (16 - off) / (int)sizeof(T) : 0;
  const int head = (int)(h < n ? h : n);
  const int64_t nvec = (n - head) / N;
  const int tail = (int)(n - head - nvec * N);
  for (int64_t i = threadIdx.x; i < nvec; i += kThreads) f(e0 + head + i * N, true);
  const int t = threadIdx.x;
  if (t < head) f(e0 + t, false);
  else if (t - head < tail) f(e0 + head + nvec * N + t - head, false);
}

template <class T>
__device__ __forceinline__ void chunk_squares(const T* x, int64_t e0, int64_t e1, float (&acc)[3]) {
  constexpr int N = 16 / sizeof(T);
  walk(x, e0, e1, [&](int64_t i, bool vec) {
    if (vec) {
      const uint4 v = *(const uint4*)(x + i);
      const T* e = (const T*)&v;
      float f[N];
#pragma unroll
      for (int k = 0; k < N; ++k) f[k] = as_float(e[k]);
      add_squares(f, acc);
    } else {
      const float f[1] = {as_float(x[i])};
      add_squares(f, acc);
    }
  });
}

template <class T>
__device__ __forceinline__ void chunk_scale(const T* x, T* o, int64_t e0, int64_t e1, float scale) {
  constexpr int N = 16 / sizeof(T);
  const bool same = ((uintptr_t)x & 15) == ((uintptr_t)o & 15);
  walk(x, e0, e1, [&](int64_t i, bool vec) {
    if (vec) {
      const uint4 v = *(const uint4*)(x + i);
      const T* e = (const T*)&v;
      uint4 w;
      T* d = (T*)&w;
#pragma unroll
      for (int k = 0; k < N; ++k) from_float(as_float(e[k]) * scale, d + k);
      if (same) {
        *(uint4*)(o + i) = w;
      } else {
#pragma unroll
        for (int k = 0; k < N; ++k) o[i + k] = d[k];
      }
    } else {
      from_float(as_float(x[i]) * scale, o + i);
    }
  });
}

// the entry that holds chunk c: the last whose first chunk is not past c
template <int K>
__device__ __forceinline__ int entry_of(const Table<K>& t, int64_t c) {
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= c) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ double cta_sum(double v, double* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = red[threadIdx.x & (kThreads / 32 - 1)];
#pragma unroll
  for (int o = kThreads / 64; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

template <int K>
__global__ void __launch_bounds__(kThreads) norm_kernel(const __grid_constant__ Table<K> tab, Sums* parts) {
  __shared__ double red[kThreads / 32];
  float acc[3] = {0.f, 0.f, 0.f};
  for (int64_t c = blockIdx.x; c < tab.chunks; c += gridDim.x) {
    const int e = entry_of(tab, c);
    const int es = tab.dtype[e] == NMD_DT_FP32 ? 4 : 2;
    const int64_t e0 = (c - tab.first[e]) * (kChunkBytes / es);
    const int64_t e1 = min(tab.n[e], e0 + kChunkBytes / es);
    if (tab.dtype[e] == NMD_DT_FP32) chunk_squares((const float*)tab.in[e], e0, e1, acc);
    else if (tab.dtype[e] == NMD_DT_BF16) chunk_squares((const bf16*)tab.in[e], e0, e1, acc);
    else chunk_squares((const __half*)tab.in[e], e0, e1, acc);
  }
  Sums s;
  s.mid = cta_sum((double)acc[0], red);
  s.big = cta_sum((double)acc[1], red);
  s.small = cta_sum((double)acc[2], red);
  if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

template <int K>
__global__ void __launch_bounds__(kThreads)
    scale_kernel(const __grid_constant__ Table<K> tab, const Sums* parts, int nparts, double max_norm, int in_place,
                 float* norm_out) {
  __shared__ double red[kThreads / 32];
  double mid = 0.0, big = 0.0, small = 0.0;
  for (int i = threadIdx.x; i < nparts; i += kThreads) {
    mid += parts[i].mid;
    big += parts[i].big;
    small += parts[i].small;
  }
  const double norm = sqrt(cta_sum(mid, red) + cta_sum(big, red) * 0x1p160 + cta_sum(small, red) * 0x1p-160);
  if (norm_out != nullptr && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
  // a norm that is not a number makes every gradient so
  const float scale = norm <= max_norm ? 1.f : (float)(max_norm / norm);
  if (in_place && scale == 1.f) return;
  for (int64_t c = blockIdx.x; c < tab.chunks; c += gridDim.x) {
    const int e = entry_of(tab, c);
    const int es = tab.dtype[e] == NMD_DT_FP32 ? 4 : 2;
    const int64_t e0 = (c - tab.first[e]) * (kChunkBytes / es);
    const int64_t e1 = min(tab.n[e], e0 + kChunkBytes / es);
    if (tab.dtype[e] == NMD_DT_FP32) chunk_scale((const float*)tab.in[e], (float*)tab.out[e], e0, e1, scale);
    else if (tab.dtype[e] == NMD_DT_BF16) chunk_scale((const bf16*)tab.in[e], (bf16*)tab.out[e], e0, e1, scale);
    else chunk_scale((const __half*)tab.in[e], (__half*)tab.out[e], e0, e1, scale);
  }
}

int sm_count() {
  static std::atomic<int> sms[kMaxDevices];
  return per_device(sms, [] {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
      return 0;
    return n;
  });
}

// One group of at most K tensors; empty ones take no chunk.
template <int K>
void fill(Table<K>& t, const void* const* in, void* const* out, const int64_t* n, const int32_t* dtype, int64_t k0,
          int64_t k1) {
  t.count = 0;
  t.chunks = 0;
  for (int64_t k = k0; k < k1; ++k) {
    if (n[k] == 0) continue;
    const int es = dtype[k] == NMD_DT_FP32 ? 4 : 2;
    const int i = t.count++;
    t.in[i] = in[k];
    t.out[i] = out ? out[k] : const_cast<void*>(in[k]);
    t.n[i] = n[k];
    t.dtype[i] = dtype[k];
    t.first[i] = t.chunks;
    t.chunks += (n[k] + kChunkBytes / es - 1) / (kChunkBytes / es);
  }
}

template <int K>
nmd_status run(int64_t count, const void* const* in, const int64_t* n, const int32_t* dtype, double max_norm,
               void* const* out, float* d_norm, Sums* parts, cudaStream_t s) {
  const int sms = sm_count();
  if (sms == 0) return NMD_ERR_CUDA;
  const int64_t groups = std::max<int64_t>(1, (count + K - 1) / K);
  // CTAs of each launch: the partial sums of all launches fit the workspace
  const int most = (int)std::max<int64_t>(1, std::min<int64_t>(sms * 8, kMaxCtas / groups));
  int nparts = 0;
  Table<K> t;
  for (int64_t g = 0; g < groups; ++g) {
    fill(t, in, out, n, dtype, g * K, std::min(count, (g + 1) * K));
    const int grid = (int)std::max<int64_t>(1, std::min<int64_t>(t.chunks, most));
    norm_kernel<K><<<grid, kThreads, 0, s>>>(t, parts + nparts);
    nparts += grid;
  }
  for (int64_t g = 0; g < groups; ++g) {
    if (groups > 1) fill(t, in, out, n, dtype, g * K, std::min(count, (g + 1) * K));
    const int grid = (int)std::max<int64_t>(1, std::min<int64_t>(t.chunks, sms * 8));
    scale_kernel<K><<<grid, kThreads, 0, s>>>(t, parts, nparts, max_norm, out == nullptr, g == 0 ? d_norm : nullptr);
  }
  return cudaGetLastError() == cudaSuccess ? NMD_OK : NMD_ERR_CUDA;
}

// tensors per launch: the table is copied with every launch, so short lists take a small one
constexpr int kSmallTable = 16, kTable = 512;

}  // namespace
}  // namespace nmd

using namespace nmd;

extern "C" {

nmd_status nmd_clip_workspace_bytes(int64_t count, size_t* bytes) {
  if (count < 0 || count > (int64_t)kTable * kMaxCtas || !bytes) return NMD_ERR_INVALID;
  *bytes = kMaxCtas * sizeof(Sums);
  return NMD_OK;
}

nmd_status nmd_clip_grad_norm(int64_t count, const void* const* d_grads, const int64_t* sizes, const int32_t* dtypes,
                              double max_norm, void* const* d_out, float* d_norm, void* d_workspace, size_t ws_bytes,
                              void* stream) {
  size_t need = 0;
  nmd_status st = nmd_clip_workspace_bytes(count, &need);
  if (st != NMD_OK) return st;
  if ((count > 0 && (!d_grads || !sizes || !dtypes)) || !d_norm || !(max_norm > 0.0) || !std::isfinite(max_norm))
    return NMD_ERR_INVALID;
  for (int64_t k = 0; k < count; ++k) {
    if (dtypes[k] < NMD_DT_FP32 || dtypes[k] > NMD_DT_FP16 || sizes[k] < 0) return NMD_ERR_INVALID;
    if (sizes[k] == 0) continue;
    const uintptr_t mis = dtypes[k] == NMD_DT_FP32 ? 3 : 1;
    const uintptr_t in = (uintptr_t)d_grads[k], out = d_out ? (uintptr_t)d_out[k] : in;
    if (!in || !out || ((in | out) & mis)) return NMD_ERR_INVALID;
  }
  if (!d_workspace || ws_bytes < need || ((uintptr_t)d_workspace & 255u)) return NMD_ERR_WORKSPACE;
  cudaStream_t s = (cudaStream_t)stream;
  Sums* parts = (Sums*)d_workspace;
  if (count <= kSmallTable) return run<kSmallTable>(count, d_grads, sizes, dtypes, max_norm, d_out, d_norm, parts, s);
  return run<kTable>(count, d_grads, sizes, dtypes, max_norm, d_out, d_norm, parts, s);
}

}  // extern "C"

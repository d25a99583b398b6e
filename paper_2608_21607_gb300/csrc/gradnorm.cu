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
// 400M elements, fp32 and bf16 in turn, in 300 tensors take 557 us, 6.2 TB/s over
// the three passes (read, read, write) or 0.92 of a plain copy's rate; two tensors
// of 8.9M fp32 elements 41 us, their second read from L2.  One load of a thread
// under way at a time instead of eight: 566 us and 80 us.
//
// Squares are summed in fp32 by each thread, in fp64 from there on.  A group of
// elements whose squares leave fp32's range, or come near its ends, is scaled
// by 2^-80 or 2^80 and summed apart; the three sums are put together in fp64,
// and norms over all of fp32's range come out right.
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "nmd_internal.cuh"

namespace nmd {
namespace {

constexpr int kThreads = 256;
constexpr int kVecs = 8;               // 16-byte loads of a thread under way together
constexpr int kChunkBytes = kThreads * kVecs * 16;   // one CTA's piece of a tensor at a time (32 KB)
constexpr int kCtasPerSm = 3, kScaleCtasPerSm = 4;
constexpr int kMaxCtas = 1024;         // CTAs of the norm pass over all launches

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

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(bf16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float as_float(__half x) { return __half2float(x); }
__device__ __forceinline__ void from_float(float v, float* x) { *x = v; }
__device__ __forceinline__ void from_float(float v, bf16* x) { *x = __float2bfloat16_rn(v); }
__device__ __forceinline__ void from_float(float v, __half* x) { *x = __float2half_rn(v); }

// Squares of elements: of the usual groups, of those whose sum is above 2^96
// (scaled by 2^-80) and of those whose sum is below 2^-60 (by 2^80).
struct Squares {
  float usual = 0.f, big = 0.f, small = 0.f;
  template <class T, int V>
  __device__ __forceinline__ void add(const uint4 (&v)[V]) {
    constexpr int N = 16 / sizeof(T);
    float t[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float f = as_float(((const T*)&v[i])[k]);
        t[k & 1] = fmaf(f, f, t[k & 1]);
      }
    const float sum = t[0] + t[1];
    if (sum >= 0x1p-60f && sum <= 0x1p96f) {
      usual += sum;
      return;
    }
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int k = 0; k < N; ++k) m = fmaxf(m, fabsf(as_float(((const T*)&v[i])[k])));
    const float scale = m > 1.f ? 0x1p-80f : 0x1p80f;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float f = as_float(((const T*)&v[i])[k]) * scale;
        s = fmaf(f, f, s);
      }
    if (m > 1.f) big += s;
    else small += s;
  }
};

// Elements [e0, e1) of a tensor by one CTA: the 16-byte vectors of the chunk
// (at most kVecs per thread), and single elements before and after them.
struct Piece {
  int head, nvec, tail;
};
template <class T>
__device__ __forceinline__ Piece piece_of(const T* x, int64_t e0, int64_t e1) {
  const int off = (int)((uintptr_t)(x + e0) & 15), n = (int)(e1 - e0);
  Piece p;
  p.head = min(off ? (16 - off) / (int)sizeof(T) : 0, n);
  p.nvec = (n - p.head) / (16 / (int)sizeof(T));
  p.tail = n - p.head - p.nvec * (16 / (int)sizeof(T));
  return p;
}
// the single element of this thread within the piece, or -1
template <class T>
__device__ __forceinline__ int single_of(const Piece& p) {
  const int t = threadIdx.x;
  return t < p.head ? t : t - p.head < p.tail ? p.nvec * (16 / (int)sizeof(T)) + t : -1;
}

template <class T>
__device__ __noinline__ void chunk_squares(const T* x, int64_t e0, int64_t e1, Squares& acc) {
  const Piece p = piece_of(x, e0, e1);
  const uint4* xv = (const uint4*)(x + e0 + p.head) + threadIdx.x;
  uint4 v[kVecs];
#pragma unroll
  for (int i = 0; i < kVecs; ++i)
    v[i] = (int)threadIdx.x + i * kThreads < p.nvec ? xv[i * kThreads] : make_uint4(0, 0, 0, 0);
  if ((int)threadIdx.x < p.nvec) acc.template add<T, kVecs>(v);
  const int s = single_of<T>(p);
  if (s >= 0) {
    uint4 w[1] = {make_uint4(0, 0, 0, 0)};
    *(T*)w = x[e0 + s];
    acc.template add<T, 1>(w);
  }
}

template <class T, bool SAME>
__device__ __noinline__ void chunk_scale(const T* x, T* o, int64_t e0, int64_t e1, float2 scale) {
  constexpr int N = 16 / sizeof(T), K = 8;
  const Piece p = piece_of(x, e0, e1);
  const uint4* xv = (const uint4*)(x + e0 + p.head);
  T* to = o + e0 + p.head;
  auto put = [&](const uint4& v, int i) {
    uint4 w;
#pragma unroll
    for (int k = 0; k < N; ++k) from_float(as_float(((const T*)&v)[k]) * scale.x * scale.y, (T*)&w + k);
    if (SAME) {
      __stcs((uint4*)to + i, w);
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k) to[i * N + k] = ((const T*)&w)[k];
    }
  };
  int i = threadIdx.x;
  for (; i + (K - 1) * kThreads < p.nvec; i += K * kThreads) {
    uint4 v[K];
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = __ldcs(xv + i + k * kThreads);   // read for the last time: room for what is written
#pragma unroll
    for (int k = 0; k < K; ++k) put(v[k], i + k * kThreads);
  }
  for (; i < p.nvec; i += kThreads) put(xv[i], i);
  const int s = single_of<T>(p);
  if (s >= 0) from_float(as_float(x[e0 + s]) * scale.x * scale.y, o + e0 + s);
}
template <class T>
__device__ __forceinline__ void scale_piece(const void* in, void* out, int64_t e0, int64_t e1, float2 scale) {
  // vectors on both sides where they start at the same offset from a 16-byte boundary
  if ((((uintptr_t)in ^ (uintptr_t)out) & 15) == 0) chunk_scale<T, true>((const T*)in, (T*)out, e0, e1, scale);
  else chunk_scale<T, false>((const T*)in, (T*)out, e0, e1, scale);
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
__global__ void __launch_bounds__(kThreads, kCtasPerSm)
    norm_kernel(const __grid_constant__ Table<K> tab, double* parts) {
  __shared__ double red[kThreads / 32];
  asm volatile("griddepcontrol.launch_dependents;");
  Squares acc;
  for (int64_t c = blockIdx.x; c < tab.chunks; c += gridDim.x) {
    const int e = entry_of(tab, c);
    const int es = tab.dtype[e] == NMD_DT_FP32 ? 4 : 2;
    const int64_t e0 = (c - tab.first[e]) * (kChunkBytes / es);
    const int64_t e1 = min(tab.n[e], e0 + kChunkBytes / es);
    if (tab.dtype[e] == NMD_DT_FP32) chunk_squares((const float*)tab.in[e], e0, e1, acc);
    else if (tab.dtype[e] == NMD_DT_BF16) chunk_squares((const bf16*)tab.in[e], e0, e1, acc);
    else chunk_squares((const __half*)tab.in[e], e0, e1, acc);
  }
  // fp64 holds all three together
  const double s = cta_sum((double)acc.usual + (double)acc.big * 0x1p160 + (double)acc.small * 0x1p-160, red);
  if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

// The chunks are taken from the last to the first: the norm pass read those
// last, and they are still in L2.  They leave it as they are read (two tensors of
// 8.9M fp32 elements: 39.3 us against 40.9 us where they stay; of 16M: 65.6
// against 68.1).
template <int K>
__global__ void __launch_bounds__(kThreads, kScaleCtasPerSm)
    scale_kernel(const __grid_constant__ Table<K> tab, const double* parts, int nparts, double max_norm, int in_place,
                 float* norm_out) {
  __shared__ double red[kThreads / 32];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  double sum = 0.0;
  for (int i = threadIdx.x; i < nparts; i += kThreads) sum += parts[i];
  const double norm = sqrt(cta_sum(sum, red));
  if (norm_out != nullptr && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
  // a norm that is not a number makes every gradient so
  const double ratio = norm <= max_norm ? 1.0 : max_norm / norm;
  // A ratio below fp32's normal numbers would lose bits: as the product of two.  (The
  // first leaves every element normal whose scaled value is, and its own product exact.)
  const float2 scale = ratio < 0x1p-126 ? make_float2(0x1p-100f, (float)(ratio * 0x1p100)) : make_float2(1.f, (float)ratio);
  if (in_place && scale.y == 1.f) return;
  for (int64_t c = tab.chunks - 1 - blockIdx.x; c >= 0; c -= gridDim.x) {
    const int e = entry_of(tab, c);
    const int es = tab.dtype[e] == NMD_DT_FP32 ? 4 : 2;
    const int64_t e0 = (c - tab.first[e]) * (kChunkBytes / es);
    const int64_t e1 = min(tab.n[e], e0 + kChunkBytes / es);
    if (tab.dtype[e] == NMD_DT_FP32) scale_piece<float>(tab.in[e], tab.out[e], e0, e1, scale);
    else if (tab.dtype[e] == NMD_DT_BF16) scale_piece<bf16>(tab.in[e], tab.out[e], e0, e1, scale);
    else scale_piece<__half>(tab.in[e], tab.out[e], e0, e1, scale);
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
               void* const* out, float* d_norm, double* parts, cudaStream_t s) {
  const int sms = sm_count();
  if (sms == 0) return NMD_ERR_CUDA;
  const int64_t groups = std::max<int64_t>(1, (count + K - 1) / K);
  // CTAs of each launch: the partial sums of all launches fit the workspace
  const int most = (int)std::max<int64_t>(1, std::min<int64_t>(sms * kCtasPerSm, kMaxCtas / groups));
  int nparts = 0;
  Table<K> t;
  for (int64_t g = 0; g < groups; ++g) {
    fill(t, in, out, n, dtype, g * K, std::min(count, (g + 1) * K));
    const int grid = (int)std::max<int64_t>(1, std::min<int64_t>(t.chunks, most));
    norm_kernel<K><<<grid, kThreads, 0, s>>>(t, parts + nparts);
    nparts += grid;
  }
  // the last group first, in line with the order of the chunks
  for (int64_t g = groups - 1; g >= 0; --g) {
    if (groups > 1) fill(t, in, out, n, dtype, g * K, std::min(count, (g + 1) * K));
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)std::max<int64_t>(1, std::min<int64_t>(t.chunks, sms * kScaleCtasPerSm)));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = s;
    cfg.attrs = &attr;
    cfg.numAttrs = groups == 1 ? 1 : 0;   // it waits for the launch just ahead only
    if (cudaLaunchKernelEx(&cfg, scale_kernel<K>, t, (const double*)parts, nparts, max_norm, (int)(out == nullptr),
                           g == 0 ? d_norm : (float*)nullptr) != cudaSuccess)
      return NMD_ERR_CUDA;
  }
  return cudaGetLastError() == cudaSuccess ? NMD_OK : NMD_ERR_CUDA;
}

// Whether each tensor that is written lies apart from every other one, read or
// written: CTAs take the pieces of tensors in no order.
struct Range {
  uintptr_t from, to;
};
nmd_status apart(int64_t count, const void* const* in, const int64_t* n, const int32_t* dtype, void* const* out) {
  const std::unique_ptr<Range[]> to(new (std::nothrow) Range[(size_t)count]);
  if (!to) return NMD_ERR_CUDA;
  auto range = [&](const void* x, int64_t k) {
    return Range{(uintptr_t)x, (uintptr_t)x + (uintptr_t)n[k] * (dtype[k] == NMD_DT_FP32 ? 4 : 2)};
  };
  Range* end = to.get();
  for (int64_t k = 0; k < count; ++k)
    if (n[k] > 0) *end++ = range(out ? out[k] : in[k], k);
  std::sort(to.get(), end, [](const Range& a, const Range& b) { return a.from < b.from; });
  for (const Range* r = to.get() + 1; r < end; ++r)
    if (r->from < r[-1].to) return NMD_ERR_INVALID;
  if (out)
    for (int64_t k = 0; k < count; ++k) {
      if (n[k] == 0 || in[k] == out[k]) continue;
      const Range r = range(in[k], k);   // against the first range that ends past its start
      const Range* at = std::upper_bound(to.get(), end, r.from, [](uintptr_t v, const Range& a) { return v < a.to; });
      if (at != end && at->from < r.to) return NMD_ERR_INVALID;
    }
  return NMD_OK;
}

// tensors per launch: the table is copied with every launch, so short lists take a small one
constexpr int kSmallTable = 16, kTable = 512;

}  // namespace
}  // namespace nmd

using namespace nmd;

extern "C" {

nmd_status nmd_clip_workspace_bytes(int64_t count, size_t* bytes) {
  if (count < 0 || count > (int64_t)kTable * kMaxCtas || !bytes) return NMD_ERR_INVALID;
  *bytes = kMaxCtas * sizeof(double);
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
  if ((count > 1 || d_out) && (st = apart(count, d_grads, sizes, dtypes, d_out)) != NMD_OK) return st;
  if (!d_workspace || ws_bytes < need || ((uintptr_t)d_workspace & 255u)) return NMD_ERR_WORKSPACE;
  cudaStream_t s = (cudaStream_t)stream;
  double* parts = (double*)d_workspace;
  if (count <= kSmallTable) return run<kSmallTable>(count, d_grads, sizes, dtypes, max_norm, d_out, d_norm, parts, s);
  return run<kTable>(count, d_grads, sizes, dtypes, max_norm, d_out, d_norm, parts, s);
}

}  // extern "C"

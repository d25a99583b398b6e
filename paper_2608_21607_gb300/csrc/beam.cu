// One step of beam search over the rows of a logits matrix, and the beams'
// states in the order of their parents (formulas in include/nmd.h).
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "nmd_internal.cuh"
#include "softmax_sum.cuh"

namespace nmd {
namespace {

constexpr int kThreads = 256;
constexpr int kMostBeams = 64, kMostWidth = 128;

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(bf16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float as_float(__half x) { return __half2float(x); }

struct Select {
  const void* x;
  int64_t V, ld;
  int K, width;
  double inv_temp;
  const float* scores;
  const uint8_t* finished;
  int64_t end;
  float* out_scores;
  int64_t* parents;
  int64_t* tokens;
  uint8_t* out_finished;
};

// an offer: its value and its place among the group's (beam, column) pairs
struct Offer {
  double value;
  int64_t at;
  __device__ __forceinline__ bool before(const Offer& o) const { return value > o.value || (value == o.value && at < o.at); }
};
__device__ __forceinline__ Offer better(Offer a, Offer b) { return b.before(a) ? b : a; }

__device__ __forceinline__ Offer cta_best(Offer o, Offer* red) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    Offer p;
    p.value = __shfl_xor_sync(0xffffffffu, o.value, d);
    p.at = __shfl_xor_sync(0xffffffffu, o.at, d);
    o = better(o, p);
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = o;
  __syncthreads();
  for (int i = 0; i < kThreads / 32; ++i) o = better(o, red[i]);
  return o;
}

// A CTA per group: every row's maximum and sum, then the offers one by one, each the
// best of those that come after the last one taken.
template <class T>
__global__ void __launch_bounds__(kThreads) select_kernel(Select a) {
  __shared__ Offer red[kThreads / 32];
  __shared__ double base[kMostBeams], top[kMostBeams], sums[kThreads / 32];
  __shared__ int kind[kMostBeams];   // 0: offers nothing, 1: a row, 2: finished
  const int64_t b = blockIdx.x;
  const int64_t none = (int64_t)1 << 62;
  for (int k = 0; k < a.K; ++k) {
    const float s = a.scores[b * a.K + k];
    const bool used = fabsf(s) < INFINITY;
    const bool done = a.finished != nullptr && a.finished[b * a.K + k] != 0;
    if (!used || done) {
      if (threadIdx.x == 0) {
        kind[k] = used ? 2 : 0;
        base[k] = s;
      }
      continue;
    }
    const T* row = (const T*)a.x + (b * a.K + k) * a.ld;
    Offer m{-INFINITY, 0};
    bool bad = false;
    for (int64_t v = threadIdx.x; v < a.V; v += kThreads) {
      const float x = as_float(row[v]);
      bad |= !(x < INFINITY);
      m.value = fmax(m.value, (double)x);
    }
    bad = __syncthreads_or(bad);
    m = cta_best(m, red);
    double sum = 0.0;
    for (int64_t v = threadIdx.x; v < a.V; v += kThreads)
      sum += m.value > -INFINITY ? exp(((double)as_float(row[v]) - m.value) * a.inv_temp) : 0.0;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
      sum = 0.0;
      for (int i = 0; i < kThreads / 32; ++i) sum += sums[i];
      kind[k] = !bad && m.value > -INFINITY;
      base[k] = s - log(sum);
      top[k] = m.value;
    }
  }
  __syncthreads();
  Offer last{INFINITY, -1};
  for (int i = 0; i < a.width; ++i) {
    Offer best{-INFINITY, none};
    for (int k = 0; k < a.K; ++k) {
      if (kind[k] == 2) {
        const Offer o{base[k], k * a.V + a.end};
        if (last.before(o)) best = better(best, o);
      }
      if (kind[k] != 1) continue;
      const T* row = (const T*)a.x + (b * a.K + k) * a.ld;
      for (int64_t v = threadIdx.x; v < a.V; v += kThreads) {
        const Offer o{base[k] + ((double)as_float(row[v]) - top[k]) * a.inv_temp, k * a.V + v};
        if (last.before(o)) best = better(best, o);
      }
    }
    last = cta_best(best, red);
    if (threadIdx.x == 0) {
      const bool offered = last.value > -INFINITY;
      const int64_t token = offered ? last.at % a.V : -1;
      a.out_scores[b * a.width + i] = offered ? (float)last.value : -INFINITY;
      a.parents[b * a.width + i] = offered ? last.at / a.V : 0;
      a.tokens[b * a.width + i] = token;
      if (a.out_finished != nullptr) a.out_finished[b * a.width + i] = offered && token == a.end;
    }
    if (!(last.value > -INFINITY)) last.value = -INFINITY, last.at = none;
  }
}

// ---------------------------------------------------------------------------- states

struct State {
  const char* in;
  char* out;
  int64_t in_outer, out_outer, in_row, out_row;
  int64_t units;    // units of a row
  int64_t slices;   // pieces of a row that a CTA takes at a time
  int64_t first;    // its first piece of work
  int unit;         // bytes: 1, 2, 4, 8 or 16
};
constexpr int kStates = 32;
struct States {
  State s[kStates];
  int count;
  int K, width, per;      // per: bytes of a row in a CTA's memory
  int64_t B, work;
  const int64_t* parents;
};

template <class U>
__device__ __forceinline__ void move(const State& s, int64_t w, const States& a, char* smem, const int* parent) {
  const int64_t slice = w % s.slices, g = w / s.slices, b = g % a.B, o = g / a.B;
  const int per = a.per / (int)sizeof(U);
  const int64_t u0 = slice * per;
  const int n = (int)min((int64_t)per, s.units - u0);
  U* buf = (U*)smem;
  const char* in = s.in + o * s.in_outer + b * a.K * s.in_row;
  char* out = s.out + o * s.out_outer + b * a.width * s.out_row;
  for (int i = threadIdx.x; i < a.K * n; i += kThreads) {
    const int k = i / n, u = i - k * n;
    buf[k * per + u] = ((const U*)(in + k * s.in_row))[u0 + u];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.width * n; i += kThreads) {
    const int k = i / n, u = i - k * n, p = parent[k];
    if (p >= 0) ((U*)(out + k * s.out_row))[u0 + u] = buf[p * per + u];
  }
}

// A CTA takes a piece of all K rows of a group at a time: it is in shared memory before
// any row is written, so that rows may change places.
__global__ void __launch_bounds__(kThreads) reorder_kernel(const __grid_constant__ States a) {
  extern __shared__ __align__(16) char smem[];
  __shared__ int parent[kMostWidth];
  for (int64_t w = blockIdx.x; w < a.work; w += gridDim.x) {
    int e = 0;
    while (e + 1 < a.count && a.s[e + 1].first <= w) ++e;
    const State& s = a.s[e];
    const int64_t mine = w - s.first, b = mine / s.slices % a.B;
    __syncthreads();
    for (int k = threadIdx.x; k < a.width; k += kThreads) {
      const int64_t p = a.parents[b * a.width + k];
      parent[k] = p >= 0 && p < a.K ? (int)p : -1;
    }
    __syncthreads();
    switch (s.unit) {
      case 16: move<uint4>(s, mine, a, smem, parent); break;
      case 8: move<uint2>(s, mine, a, smem, parent); break;
      case 4: move<uint32_t>(s, mine, a, smem, parent); break;
      case 2: move<uint16_t>(s, mine, a, smem, parent); break;
      default: move<uint8_t>(s, mine, a, smem, parent);
    }
  }
}

bool beams_ok(int64_t B, int64_t K, int64_t width) {
  return B >= 0 && B <= (1 << 20) && K >= 1 && K <= kMostBeams && width >= 1 && width <= kMostWidth &&
         B * K <= ((int64_t)1 << 27);
}

constexpr int64_t kMostBytes = (int64_t)1 << 46;
// Whether rows of `bytes` at o `outer` + i `row` lie apart, and how far they reach.
bool rows_apart(int64_t outer, int64_t so, int64_t rows, int64_t sr, int64_t bytes, int64_t* reach) {
  if (so < 0 || sr < 0 || so > kMostBytes || sr > kMostBytes) return false;
  if ((outer > 1 && so > kMostBytes / outer) || (rows > 1 && sr > kMostBytes / rows)) return false;
  int64_t n[2] = {outer, rows}, s[2] = {so, sr};
  if (n[0] > 1 && (n[1] <= 1 || s[0] < s[1])) {   // the closer ones first
    std::swap(n[0], n[1]);
    std::swap(s[0], s[1]);
  }
  if (n[0] > 1 && n[1] <= 1) std::swap(n[0], n[1]), std::swap(s[0], s[1]);
  int64_t span = bytes;
  for (int i = 1; i >= 0; --i) {
    if (n[i] <= 1) continue;
    if (s[i] < span) return false;
    span += (n[i] - 1) * s[i];
  }
  *reach = span;
  return true;
}

}  // namespace
}  // namespace nmd

using namespace nmd;

extern "C" {

nmd_status nmd_beam_select(const void* d_logits, int32_t dtype, int64_t B, int64_t K, int64_t V, int64_t ld,
                           const float* d_scores, const uint8_t* d_finished, int64_t end, int64_t width,
                           double temperature, float* d_out_scores, int64_t* d_parents, int64_t* d_tokens,
                           uint8_t* d_out_finished, void* stream) {
  Scale c;
  if (!beams_ok(B, K, width) || dtype < NMD_DT_FP32 || dtype > NMD_DT_FP16 || V < 1 || V >= ((int64_t)1 << 31) || ld < 0 ||
      ld > ((int64_t)1 << 40) || !scale_of(temperature, &c) || end < -1 || end >= V || (d_finished && end < 0))
    return NMD_ERR_INVALID;
  if (B == 0) return NMD_OK;
  const uintptr_t mis = dtype == NMD_DT_FP32 ? 3 : 1;
  if (!d_logits || ((uintptr_t)d_logits & mis) || !d_scores || !d_out_scores || !d_parents || !d_tokens)
    return NMD_ERR_INVALID;
  const Select a{d_logits, V, ld, (int)K, (int)width, 1.0 / temperature, d_scores, d_finished, end,
                 d_out_scores, d_parents, d_tokens, d_out_finished};
  cudaStream_t s = (cudaStream_t)stream;
  if (dtype == NMD_DT_FP32) select_kernel<float><<<(unsigned)B, kThreads, 0, s>>>(a);
  else if (dtype == NMD_DT_BF16) select_kernel<bf16><<<(unsigned)B, kThreads, 0, s>>>(a);
  else select_kernel<__half><<<(unsigned)B, kThreads, 0, s>>>(a);
  return cudaGetLastError() == cudaSuccess ? NMD_OK : NMD_ERR_CUDA;
}

nmd_status nmd_beam_reorder(int64_t count, const nmd_beam_state* states, int64_t B, int64_t K, int64_t width,
                            const int64_t* d_parents, void* stream) {
  if (!beams_ok(B, K, width) || count < 0 || count > (1 << 20) || (count > 0 && !states) || (B > 0 && !d_parents))
    return NMD_ERR_INVALID;
  // What is read only, what is written only, and what changes in place: the first may
  // lie among itself, and so may the last.
  enum Kind { kRead, kWritten, kPlace };
  struct Range {
    uintptr_t from, to;
    Kind kind;
  };
  const std::unique_ptr<Range[]> ranges(new (std::nothrow) Range[(size_t)(2 * count + 1)]);
  if (!ranges) return NMD_ERR_CUDA;
  Range* end = ranges.get();
  for (int64_t k = 0; k < count; ++k) {
    const nmd_beam_state& s = states[k];
    if (s.outer < 0 || s.bytes < 0 || s.bytes > kMostBytes || s.outer > kMostBytes) return NMD_ERR_INVALID;
    if (s.outer == 0 || s.bytes == 0 || B == 0) continue;
    int64_t in = 0, out = 0;
    if (!s.in || !s.out || !rows_apart(s.outer, s.in_outer, B * K, s.in_row, s.bytes, &in) ||
        !rows_apart(s.outer, s.out_outer, B * width, s.out_row, s.bytes, &out))
      return NMD_ERR_INVALID;
    const bool place = s.in == s.out;
    if (place && (K != width || s.in_row != s.out_row || s.in_outer != s.out_outer)) return NMD_ERR_INVALID;
    if (!place) *end++ = Range{(uintptr_t)s.in, (uintptr_t)s.in + (uintptr_t)in, kRead};
    *end++ = Range{(uintptr_t)s.out, (uintptr_t)s.out + (uintptr_t)out, place ? kPlace : kWritten};
  }
  std::sort(ranges.get(), end, [](const Range& x, const Range& y) { return x.from < y.from; });
  uintptr_t to[3] = {0, 0, 0};
  for (const Range* q = ranges.get(); q < end; ++q) {
    const Range& r = *q;
    for (int o = 0; o < 3; ++o)
      if (r.from < to[o] && (o != r.kind || r.kind == kWritten)) return NMD_ERR_INVALID;
    to[r.kind] = std::max(to[r.kind], r.to);
  }
  int64_t k = 0;
  while (k < count) {
    States a{};
    a.B = B;
    a.K = (int)K;
    a.width = (int)width;
    a.parents = d_parents;
    a.per = (int)std::max<int64_t>(16, std::min<int64_t>(4096, 32768 / K / 16 * 16));
    for (; k < count && a.count < 1; ++k) {
      const nmd_beam_state& s = states[k];
      if (s.outer == 0 || s.bytes == 0 || B == 0) continue;
      uintptr_t all = (uintptr_t)s.in | (uintptr_t)s.out | (uintptr_t)s.bytes | 16;
      all |= (uintptr_t)s.in_row | (uintptr_t)s.out_row;
      if (s.outer > 1) all |= (uintptr_t)s.in_outer | (uintptr_t)s.out_outer;
      State& t = a.s[a.count++];
      t = State{(const char*)s.in, (char*)s.out, s.in_outer, s.out_outer, s.in_row, s.out_row, 0, 0, a.work,
                (int)(all & (~all + 1))};
      t.units = s.bytes / t.unit;
      t.slices = (s.bytes + a.per - 1) / a.per;
      a.work += t.slices * B * s.outer;
    }
    if (a.count == 0) break;
    reorder_kernel<<<(unsigned)std::min<int64_t>(a.work, 152 * 6), kThreads, a.per * K, (cudaStream_t)stream>>>(a);
    if (cudaGetLastError() != cudaSuccess) return NMD_ERR_CUDA;
  }
  return NMD_OK;
}

}  // extern "C"

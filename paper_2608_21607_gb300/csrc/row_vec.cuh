// What the kernels over the rows of a logits matrix share: 16-byte vectors of the
// three element types, running sums over them, where a row's vectors lie, copies
// into shared memory.
#pragma once

#include <cuda_fp16.h>

#include "nmd_internal.cuh"
#include "softmax_sum.cuh"

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
  // Four vectors: get(0) to get(3), asked for again where the group is not a usual one.
  // Returns the group's sum against the reference, infinity where it was not a usual one.
  template <class G>
  __device__ __forceinline__ float add(G get, Scale c) {
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
          return group;
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
      return INFINITY;
    }
  }
  // one value
  __device__ __forceinline__ void add(float x, Scale c) {
    raise(max_nan(s.m, x), c);
    if (usual) s.S += ex2(fmaf(x, c.hi, -r) + x * c.lo);
    else s.S += power(x, s.m == -INFINITY ? 0.f : s.m, c);
  }
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

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

template <int bytes = 16>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src) {
  if constexpr (bytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int left>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(left) : "memory"); }

}  // namespace
}  // namespace nmd

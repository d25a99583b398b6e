// What the kernels of the orthogonalised update share: matrices of any type and
// strides, the pieces that the tensor cores take, and the two ways to run the steps.
#pragma once

#include <cuda_fp16.h>

#include "nmd_internal.cuh"
#include "tc_pipe.cuh"
#include "tc_ptx.cuh"

namespace nmd {
namespace muon {

constexpr float kUnit = 4096.f;      // pieces hold 2^12 x

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(bf16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float as_float(__half x) { return __half2float(x); }
__device__ __forceinline__ void from_float(float v, float* x) { *x = v; }
__device__ __forceinline__ void from_float(float v, bf16* x) { *x = __float2bfloat16_rn(v); }
__device__ __forceinline__ void from_float(float v, __half* x) { *x = __float2half_rn(v); }

struct Matrix {   // elements at i rs + j cs
  void* x;
  int dtype;
  int64_t rs, cs;
  template <class T>
  __device__ __forceinline__ T& at(int64_t i, int64_t j) const {
    return ((T*)x)[i * rs + j * cs];
  }
};

// What becomes of the update: an R x C matrix, C the side whose elements are
// adjacent in memory (or nearer).
struct Job {
  int64_t R, C;
  Matrix grad, momentum, out;   // out: the result, or the weights
  int step;                     // 1: a training step (momentum and weights)
  float beta, rest;             // rest = 1 - beta
  int nesterov;
  float keep, lr;               // 1 - lr weight_decay, lr scale
  double eps;
  int flat;                     // the update's matrices fill memory row by row, from 16-byte boundaries
};

// Two fp16 pieces of an R x C matrix: plane 0 hi, plane 1 lo, rows of ld elements
struct Pieces {
  __half* hi;
  int64_t rows, cols, ld;
  __host__ __device__ int64_t plane() const { return rows * ld; }
};
__device__ __forceinline__ void split2(float a, float b, uint32_t& hi, uint32_t& lo) {
  const __half2 h = __floats2half2_rn(a, b);
  const float2 f = __half22float2(h);
  const __half2 l = __floats2half2_rn(a - f.x, b - f.y);
  hi = *(const uint32_t*)&h;
  lo = *(const uint32_t*)&l;
}
__device__ __forceinline__ void split(float v, __half& hi, __half& lo) {
  hi = __float2half_rn(v);
  lo = __float2half_rn(v - __half2float(hi));   // an overflow leaves infinities of both signs: NaN in the next product
}

// Every kernel here lets the next one start and waits for the one before to have ended
// before it touches memory, so that launches and set-up overlap.
__device__ __forceinline__ void ready_for_next() { asm volatile("griddepcontrol.launch_dependents;"); }
__device__ __forceinline__ void after_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// boxes of 64 (or 32) columns x `rows` rows x both pieces
inline bool map_of(const Pieces& x, int rows, CUtensorMap* m, int cols = 64) {
  const auto encode = tc::encode_fn();
  if (!encode) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)x.cols, (cuuint64_t)x.rows, 2};
  const cuuint64_t strides[2] = {(cuuint64_t)x.ld * 2, (cuuint64_t)x.plane() * 2};
  const cuuint32_t box[3] = {(cuuint32_t)cols, (cuuint32_t)rows, 2}, one[3] = {1, 1, 1};
  return encode(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, x.hi, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// ints at the start of a call's workspace: status and its detail, the shift t of X before
// each step and after the last, and on lines of their own a barrier's count and its flag
constexpr int kShift = 4, kBarrier = 32, kFlag = 64, kInts = 96;

// Updates with a short side of at most 64, and a long one that fits on chip: all steps in
// one kernel (muon_strip.cu).  X comes in pieces, a row per row of the long side and 64
// columns.  `ws`: strip_bytes.
constexpr int64_t kStripSide = 64, kStripMost = 152 * 8 * 128;
size_t strip_bytes(int64_t M);
nmd_status strip_run(const Job& j, const Pieces& X, int steps, const double* k, int* ints, void* ws, cudaStream_t s);

}  // namespace muon
}  // namespace nmd

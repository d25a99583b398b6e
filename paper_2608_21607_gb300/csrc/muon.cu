// An update replaced by a matrix near its orthogonal factor, by Newton-Schulz
// products, and the training step with it (formulas in include/nmd.h).
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include "nmd_internal.cuh"

namespace nmd {
namespace {

constexpr int kThreads = 256;
constexpr int kParts = 608;          // CTAs of the norm's pass
constexpr int64_t kMostSide = 16384;

struct Matrix {
  void* x;
  int dtype;
  int64_t rs, cs;
  __device__ __forceinline__ float get(int64_t i, int64_t j) const {
    const int64_t e = i * rs + j * cs;
    return dtype == NMD_DT_FP32 ? ((const float*)x)[e]
                                : dtype == NMD_DT_BF16 ? __bfloat162float(((const bf16*)x)[e]) : __half2float(((const __half*)x)[e]);
  }
  __device__ __forceinline__ void put(int64_t i, int64_t j, float v) const {
    const int64_t e = i * rs + j * cs;
    if (dtype == NMD_DT_FP32) ((float*)x)[e] = v;
    else if (dtype == NMD_DT_BF16) ((bf16*)x)[e] = __float2bfloat16_rn(v);
    else ((__half*)x)[e] = __float2half_rn(v);
  }
};

// What becomes of the update: rows x cols of it are G, or a momentum that G goes into.
struct Job {
  int64_t rows, cols;
  Matrix grad, momentum, out;   // out: the result, or the weights
  int step;                     // 1: a training step (momentum and weights)
  float beta, rest;             // rest = 1 - beta
  int nesterov;
  float keep, lr;               // 1 - lr weight_decay, lr scale
  double eps;
};

// U = M or beta M + (1 - beta) G after M <- beta M + (1 - beta) G, and its sum of squares
__global__ void __launch_bounds__(kThreads) update_kernel(Job j, float* X, double* parts) {
  __shared__ double red[kThreads / 32];
  double sum = 0.0;
  const int64_t n = j.rows * j.cols;
  for (int64_t e = blockIdx.x * (int64_t)kThreads + threadIdx.x; e < n; e += (int64_t)gridDim.x * kThreads) {
    const int64_t r = e / j.cols, c = e % j.cols;
    float u = j.grad.get(r, c);
    if (j.step) {
      const float g = u, m = j.beta * j.momentum.get(r, c) + j.rest * g;
      j.momentum.put(r, c, m);
      u = j.momentum.get(r, c);
      if (j.nesterov) u = j.beta * u + j.rest * g;
    }
    X[e] = u;
    sum += (double)u * (double)u;
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0.0;
    for (int i = 0; i < kThreads / 32; ++i) sum += red[i];
    parts[blockIdx.x] = sum;
  }
}
__global__ void __launch_bounds__(kThreads) normalise_kernel(float* X, int64_t n, const double* parts, int count, double eps) {
  __shared__ double inv;
  if (threadIdx.x == 0) {
    double sum = 0.0;
    for (int i = 0; i < count; ++i) sum += parts[i];
    inv = 1.0 / (sqrt(sum) + eps);
  }
  __syncthreads();
  for (int64_t e = blockIdx.x * (int64_t)kThreads + threadIdx.x; e < n; e += (int64_t)gridDim.x * kThreads)
    X[e] = (float)((double)X[e] * inv);
}

// C = alpha A B + beta D, elements at i * row + j * col
struct View {
  float* x;
  int64_t row, col;
  __device__ __forceinline__ float& at(int64_t i, int64_t j) const { return x[i * row + j * col]; }
};
constexpr int kTile = 32;
__global__ void __launch_bounds__(kThreads) product_kernel(View A, View B, View C, View D, int64_t m, int64_t n, int64_t k,
                                                           float alpha, float beta) {
  __shared__ float a[kTile][kTile + 1], b[kTile][kTile + 1];
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const int64_t i0 = (int64_t)blockIdx.y * kTile, j0 = (int64_t)blockIdx.x * kTile;
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  for (int64_t k0 = 0; k0 < k; k0 += kTile) {
    for (int q = 0; q < 4; ++q) {
      const int r = ty + 8 * q;
      a[r][tx] = i0 + r < m && k0 + tx < k ? A.at(i0 + r, k0 + tx) : 0.f;
      b[r][tx] = k0 + r < k && j0 + tx < n ? B.at(k0 + r, j0 + tx) : 0.f;
    }
    __syncthreads();
    for (int e = 0; e < kTile; ++e)
      for (int q = 0; q < 4; ++q) sum[q] = fmaf(a[ty + 8 * q][e], b[e][tx], sum[q]);
    __syncthreads();
  }
  for (int q = 0; q < 4; ++q) {
    const int64_t i = i0 + ty + 8 * q, j = j0 + tx;
    if (i < m && j < n) C.at(i, j) = alpha * sum[q] + (D.x ? beta * D.at(i, j) : 0.f);
  }
}
void product(View A, View B, View C, View D, int64_t m, int64_t n, int64_t k, float alpha, float beta, cudaStream_t s) {
  product_kernel<<<dim3((unsigned)((n + 31) / 32), (unsigned)((m + 31) / 32)), kThreads, 0, s>>>(A, B, C, D, m, n, k, alpha, beta);
}

__global__ void __launch_bounds__(kThreads) finish_kernel(Job j, const float* X) {
  const int64_t n = j.rows * j.cols;
  for (int64_t e = blockIdx.x * (int64_t)kThreads + threadIdx.x; e < n; e += (int64_t)gridDim.x * kThreads) {
    const int64_t r = e / j.cols, c = e % j.cols;
    j.out.put(r, c, j.step ? j.keep * j.out.get(r, c) - j.lr * X[e] : X[e]);
  }
}

inline size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

nmd_status run(const Job& j, int steps, const double* k, void* ws, cudaStream_t s) {
  const int64_t n = j.rows * j.cols, r = std::min(j.rows, j.cols), M = std::max(j.rows, j.cols);
  char* w = (char*)ws;
  double* parts = (double*)w;
  w += align256(kParts * sizeof(double));
  float* X = (float*)w;
  w += align256((size_t)n * 4);
  float* Y = (float*)w;
  w += align256((size_t)n * 4);
  float* A = (float*)w;
  w += align256((size_t)(r * r) * 4);
  float* P = (float*)w;
  update_kernel<<<kParts, kThreads, 0, s>>>(j, X, parts);
  normalise_kernel<<<kParts, kThreads, 0, s>>>(X, n, parts, kParts, j.eps);
  const bool tall = j.rows > j.cols;
  const View none{nullptr, 0, 0}, VA{A, r, 1}, VP{P, r, 1};
  for (int i = 0; i < steps; ++i) {
    const View x{X, tall ? 1 : j.cols, tall ? j.cols : 1}, xt{X, x.col, x.row}, y{Y, x.row, x.col};   // r x M
    product(x, xt, VA, none, r, r, M, 1.f, 0.f, s);
    product(VA, VA, VP, VA, r, r, r, (float)k[2], (float)k[1], s);
    product(VP, x, y, x, r, M, r, 1.f, (float)k[0], s);
    std::swap(X, Y);
  }
  finish_kernel<<<kParts, kThreads, 0, s>>>(j, X);
  return cudaGetLastError() == cudaSuccess ? NMD_OK : NMD_ERR_CUDA;
}

// Whether the elements of a matrix lie apart, and the bytes from its first to its last
bool apart(int64_t rows, int64_t cols, int64_t rs, int64_t cs, int64_t es, int64_t* reach) {
  if (rs < 0 || cs < 0 || rs > ((int64_t)1 << 40) || cs > ((int64_t)1 << 40)) return false;
  int64_t n[2] = {rows, cols}, st[2] = {rs, cs};
  if (n[0] > 1 && n[1] > 1 && st[0] < st[1]) std::swap(n[0], n[1]), std::swap(st[0], st[1]);
  int64_t span = 1;
  bool ok = true;
  for (int i = 1; i >= 0; --i) {
    if (n[i] <= 1) continue;
    ok &= st[i] >= span;
    span += (n[i] - 1) * st[i];
  }
  *reach = span * es;
  return ok;
}
inline int64_t size_of(int dtype) { return dtype == NMD_DT_FP32 ? 4 : 2; }

struct Range {
  uintptr_t from, to;
  bool meets(const Range& o) const { return from < o.to && o.from < to; }
};
// a matrix's arguments; `unique`: its elements have to lie apart
bool check(const void* x, int dtype, int64_t rows, int64_t cols, int64_t rs, int64_t cs, bool unique, Range* at) {
  if (dtype < NMD_DT_FP32 || dtype > NMD_DT_FP16 || !x || ((uintptr_t)x & (uintptr_t)(size_of(dtype) - 1))) return false;
  int64_t reach = 0;
  const bool ok = apart(rows, cols, rs, cs, size_of(dtype), &reach);
  if ((unique && !ok) || rs < 0 || cs < 0 || rs > ((int64_t)1 << 40) || cs > ((int64_t)1 << 40)) return false;
  *at = Range{(uintptr_t)x, (uintptr_t)x + (uintptr_t)reach};
  return true;
}
bool sizes_ok(int64_t rows, int64_t cols) {
  return rows >= 0 && cols >= 0 && rows < ((int64_t)1 << 31) && cols < ((int64_t)1 << 31) && std::min(rows, cols) <= kMostSide &&
         (rows == 0 || cols <= ((int64_t)1 << 36) / rows);
}
bool map_ok(int32_t steps, const double* k, double eps) {
  return steps >= 1 && steps <= 16 && k && std::isfinite(k[0]) && std::isfinite(k[1]) && std::isfinite(k[2]) && eps > 0.0 &&
         std::isfinite(eps);
}

}  // namespace
}  // namespace nmd

using namespace nmd;

extern "C" {

nmd_status nmd_orthogonalize_workspace_bytes(int64_t rows, int64_t cols, size_t* bytes) {
  if (!sizes_ok(rows, cols) || !bytes) return NMD_ERR_INVALID;
  const size_t n = (size_t)rows * (size_t)cols, r = (size_t)std::min(rows, cols);
  *bytes = align256(kParts * sizeof(double)) + 2 * align256(n * 4) + 2 * align256(r * r * 4);
  return NMD_OK;
}

nmd_status nmd_orthogonalize(const void* d_update, int32_t dtype, int64_t rows, int64_t cols, int64_t row_stride,
                             int64_t col_stride, int32_t steps, const double* coefficients, double eps, void* d_out,
                             int64_t out_row_stride, int64_t out_col_stride, void* d_workspace, size_t ws_bytes,
                             void* stream) {
  size_t need = 0;
  nmd_status st = nmd_orthogonalize_workspace_bytes(rows, cols, &need);
  if (st != NMD_OK) return st;
  if (!map_ok(steps, coefficients, eps)) return NMD_ERR_INVALID;
  if (rows == 0 || cols == 0) return NMD_OK;
  Range in, out;
  const bool place = d_update == d_out && row_stride == out_row_stride && col_stride == out_col_stride;
  if (!check(d_update, dtype, rows, cols, row_stride, col_stride, false, &in) ||
      !check(d_out, dtype, rows, cols, out_row_stride, out_col_stride, true, &out) || (!place && in.meets(out)))
    return NMD_ERR_INVALID;
  if (!d_workspace || ws_bytes < need || ((uintptr_t)d_workspace & 255u)) return NMD_ERR_WORKSPACE;
  Job j{};
  j.rows = rows;
  j.cols = cols;
  j.grad = Matrix{(void*)d_update, dtype, row_stride, col_stride};
  j.out = Matrix{d_out, dtype, out_row_stride, out_col_stride};
  j.eps = eps;
  return run(j, steps, coefficients, d_workspace, (cudaStream_t)stream);
}

nmd_status nmd_muon_step(const nmd_matrix* weight, const nmd_matrix* grad, const nmd_matrix* momentum, int64_t rows,
                         int64_t cols, double lr, double beta, int32_t nesterov, double weight_decay, double scale,
                         int32_t steps, const double* coefficients, double eps, void* d_workspace, size_t ws_bytes,
                         void* stream) {
  size_t need = 0;
  nmd_status st = nmd_orthogonalize_workspace_bytes(rows, cols, &need);
  if (st != NMD_OK) return st;
  if (!map_ok(steps, coefficients, eps) || !weight || !grad || !momentum || !(lr >= 0.0 && std::isfinite(lr)) ||
      !(beta >= 0.0 && beta < 1.0) || !(weight_decay >= 0.0 && std::isfinite(weight_decay)) || !std::isfinite(scale))
    return NMD_ERR_INVALID;
  if (rows == 0 || cols == 0) return NMD_OK;
  Range w, g, m;
  if (!check(weight->data, weight->dtype, rows, cols, weight->row_stride, weight->col_stride, true, &w) ||
      !check(grad->data, grad->dtype, rows, cols, grad->row_stride, grad->col_stride, false, &g) ||
      !check(momentum->data, momentum->dtype, rows, cols, momentum->row_stride, momentum->col_stride, true, &m) ||
      w.meets(g) || w.meets(m) || m.meets(g))
    return NMD_ERR_INVALID;
  if (!d_workspace || ws_bytes < need || ((uintptr_t)d_workspace & 255u)) return NMD_ERR_WORKSPACE;
  Job j{};
  j.rows = rows;
  j.cols = cols;
  j.grad = Matrix{grad->data, grad->dtype, grad->row_stride, grad->col_stride};
  j.momentum = Matrix{momentum->data, momentum->dtype, momentum->row_stride, momentum->col_stride};
  j.out = Matrix{weight->data, weight->dtype, weight->row_stride, weight->col_stride};
  j.step = 1;
  j.beta = (float)beta;
  j.rest = (float)(1.0 - beta);
  j.nesterov = nesterov != 0;
  j.keep = (float)(1.0 - lr * weight_decay);
  j.lr = (float)(lr * scale);
  j.eps = eps;
  return run(j, steps, coefficients, d_workspace, (cudaStream_t)stream);
}

}  // extern "C"

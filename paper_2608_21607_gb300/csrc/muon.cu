// An update replaced by a matrix near its orthogonal factor, by Newton-Schulz
// products, and the training step with it (formulas in include/nmd.h).
//
// The products run on the tcgen05 tensor cores.  Every matrix on the way (X, A =
// X X^T, P = a I + b A + c A^2) is kept as two fp16 pieces of 2^12 x, hi =
// fp16(v), lo = fp16(v - hi): 22 bits, or an absolute error below 2^-37 where that is
// more.  (|X|_F starts at 1, or less where eps is much of the divisor; below 2^-8 X is
// kept 2^t larger, t at most 100 and falling to 0 as the steps raise it.)  A product
// is hi hi + hi lo + lo hi, three MMAs; what lo lo would add is below 2^-22.  In fp32
// throughout the errors of early steps grow by up to a per step just the same, and the
// two come out equally far from the definition (a gradient of 139,255 x 64: 7.6e-7, fp32
// products 9.1e-7; 64 x 64: 1.4e-6 and 1.0e-6).  With one piece (11 bits) of everything the
// result would be off by parts in a hundred, and with one piece in the last two steps
// alone a 16-bit result by up to twice its rounding.
// The tensor cores add in fp32 but round towards zero, which leans by up to a unit of
// the sum so far per addition; so the two small products of 64 columns come first,
// and after each 64 columns (256 for 16-bit results, see run()) the sum leaves TMEM and
// goes on in the epilogue's registers, rounded to nearest.
//
// A step is three products: the Gram matrix (half of its tiles, the sum split where there
// are few), the polynomial (likewise half), and the update.  4096 x 4096 in bf16 takes
// 3.2 ms: 0.16 + 0.18 + 0.29 ms a step, the update at 1.41 PFLOP/s of MMAs, 0.75 of the
// measured burst rate.  There the operands' way bounds it: shared memory takes a block of
// 64 KB and gives three reads of its tiles for 768 cycles of products, 160 KB at 128 bytes
// a cycle (1240 cycles measured); call after call it is the power limit (3.45 ms at 1,370 W).
// 256 x 139,255 in bf16 takes 0.69 ms: its pieces, 142 MB, do not stay in L2 and are read
// twice and written once a step.  Small matrices are bound
// by the launches, 4 us each (2047 x 1001 in 0.31 ms).  Short sides up to 64: muon_strip.cu.
#include <algorithm>
#include <cmath>

#include "muon.cuh"

namespace nmd {
namespace {

using namespace tc;
using namespace muon;

constexpr int64_t kMostSide = 16384;
constexpr int kThreads = 256;
constexpr int kParts = 608;          // CTAs of the norm's pass: four per SM
constexpr int kSms = 152;            // the splitting of sums goes by this number, not by the device, for equal bits

// ------------------------------------------------------------------ the update and its norm

// fp32 squares of a few values, in fp64 where they leave fp32's range or come near its ends
template <int N>
__device__ __forceinline__ double squares(const float (&f)[N]) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) s = fmaf(f[i], f[i], s);
  if (s >= 0x1p-60f && s <= 0x1p96f) return (double)s;
  double d = 0.0;
#pragma unroll
  for (int i = 0; i < N; ++i) d += (double)f[i] * (double)f[i];
  return d;
}
__device__ __forceinline__ float update_of(const Job& j, float m, float g) { return j.nesterov ? fmaf(j.beta, m, j.rest * g) : m; }

// A warp takes kEach groups of 32 adjacent elements at a time: of as many rows, or of
// one row where there are fewer.
constexpr int kEach = 8;
struct Walk {
  int64_t across, work;   // pieces of work of a row (of rows), and in all
  int down, step;         // rows and columns from one group to the next
};
__host__ __device__ __forceinline__ Walk walk_of(int64_t R, int64_t C) {
  Walk w;
  const bool rows = R >= kEach;
  w.down = rows ? 1 : 0;
  w.step = rows ? 0 : 32;
  const int wide = rows ? 32 : 32 * kEach;
  w.across = (C + wide - 1) / wide;
  w.work = w.across * (rows ? (R + kEach - 1) / kEach : R);
  return w;
}
// the elements of one piece of work: f(i, row, column) for those that there are
template <class F>
__device__ __forceinline__ void each(const Walk& w, const Job& j, int64_t at, F f) {
  const int64_t q = at / w.across, r0 = q * (w.down ? kEach : 1), c0 = (at - q * w.across) * (w.down ? 32 : 32 * kEach) + (threadIdx.x & 31);
#pragma unroll
  for (int i = 0; i < kEach; ++i)
    if (r0 + i * w.down < j.R && c0 + i * w.step < j.C) f(i, r0 + i * w.down, c0 + i * w.step);
}

// Matrices whose elements fill memory row by row from a 16-byte boundary are read eight
// elements at a time, whatever their rows' length: the window from element f on comes out
// of the vectors that hold it.
__device__ __forceinline__ void window(const uint32_t* base, int64_t f, int64_t n, uint32_t (&w)[8]) {   // 8 of 32 bits
  const int s = (int)(f & 3);
  const uint4* v = (const uint4*)base + (f >> 2);
  if (f - s + 12 > n) {   // near the end: no vector beyond it
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = f + i < n ? base[f + i] : 0u;
    return;
  }
  const uint4 a = v[0], b = v[1];
  uint32_t u[11] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w, 0u, 0u, 0u};
  if (s != 0) {
    const uint4 c = v[2];
    u[8] = c.x;
    u[9] = c.y;
    u[10] = c.z;
  }
#pragma unroll
  for (int i = 0; i < 9; ++i) u[i] = s & 2 ? u[i + 2] : u[i];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = s & 1 ? u[i + 1] : u[i];
}
__device__ __forceinline__ void window(const uint16_t* base, int64_t f, int64_t n, uint32_t (&w)[4]) {   // 8 of 16 bits
  const int s = (int)(f & 7);
  const uint4* v = (const uint4*)base + (f >> 3);
  if (f - s + 16 > n) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = (f + 2 * i < n ? base[f + 2 * i] : 0u) | (f + 2 * i + 1 < n ? (uint32_t)base[f + 2 * i + 1] << 16 : 0u);
    return;
  }
  const uint4 a = v[0];
  uint32_t u[8] = {a.x, a.y, a.z, a.w, 0u, 0u, 0u, 0u};
  if (s != 0) {
    const uint4 b = v[1];
    u[4] = b.x;
    u[5] = b.y;
    u[6] = b.z;
    u[7] = b.w;
  }
#pragma unroll
  for (int i = 0; i < 6; ++i) u[i] = s & 4 ? u[i + 2] : u[i];
#pragma unroll
  for (int i = 0; i < 5; ++i) u[i] = s & 2 ? u[i + 1] : u[i];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = s & 1 ? __funnelshift_r(u[i], u[i + 1], 16) : u[i];
}
template <class T>
struct Eight {   // elements of a thread
  uint32_t w[2 * sizeof(T)];
  __device__ __forceinline__ void load(const T* base, int64_t f, int64_t n) {
    if constexpr (sizeof(T) == 4) window((const uint32_t*)base, f, n, w);
    else window((const uint16_t*)base, f, n, w);
  }
  __device__ __forceinline__ float get(int i) const { return as_float(((const T*)w)[i]); }
  __device__ __forceinline__ void set(int i, float v) { from_float(v, (T*)w + i); }
};
__host__ __device__ inline bool filled(const Matrix& m, int64_t C) { return m.cs == 1 && m.rs == C && ((uintptr_t)m.x & 15) == 0; }

// M <- beta M + (1 - beta) G, and the sum of squares of the update
template <class G, class M, bool STEP>
__global__ void __launch_bounds__(kThreads) norm_kernel(Job j, double* parts, int* status) {
  __shared__ double red[kThreads / 32];
  ready_for_next();
  after_previous();   // the kernels of an earlier call have done with the workspace
  if (blockIdx.x == 0 && threadIdx.x < kInts) status[threadIdx.x] = 0;
  double sum = 0.0;
  if (j.flat) {
    const int64_t n = j.R * j.C, vectors = (n + 7) / 8;
#pragma unroll 2
    for (int64_t v = blockIdx.x * (int64_t)kThreads + threadIdx.x; v < vectors; v += (int64_t)gridDim.x * kThreads) {
      Eight<G> g;
      Eight<M> m;
      float u[8];
      g.load((const G*)j.grad.x, v * 8, n);
      if (STEP) m.load((const M*)j.momentum.x, v * 8, n);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        u[i] = g.get(i);
        if (STEP) {
          m.set(i, fmaf(j.beta, m.get(i), j.rest * u[i]));
          u[i] = update_of(j, m.get(i), u[i]);   // of the momentum as it is stored
        }
      }
      if (STEP) {
        M* to = (M*)j.momentum.x + v * 8;
        if (v * 8 + 8 <= n) {
#pragma unroll
          for (int i = 0; i < (int)sizeof(M) / 2; ++i) ((uint4*)to)[i] = ((const uint4*)m.w)[i];
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (v * 8 + i < n) to[i] = ((const M*)m.w)[i];
        }
      }
      sum += squares(u);   // (what is past the end is 0 in all of them)
    }
  }
  const Walk w = walk_of(j.R, j.C);
  for (int64_t at = j.flat ? w.work : blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); at < w.work; at += gridDim.x * (kThreads / 32)) {
    G g[kEach];
    M m[kEach];
    float u[kEach];
    each(w, j, at, [&](int i, int64_t r, int64_t c) { g[i] = j.grad.at<G>(r, c); });
    if (STEP) each(w, j, at, [&](int i, int64_t r, int64_t c) { m[i] = j.momentum.at<M>(r, c); });
#pragma unroll
    for (int i = 0; i < kEach; ++i) u[i] = 0.f;
    each(w, j, at, [&](int i, int64_t r, int64_t c) {
      u[i] = as_float(g[i]);
      if (STEP) {
        from_float(fmaf(j.beta, as_float(m[i]), j.rest * u[i]), &m[i]);
        j.momentum.at<M>(r, c) = m[i];
        u[i] = update_of(j, as_float(m[i]), u[i]);   // of the momentum as it is stored
      }
    });
    sum += squares(u);
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

// What a value of the update is multiplied by, 2^(12 + t) / (norm + eps): a number near 1 and a power of two
// in two halves, so that norms of 1e-40 and 1e38 do.  By a whole CTA; the first one of the grid writes the
// shifts, t of X before each step and after the last.
struct Factor3 {
  float f, p, q;
  __device__ __forceinline__ float of(float u) const { return u * p * q * f; }
};
__device__ __forceinline__ Factor3 factor_of(const double* parts, int count, double eps, int* shift, int steps, int grows) {
  __shared__ double red[kThreads / 32];
  double sum = 0.0;
  for (int i = threadIdx.x; i < count; i += kThreads) sum += parts[i];
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = sum;
  __syncthreads();
  sum = 0.0;
  for (int i = 0; i < kThreads / 32; ++i) sum += red[i];
  // norm = s 2^h with s in [1, 2), so that one fp64 product and fp32 do for the rest
  const bool usual = sum > 0.0 && sum < INFINITY;
  const int h = usual ? (ilogb(sum) >> 1) : 0;
  const float s = usual ? sqrtf((float)ldexp(sum, -2 * h)) : (float)sum;
  const float both = s + (float)ldexp(eps, -h);
  // |X| = 2^-t at most; `grows`: a step takes a small X to 2^grows times itself at most
  const float size = s / both;
  const int small = size > 0.f && size < 0x1p-8f ? min(100, -ilogbf(size) - 1) : 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    int t = small;
    for (int i = 0; i <= steps; ++i) {
      shift[i] = t;
      t = t < 8 ? 0 : max(0, t - grows);
    }
  }
  int e = 0;
  Factor3 r;
  r.f = frexpf(sum == 0.0 ? 0.f : kUnit / both, &e);   // (an eps below fp32's range is 0 in it)
  e = max(-280, min(280, e - h + small));
  r.p = ldexpf(1.f, e / 2);
  r.q = ldexpf(1.f, e - e / 2);
  return r;
}

// X = update / (norm + eps) in pieces
template <class G, class M, bool STEP>
__global__ void __launch_bounds__(kThreads) pieces_kernel(Job j, Pieces X, const double* parts, int count, int* shift, int steps,
                                                          int grows) {
  ready_for_next();
  after_previous();
  const Factor3 f = factor_of(parts, count, j.eps, shift, steps, grows);
  if (j.flat) {   // by vectors of what is written
    const int64_t n = j.R * j.C, across = X.ld / 8, vectors = j.R * across;
#pragma unroll 2
    for (int64_t v = blockIdx.x * (int64_t)kThreads + threadIdx.x; v < vectors; v += (int64_t)gridDim.x * kThreads) {
      const int64_t r = vectors >> 31 ? v / across : (int64_t)((uint32_t)v / (uint32_t)across), c = (v - r * across) * 8;
      if (c >= j.C) continue;
      Eight<G> g;
      Eight<M> m;
      g.load((const G*)j.grad.x, r * j.C + c, n);
      if (STEP) m.load((const M*)j.momentum.x, r * j.C + c, n);
      float u[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = f.of(STEP ? update_of(j, m.get(i), g.get(i)) : g.get(i));   // (past the row's end: padding)
      uint4 h, l;
      split2(u[0], u[1], h.x, l.x);
      split2(u[2], u[3], h.y, l.y);
      split2(u[4], u[5], h.z, l.z);
      split2(u[6], u[7], h.w, l.w);
      __half* to = X.hi + r * X.ld + c;
      *(uint4*)to = h;
      *(uint4*)(to + X.plane()) = l;
    }
    return;
  }
  const Walk w = walk_of(j.R, j.C);
  for (int64_t at = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); at < w.work; at += gridDim.x * (kThreads / 32)) {
    G g[kEach];
    M m[kEach];
    each(w, j, at, [&](int i, int64_t r, int64_t c) { g[i] = j.grad.at<G>(r, c); });
    if (STEP) each(w, j, at, [&](int i, int64_t r, int64_t c) { m[i] = j.momentum.at<M>(r, c); });
    each(w, j, at, [&](int i, int64_t r, int64_t c) {
      const float u = STEP ? update_of(j, as_float(m[i]), as_float(g[i])) : as_float(g[i]);
      __half hi, lo;
      split(f.of(u), hi, lo);
      X.hi[r * X.ld + c] = hi;
      X.hi[X.plane() + r * X.ld + c] = lo;
    });
  }
}

// The same of a wide update turned over: row c of X is column c of the update, 64
// columns.  A lane reads 32 elements of its column, adjacent lanes adjacent columns, and
// writes them as vectors.
template <class G, class M, bool STEP>
__global__ void __launch_bounds__(kThreads) turned_kernel(Job j, Pieces X, const double* parts, int count, int* shift, int steps,
                                                          int grows) {
  ready_for_next();
  after_previous();
  const Factor3 f = factor_of(parts, count, j.eps, shift, steps, grows);
  const int64_t half = (j.R + 31) / 32, work = (j.C + 31) / 32 * half;
  for (int64_t at = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); at < work; at += gridDim.x * (kThreads / 32)) {
    const int64_t c = at / half * 32 + (threadIdx.x & 31), r0 = at % half * 32;
    if (c >= j.C) continue;
#pragma unroll 1
    for (int q = 0; q < 4; ++q) {
      G g[8];
      M m[8];
      float u[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t r = r0 + q * 8 + i;
        if (r < j.R) g[i] = j.grad.at<G>(r, c);
        if (STEP && r < j.R) m[i] = j.momentum.at<M>(r, c);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        u[i] = r0 + q * 8 + i < j.R ? f.of(STEP ? update_of(j, as_float(m[i]), as_float(g[i])) : as_float(g[i])) : 0.f;
      uint4 h, l;
      split2(u[0], u[1], h.x, l.x);
      split2(u[2], u[3], h.y, l.y);
      split2(u[4], u[5], h.z, l.z);
      split2(u[6], u[7], h.w, l.w);
      __half* to = X.hi + c * X.ld + r0 + q * 8;
      *(uint4*)to = h;
      *(uint4*)(to + X.plane()) = l;
    }
  }
}

// ---------------------------------------------------------------------------- products

enum Mode { kSymmetric, kPartial, kMatrix, kResult };

struct Gemm {
  int64_t M, N;             // D is M x N
  int kblocks, splits;      // stages of the sum; parts of it that are tiles of their own
  int chunk;                // stages whose sum stays in TMEM
  int tiles_m, tiles_n, items;   // tiles down and across; tiles x splits
  int lower;                // 1: D is symmetric (B is A), tiles below and on the diagonal only
  int mode;
  float alpha, beta, diag;  // D = alpha 2^(*up - times *down) (sum) + beta C + diag I, in pieces
  const int *up, *down;     // or nullptr
  int times;
  Pieces c, d;
  float* part;              // items x 128 x BN
  Job out;
  int* status;
};

constexpr int kBM = 128, kBK = 64;   // rows of a tile, products of a stage
// (of tiles of 256 columns half as many, four stages: 3.13 ms for 4096 x 4096, in two 3.30)
__host__ __device__ constexpr int depth_of(int BN) { return BN > 128 ? kBK / 2 : kBK; }
template <int BN>
struct Cfg {
  static constexpr int BK = depth_of(BN), A_BYTES = 2 * kBM * BK * 2, B_BYTES = 2 * BN * BK * 2, STAGE = A_BYTES + B_BYTES;
  static constexpr int NS = 196608 / STAGE;
  static constexpr int TMEM = 2 * BN;
  static constexpr int EPILOGUE = BN > 128 ? 16 : 8, PRODUCER = EPILOGUE, ISSUER = EPILOGUE + 1, THREADS = 32 * (EPILOGUE + 2);   // warps
  static constexpr size_t OFF_TURN = (size_t)NS * STAGE;                // eight 32 x 32 squares for the epilogue's warps
  static constexpr size_t OFF_BARS = OFF_TURN + 8 * 4096;
  static constexpr int NBAR = 2 * NS + 5;
  static constexpr size_t SMEM = 1024 + OFF_BARS + NBAR * 8 + 16;
  static_assert(SMEM <= 227 * 1024, "shared memory");
};

__device__ __forceinline__ float scale_of_sum(const Gemm& p) {
  return ldexpf(p.alpha, (p.up ? *p.up : 0) - (p.down ? p.times * *p.down : 0));
}

// tile (i, j) and the part of the sum of a work item
struct Item {
  int i, j, k0, k1;
};
__device__ __forceinline__ Item item_of(const Gemm& p, int w, int BN) {
  Item t;
  const int tile = w / p.splits, part = w - tile * p.splits;
  if (p.lower) {
    int left = tile;
    t.i = 0;
    for (;;) {
      const int n = min((kBM * (t.i + 1) - 1) / BN + 1, p.tiles_n);
      if (left < n) break;
      left -= n;
      ++t.i;
    }
    t.j = left;
  } else {
    // the shorter side first: tiles that read the same part of the longer operand run together
    if (p.tiles_m < p.tiles_n) {
      t.j = tile / p.tiles_m;
      t.i = tile - t.j * p.tiles_m;
    } else {
      t.i = tile / p.tiles_n;
      t.j = tile - t.i * p.tiles_n;
    }
  }
  t.k0 = (int)((int64_t)p.kblocks * part / p.splits);
  t.k1 = (int)((int64_t)p.kblocks * (part + 1) / p.splits);
  return t;
}

// What a warp writes goes through a 32 x 32 square of its own in shared memory, element
// (r, c) at r 32 + (c ^ r), so that adjacent lanes write adjacent elements.  (A row per
// lane, 16 bytes at a time, are as many requests to L2 as there are half sectors.)  The
// code is one copy for all columns of a tile: most tiles are few per CTA, and fetching
// instructions counted for more than executing them.
__device__ __forceinline__ float& in_square(float* sq, int r, int c) { return sq[r * 32 + (c ^ r)]; }

// 32 rows x 32 columns of D in pieces, from row0 and col0 on: alpha (the square, or with
// `turned` its transpose) + beta C + diag I.  Four lanes write 64 adjacent bytes of a row.
// Rows past the last are not written; columns up to the row's stride are.
template <bool WIDE>
__device__ __forceinline__ void put_block(const Gemm& p, float alpha, float* sq, int64_t row0, int64_t col0, bool turned, bool lower) {
  const int lane = threadIdx.x & 31, c = (lane & 3) * 8;
  // C, all of it under way together where a thread has the registers
  constexpr int kAhead = WIDE ? 1 : 4;
#pragma unroll 1
  for (int i0 = 0; i0 < 4; i0 += kAhead) {
    uint4 ch[kAhead], cl[kAhead];
    if (p.beta != 0.f) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int64_t row = row0 + (i0 + i) * 8 + (lane >> 2);
        if (row >= p.M) break;
        const __half* at = p.c.hi + row * p.c.ld + col0 + c;
        ch[i] = *(const uint4*)at;
        cl[i] = *(const uint4*)(at + p.c.plane());
      }
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int r = (i0 + i) * 8 + (lane >> 2);
      const int64_t row = row0 + r, col = col0 + c;
      if (row >= p.M) return;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        // on the diagonal what is above it is what is below it, in every bit
        const bool swap = turned || (lower && c + e > r);
        v[e] = alpha * (swap ? in_square(sq, c + e, r) : in_square(sq, r, c + e));
      }
      if (p.beta != 0.f) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          v[e] = fmaf(p.beta, __half2float(((const __half*)&ch[i])[e]) + __half2float(((const __half*)&cl[i])[e]), v[e]);
      }
      if (lower) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (c + e == r) v[e] += p.diag;
      }
      uint4 h, l;
      split2(v[0], v[1], h.x, l.x);
      split2(v[2], v[3], h.y, l.y);
      split2(v[4], v[5], h.z, l.z);
      split2(v[6], v[7], h.w, l.w);
      __half* to = p.d.hi + row * p.d.ld + col;
      *(uint4*)to = h;
      *(uint4*)(to + p.d.plane()) = l;
    }
  }
}

template <class T>
__device__ __forceinline__ void put_rows(const Gemm& p, float alpha, int64_t row0, int rows, int64_t col, float* sq) {
  const int lane = threadIdx.x & 31;
  T* at = &p.out.out.at<T>(row0, col);
  const int64_t rs = p.out.out.rs;
#pragma unroll 1
  for (int r0 = 0; r0 < rows; r0 += 8) {
    T w[8];
    if (p.out.step) {   // all loads, then all stores
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (r0 + i < rows) w[i] = at[(r0 + i) * rs];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = r0 + i;
      if (r >= rows) break;
      float x = alpha * in_square(sq, r, lane);
      if (p.out.step) x = fmaf(-p.out.lr, x, p.out.keep * as_float(w[i]));
      from_float(x, &at[r * rs]);
    }
  }
}
// 32 x 32 of D in pieces from a row per lane, without C: each lane's vectors of pieces go
// through shared memory instead (a fifth of the instructions)
__device__ __forceinline__ void put_rows_of(const Gemm& p, float alpha, const float (&v)[32], float* sq, int64_t row0, int64_t col0) {
  const int lane = threadIdx.x & 31;
  uint4* s = (uint4*)sq;   // [piece][row][four vectors], a row's in an order that spreads over the banks
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    uint4 h, l;
    split2(v[8 * q] * alpha, v[8 * q + 1] * alpha, h.x, l.x);
    split2(v[8 * q + 2] * alpha, v[8 * q + 3] * alpha, h.y, l.y);
    split2(v[8 * q + 4] * alpha, v[8 * q + 5] * alpha, h.z, l.z);
    split2(v[8 * q + 6] * alpha, v[8 * q + 7] * alpha, h.w, l.w);
    s[lane * 4 + (q ^ (lane >> 1 & 3))] = h;
    s[128 + lane * 4 + (q ^ (lane >> 1 & 3))] = l;
  }
  __syncwarp();
  if (col0 >= p.d.ld) return;
  __half* to = p.d.hi + (row0 + (lane >> 2)) * p.d.ld + col0 + (lane & 3) * 8;
  const int64_t plane = p.d.plane(), step = 8 * p.d.ld;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = i * 8 + (lane >> 2), at = r * 4 + ((lane & 3) ^ (r >> 1 & 3));
    if (row0 + r < p.M) {
      *(uint4*)(to + i * step) = s[at];
      *(uint4*)(to + i * step + plane) = s[128 + at];
    }
  }
}
// the square of rows from row0 and columns from col0 on, by the kernel's mode
template <bool WIDE>
__device__ __forceinline__ void put_square(const Gemm& p, float alpha, float* sq, int64_t row0, int64_t col0) {
  const int lane = threadIdx.x & 31;
  if (p.mode == kResult) {
    if (col0 + lane >= p.N) return;
    const Matrix& o = p.out.out;
    const int rows = (int)min((int64_t)32, p.M - row0);
    if (o.dtype == NMD_DT_FP32) put_rows<float>(p, alpha, row0, rows, col0 + lane, sq);
    else if (o.dtype == NMD_DT_BF16) put_rows<bf16>(p, alpha, row0, rows, col0 + lane, sq);
    else put_rows<__half>(p, alpha, row0, rows, col0 + lane, sq);
  } else if (col0 < p.d.ld) {
    if (p.mode == kSymmetric && col0 > row0) return;   // above the diagonal
    put_block<WIDE>(p, alpha, sq, row0, col0, false, p.mode == kSymmetric && col0 == row0);
    if (p.mode == kSymmetric && col0 < row0 && row0 < p.M) {
      put_block<WIDE>(p, alpha, sq, col0, row0, true, false);
    }
  }
}

// D = A B^T in tiles of 128 x BN.  An operand whose sum runs along its rows in memory
// (AMN = false: A[m][k]) comes in tiles of 64 adjacent k (32 for BN = 256); one whose sum runs
// across them (AMN: A[k][m]) in panels of 64 adjacent m, and the tensor cores take
// it as MN-major.  Hi and lo pieces are the two planes of one tensor map.
//   epilogue    8 warps, or 16 for tiles of 256 columns: a sum's chunks from TMEM (a
//               lane a row; two or four parts of the columns), added up in registers,
//               then written; of 16, the two warps of the same rows share a square of
//               shared memory and use it in turn
//   one warp    loads, one elected lane
//   one warp    issues the products
// Work items (tile, part of the sum) are dealt to one CTA per SM in turn; two TMEM
// buffers and the ring of stages run on from one item to the next.
template <int BN, bool AMN, bool BMN>
__global__ void __launch_bounds__(Cfg<BN>::THREADS, 1)
    gemm_kernel(const __grid_constant__ CUtensorMap ta, const __grid_constant__ CUtensorMap tb, const __grid_constant__ Gemm p) {
  using C = Cfg<BN>;
  constexpr int BK = C::BK;
  constexpr uint32_t kAlong = BK == 64 ? SWZ_128B : SWZ_64B;   // of an operand whose sum runs along its rows
  extern __shared__ char smem_raw[];
  char* smem = (char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  const uint32_t stage0 = smem_u32(smem);
  const uint32_t bars = smem_u32(smem + C::OFF_BARS);
  const uint32_t b_full = bars, b_empty = bars + 8 * C::NS, b_tfull = bars + 16 * C::NS, b_tempty = b_tfull + 16, b_drain = b_tempty + 16;
  uint32_t* slot = (uint32_t*)(smem + C::OFF_BARS + C::NBAR * 8);
  volatile int* abort_flag = (volatile int*)(slot + 1);
  int* dead_word = (int*)(slot + 2);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  ready_for_next();
  if (threadIdx.x == 0) {
    prefetch_tmap(&ta);
    prefetch_tmap(&tb);
    for (int s = 0; s < C::NS; ++s) {
      mbar_init(b_full + 8 * s, 1);
      mbar_init(b_empty + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(b_tfull + 8 * b, 1);
      mbar_init(b_tempty + 8 * b, C::EPILOGUE);
    }
    mbar_init(b_drain, 1);
    fence_mbar_init();
    *abort_flag = 0;
  }
  if (warp == C::ISSUER) {
    tmem_alloc(smem_u32(slot), C::TMEM);
    tmem_relinquish();
  }
  after_previous();
  if (threadIdx.x == 0) *dead_word = *(volatile int*)p.status;   // an earlier product's wait ran out: what follows has no input
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = *(volatile uint32_t*)slot;
  const bool dead = *dead_word != 0;
  if (warp == C::PRODUCER) {
    if (lane == 0 && !dead) {
      int64_t n = 0;
      bool ok = true;
      for (int w = blockIdx.x; w < p.items && ok; w += gridDim.x) {
        const Item t = item_of(p, w, BN);
        for (int k = t.k0; k < t.k1; ++k, ++n) {
          const int s = (int)(n % C::NS);
          if (!(ok = wait_bar(b_empty + 8 * s, (uint32_t)((n / C::NS) & 1) ^ 1u, abort_flag, p.status, 1))) break;
          const uint32_t full = b_full + 8 * s, dst = stage0 + s * C::STAGE;
          const bool once = BN == kBM && p.lower && t.i == t.j;   // on the diagonal both operands are one
          mbar_expect_tx(full, once ? C::A_BYTES : C::STAGE);
          if (AMN) {
#pragma unroll
            for (int q = 0; q < kBM / 64; ++q) tma_load_3d(dst + q * 2 * BK * 128, &ta, full, t.i * kBM + q * 64, k * BK, 0);
          } else {
            tma_load_3d(dst, &ta, full, k * BK, t.i * kBM, 0);
          }
          if (once) {
          } else if (BMN) {
#pragma unroll
            for (int q = 0; q < BN / 64; ++q)
              tma_load_3d(dst + C::A_BYTES + q * 2 * BK * 128, &tb, full, t.j * BN + q * 64, k * BK, 0);
          } else {
            tma_load_3d(dst + C::A_BYTES, &tb, full, k * BK, t.j * BN, 0);
          }
        }
      }
      if (!ok)   // copies still under way land before shared memory goes away
        for (int64_t k = n > C::NS ? n - C::NS : 0; k < n; ++k) {
          const uint64_t t0 = globaltimer_ns();
          while (!mbar_try_wait(b_full + 8 * (int)(k % C::NS), (uint32_t)((k / C::NS) & 1)) && globaltimer_ns() - t0 < 100000000ull) {
          }
        }
    }
    __syncwarp();
  } else if (warp == C::ISSUER) {
    if (!dead) {
      constexpr uint32_t idesc = idesc_fp16(kBM, BN, AMN, BMN);
      // between the hi and the lo tile of a stage, and between steps of 16 products
      constexpr uint32_t A_LO = AMN ? BK * 128 : kBM * BK * 2, B_LO = BMN ? BK * 128 : BN * BK * 2;
      constexpr uint32_t A_STEP = AMN ? 16 * 128 : 32, B_STEP = BMN ? 16 * 128 : 32;
      int64_t n = 0, ch = 0;
      bool ok = true;
      for (int w = blockIdx.x; w < p.items && ok; w += gridDim.x) {
        const Item t = item_of(p, w, BN);
        for (int k = t.k0; k < t.k1; ++k, ++n) {
          const int s = (int)(n % C::NS), buf = (int)(ch & 1);
          const int in = (k - t.k0) % p.chunk;
          if (in == 0 && !(ok = conv_wait(b_tempty + 8 * buf, (uint32_t)((ch >> 1) & 1) ^ 1u, abort_flag, p.status, 2))) break;
          if (!(ok = conv_wait(b_full + 8 * s, (uint32_t)((n / C::NS) & 1), abort_flag, p.status, 3))) break;
          fence_after();
          const bool once = BN == kBM && p.lower && t.i == t.j;
          const uint32_t a0 = stage0 + s * C::STAGE, b0 = once ? a0 : a0 + C::A_BYTES, d = tmem + buf * BN;
          const uint64_t ah = AMN ? sdesc(a0, 2 * BK * 128, 1024, SWZ_128B) : sdesc(a0, 16, BK * 16, kAlong);
          const uint64_t bh = BMN ? sdesc(b0, 2 * BK * 128, 1024, SWZ_128B) : sdesc(b0, 16, BK * 16, kAlong);
          // the small products first: what an addition loses is a part of the sum so far
#pragma unroll
          for (int q = 0; q < BK / 16; ++q) {
            const uint64_t a = ah + ((q * A_STEP) >> 4), b = bh + ((q * B_STEP) >> 4);
            mma_ss_elect(d, a + (A_LO >> 4), b, idesc, q > 0 || in > 0);
            mma_ss_elect(d, a, b + (B_LO >> 4), idesc, 1);
          }
#pragma unroll
          for (int q = 0; q < BK / 16; ++q) mma_ss_elect(d, ah + ((q * A_STEP) >> 4), bh + ((q * B_STEP) >> 4), idesc, 1);
          commit_elect(b_empty + 8 * s);
          if (in == p.chunk - 1 || k + 1 == t.k1) {
            commit_elect(b_tfull + 8 * buf);
            ++ch;
          }
        }
      }
      commit_elect(b_drain);   // every product issued has ended before TMEM is given back
      if (lane == 0) {
        const uint64_t t0 = globaltimer_ns();
        while (!mbar_try_wait(b_drain, 0) && globaltimer_ns() - t0 < 200000000ull) {
        }
      }
      __syncwarp();
    }
  } else if (warp < C::EPILOGUE) {
    constexpr int G = BN / 8 / C::EPILOGUE;   // groups of 32 columns of a warpgroup
    constexpr bool kShared = C::EPILOGUE > 8;   // two warps of the same rows use a square in turn
    const int part = warp >> 2, row = (warp & 3) * 32;
    const uint32_t lanes = (uint32_t)row << 16;
    float* square = (float*)(smem + C::OFF_TURN) + (warp & 7) * 1024;
    const float alpha = scale_of_sum(p);
    int64_t ch = 0;
    bool ok = !dead;
    for (int w = blockIdx.x; w < p.items; w += gridDim.x) {
      const Item t = item_of(p, w, BN);
      const int chunks = (t.k1 - t.k0 + p.chunk - 1) / p.chunk;
      float acc[G][32];
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int i = 0; i < 32; ++i) acc[g][i] = 0.f;
      for (int c = 0; c < chunks && ok; ++c, ++ch) {
        const int buf = (int)(ch & 1);
        if (!(ok = warp_wait(b_tfull + 8 * buf, (uint32_t)((ch >> 1) & 1), abort_flag, p.status, 4))) break;
        fence_after();
        if constexpr (kShared) {   // (96 registers a thread: half a group at a time)
#pragma unroll
          for (int h = 0; h < 2 * G; ++h) {
            uint32_t v[16];
            tmem_ld16(tmem + lanes + buf * BN + part * G * 32 + h * 16, v);
            tmem_wait_ld(v);
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[h / 2][h % 2 * 16 + i] += __uint_as_float(v[i]);
          }
          fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(b_tempty + 8 * buf);
        } else {
          uint32_t v[G][32];   // all loads, and the buffer is free again
#pragma unroll
          for (int g = 0; g < G; ++g) tmem_ld32(tmem + lanes + buf * BN + (part * G + g) * 32, v[g]);
#pragma unroll
          for (int g = 0; g < G; ++g) tmem_wait_ld(v[g]);
          fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(b_tempty + 8 * buf);
#pragma unroll
          for (int g = 0; g < G; ++g)
#pragma unroll
            for (int i = 0; i < 32; ++i) acc[g][i] += __uint_as_float(v[g][i]);
        }
      }
      if (!ok && p.mode != kResult && !kShared) break;   // (two warps that share a square meet to the end)
      const int64_t r = (int64_t)t.i * kBM + row;
      if (r >= p.M && p.mode != kPartial) continue;
#pragma unroll(kShared ? G : 1)
      for (int g = 0; g < G; ++g) {
        const int col = (part * G + g) * 32;
        if (kShared && part >= 2) named_bar_sync(1 + (warp & 7), 64);
        __syncwarp();
        float v[32];
#pragma unroll
        for (int k = 0; k < G; ++k)
          if (k == g) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = acc[k][i];
          }
        if (p.mode == kMatrix) {
          put_rows_of(p, alpha, v, square, r, (int64_t)t.j * BN + col);
        } else if (p.mode == kPartial) {
          float4* at = (float4*)(p.part + ((int64_t)w * kBM + row + lane) * BN + col);
#pragma unroll
          for (int q = 0; q < 8; ++q) at[q] = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) in_square(square, lane, i) = ok ? v[i] : NAN;   // the result of a wait that ran out shows
          __syncwarp();
          put_square<(BN > 64)>(p, alpha, square, r, (int64_t)t.j * BN + col);
        }
        if (kShared) {
          named_bar_sync(1 + (warp & 7), 64);
          if (part < 2) named_bar_sync(1 + (warp & 7), 64);
        }
      }
    }
  }
  fence_before();
  __syncthreads();
  if (warp == C::ISSUER) {
    fence_after();
    tmem_dealloc(tmem, C::TMEM);
  }
}

// The parts of a symmetric D added up in order, in pieces.  MANY: a CTA takes 32 columns
// of one row of a tile, eight groups of lanes every eighth part each; otherwise 32 rows
// and columns, which it turns in shared memory for the copy above the diagonal.
template <bool MANY>
__global__ void __launch_bounds__(kThreads) join_kernel(Gemm p, int BN) {
  __shared__ float sums[32][33];
  const int lane = threadIdx.x & 31, g = threadIdx.x >> 5;
  const int down = MANY ? kBM : kBM / 32, per = down * (BN / 32);
  ready_for_next();
  after_previous();
  const int tile = blockIdx.x / per, at = blockIdx.x - tile * per, r0 = at / (BN / 32) * (MANY ? 1 : 32), c0 = at % (BN / 32) * 32;
  const Item t = item_of(p, tile * p.splits, BN);
  const int64_t row0 = (int64_t)t.i * kBM + r0, col0 = (int64_t)t.j * BN + c0;
  if (row0 >= p.M || col0 > row0 + (MANY ? 0 : 31)) return;
  const float* x = p.part + ((int64_t)tile * p.splits * kBM + r0) * BN + c0 + lane;
  const int64_t apart = (int64_t)kBM * BN, plane = p.d.plane();
  const float scale = scale_of_sum(p);
  auto put = [&](int64_t row, int64_t col, float v) {
    __half hi, lo;
    split(v * scale, hi, lo);
    p.d.hi[row * p.d.ld + col] = hi;
    p.d.hi[plane + row * p.d.ld + col] = lo;
  };
  if (MANY) {
    float sum = 0.f;
#pragma unroll 8
    for (int s = g; s < p.splits; s += 8) sum += x[s * apart];
    sums[g][lane] = sum;
    __syncthreads();
    if (g != 0 || col0 + lane > row0) return;
#pragma unroll
    for (int i = 1; i < 8; ++i) sum += sums[i][lane];
    put(row0, col0 + lane, sum);
    if (col0 + lane < row0) put(col0 + lane, row0, sum);
    return;
  }
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = 0; s < p.splits; ++s)
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] += x[s * apart + (int64_t)(g + 8 * i) * BN];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = g + 8 * i;
    sums[r][lane] = sum[i];
    if (row0 + r < p.M && col0 + lane <= row0 + r) put(row0 + r, col0 + lane, sum[i]);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = g + 8 * i;
    if (row0 + lane < p.M && col0 + c < row0 + lane) put(col0 + c, row0 + lane, sums[lane][c]);
  }
}

// ------------------------------------------------------------------------------- host

inline size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

int sm_count() {
  static std::atomic<int> sms[kMaxDevices];
  return per_device(sms, [] {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
      return 0;
    return n;
  });
}

template <class... P, class... A>
nmd_status start(void (*kernel)(P...), int64_t grid, int threads, size_t smem, cudaStream_t s, A... args) {
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess ? NMD_OK : NMD_ERR_CUDA;
}

template <int BN, bool AMN, bool BMN>
nmd_status launch_bn(const Pieces& a, const Pieces& b, const Gemm& g, cudaStream_t s) {
  static std::atomic<int> ready[kMaxDevices];
  auto kernel = gemm_kernel<BN, AMN, BMN>;
  if (!per_device(ready, [&] {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg<BN>::SMEM) == cudaSuccess;
      }))
    return NMD_ERR_CUDA;
  CUtensorMap ta, tb;
  constexpr int BK = Cfg<BN>::BK;
  if (!map_of(a, AMN ? BK : kBM, &ta, AMN ? 64 : BK) || !map_of(b, BMN ? BK : BN, &tb, BMN ? 64 : BK)) return NMD_ERR_CUDA;
  const int sms = sm_count();
  if (sms == 0) return NMD_ERR_CUDA;
  return start(kernel, std::min(g.items, sms), Cfg<BN>::THREADS, Cfg<BN>::SMEM, s, ta, tb, g);
}
template <bool AMN, bool BMN>
nmd_status launch(int BN, const Pieces& a, const Pieces& b, const Gemm& g, cudaStream_t s) {
  if (BN == 256) return launch_bn<256, AMN, BMN>(a, b, g, s);
  if (BN == 128) return launch_bn<128, AMN, BMN>(a, b, g, s);
  return launch_bn<64, AMN, BMN>(a, b, g, s);
}

int64_t tiles_of(int64_t M, int64_t N, int BN, bool lower) {
  const int64_t tm = (M + kBM - 1) / kBM, tn = (N + BN - 1) / BN;
  if (!lower) return tm * tn;
  int64_t n = 0;
  for (int64_t i = 0; i < tm; ++i) n += std::min<int64_t>((kBM * (i + 1) - 1) / BN + 1, tn);
  return n;
}
// Tiles of 256, 128 or 64 columns: those whose rounds over the SMs take least, at 2200,
// 1250 and 940 cycles a block of the sum.  Tiles of 256 move a quarter less per product
// through shared memory (1875 cycles for 1536 of products), but take twice as long after their last one, and lose where a sum leaves TMEM every 64
// columns: `wide` for 16-bit results and deep sums.  With them 4096 x 4096 in bf16 takes
// 3.17 instead of 3.33 ms, 8192 x 2560 2.22 instead of 2.39, 11008 x 4096 7.1 instead of
// 7.5; sums of 512 (16384 x 512) 416 instead of 405 us, fp32 4096 x 4096 4.02 instead of
// 3.88 ms.  (Pairs of CTAs that share the second operand, 256 x 256 by both: 3.21 ms in
// three stages, 3.39 in six of half the depth.)
constexpr int64_t kWideDepth = 1280;
int columns_of(int64_t M, int64_t N, bool lower, bool wide) {
  int best = 64;
  int64_t least = INT64_MAX;
  for (const int BN : {256, 128, 64}) {
    if ((BN > 64 && N <= BN / 2) || (BN > 128 && !wide)) continue;
    const int64_t cycles = (tiles_of(M, N, BN, lower) + kSms - 1) / kSms * (BN == 256 ? 2200 : BN == 128 ? 1250 : 940);
    if (cycles < least) {
      least = cycles;
      best = BN;
    }
  }
  return best;
}

// The sums of a Gram matrix run over the long side: tiles, and parts of the sum where there are few of them
struct GramPlan {
  int BN;
  int64_t tiles, splits;
};
GramPlan gram_plan(int64_t r, int64_t M, bool wide) {
  GramPlan g;
  const int64_t blocks = (M + kBK - 1) / kBK;
  // A sum of 20 blocks takes what adding parts up would (8 us).  Five steps with whole sums and
  // with parts: 318 x 1280 185 and 182 us, x 1920 215 and 203, x 2560 246 and 185; 556 x 960
  // 194 and 213, x 1280 211 and 233, x 1920 248 and 238; 1001 x 1280 278 and 298.
  if (blocks <= 20) {
    g.BN = columns_of(r, r, true, wide);
    g.tiles = tiles_of(r, r, g.BN, true);
    g.splits = 1;
    return g;
  }
  g.BN = r <= 64 ? 64 : 128;
  g.tiles = tiles_of(r, r, g.BN, true);
  g.splits = std::max<int64_t>(1, std::min<int64_t>(kSms / g.tiles, blocks / 2));
  if (g.splits == 1) {
    g.BN = columns_of(r, r, true, wide);
    g.tiles = tiles_of(r, r, g.BN, true);
  }
  return g;
}

// What a call keeps in its workspace
struct Layout {
  size_t status, parts, X[2], A, P, part, bytes;
  int64_t R, C, ldx, r, ldr;
  bool strip;
};
Layout layout_of(int64_t R, int64_t C) {
  Layout l;
  l.R = R;
  l.C = C;
  l.ldx = (C + 63) / 64 * 64;
  l.r = std::min(R, C);
  l.ldr = (l.r + 63) / 64 * 64;
  const GramPlan g = gram_plan(l.r, std::max(R, C), false);
  l.strip = l.r <= kStripSide && std::max(R, C) <= kStripMost;
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t here = at;
    at += align256(n);
    return here;
  };
  l.status = take(kInts * sizeof(int));
  l.parts = take(kParts * sizeof(double));
  // A strip's X in pieces, a row per row of the long side; the rest where the products take its place
  const size_t x_bytes = l.strip ? (size_t)std::max(R, C) * 64 * 4 : (size_t)R * l.ldx * 4;
  for (size_t& x : l.X) x = take(x_bytes);
  l.A = take((size_t)l.r * l.ldr * 4);
  l.P = take((size_t)l.r * l.ldr * 4);
  l.part = take(std::max(g.splits > 1 ? (size_t)(g.tiles * g.splits) * kBM * g.BN * 4 : 0,
                         l.strip ? strip_bytes(std::max(R, C)) : 0));
  l.bytes = at;
  return l;
}

template <class F>
void with_type(int dtype, F f) {
  if (dtype == NMD_DT_FP32) f(0.f);
  else if (dtype == NMD_DT_BF16) f(bf16{});
  else f(__half{});
}

void turn(Job* j) {   // the transpose of every matrix: the steps are the same
  std::swap(j->R, j->C);
  for (Matrix* m : {&j->grad, &j->momentum, &j->out}) std::swap(m->rs, m->cs);
}

nmd_status run(Job j, int steps, const double* k, void* ws, cudaStream_t s) {
  const Layout l = layout_of(j.R, j.C);
  char* w = (char*)ws;
  int* status = (int*)(w + l.status);
  int* shift = status + kShift;
  double* parts = (double*)(w + l.parts);
  Pieces X{(__half*)(w + l.X[0]), j.R, j.C, l.ldx}, Y{(__half*)(w + l.X[1]), j.R, j.C, l.ldx};
  const bool turned = l.strip && j.R <= j.C;
  j.flat = filled(j.grad, j.C) && (!j.step || filled(j.momentum, j.C));
  if (l.strip) X = Pieces{X.hi, std::max(j.R, j.C), l.r, 64};
  const Pieces A{(__half*)(w + l.A), l.r, l.r, l.ldr}, P{(__half*)(w + l.P), l.r, l.r, l.ldr};
  const int64_t r = l.r, M = std::max(j.R, j.C);
  const int grid = (int)std::min<int64_t>(j.flat ? (j.R * j.C + 8 * kThreads - 1) / (8 * kThreads)
                                                 : (walk_of(j.R, j.C).work + kThreads / 32 - 1) / (kThreads / 32), kParts);
  const int grid_x = (int)std::min<int64_t>((X.rows * X.ld / 8 + kThreads - 1) / kThreads, kParts);
  const int grows = (int)std::ceil(std::log2(std::max(1.0, 1.001 * std::fabs(k[0]))));
  nmd_status st = NMD_OK;
  with_type(j.grad.dtype, [&](auto g) {
    with_type(j.step ? j.momentum.dtype : j.grad.dtype, [&](auto m) {
      typedef decltype(g) G;
      typedef decltype(m) M;
      auto both = [&](auto norm, auto pieces) {
        st = start(norm, grid, kThreads, 0, s, j, parts, status);
        if (st == NMD_OK) st = start(pieces, grid_x, kThreads, 0, s, j, X, (const double*)parts, grid, shift, steps, grows);
      };
      if (j.step) both(norm_kernel<G, M, true>, turned ? turned_kernel<G, M, true> : pieces_kernel<G, M, true>);
      else both(norm_kernel<G, G, false>, turned ? turned_kernel<G, G, false> : pieces_kernel<G, G, false>);
    });
  });
  if (st != NMD_OK) return st;
  if (l.strip) {
    if (strip_run(j, X, steps, k, status, w + l.part, s) == NMD_OK) return NMD_OK;
    // Its CTAs wait for one another and are launched only if all can run at a time, which a
    // context with a part of the SMs does not give.  The momentum is on its way, so the
    // products below, which wait for none, take X as it is.
    (void)cudaGetLastError();
    if (turned) turn(&j);
    Y = Pieces{Y.hi, X.rows, X.cols, X.ld};
  }
  const bool wide = j.R <= j.C;   // X is r x M; otherwise M x r
  auto wide_tiles = [&](int64_t depth) { return j.out.dtype != NMD_DT_FP32 && depth >= kWideDepth; };
  const GramPlan plan = gram_plan(r, M, wide_tiles(M));
  const int bn_r = columns_of(r, r, true, wide_tiles(r)), bn_x = columns_of(j.R, j.C, false, wide_tiles(r));
  auto product = [&](int64_t m, int64_t n, int64_t depth, int BN, bool lower, Mode mode) {
    Gemm g{};
    g.M = m;
    g.N = n;
    g.kblocks = (int)((depth + depth_of(BN) - 1) / depth_of(BN));
    g.splits = 1;
    g.tiles_m = (int)((m + kBM - 1) / kBM);
    g.tiles_n = (int)((n + BN - 1) / BN);
    g.items = (int)tiles_of(m, n, BN, lower);
    g.lower = lower;
    g.mode = mode;
    g.status = status;
    // Sums of 256 lean more than those of 64: before its rounding (1.66e-3 of the norm in
    // bf16) a result of 256 x 139,255 is 1.5e-5 off instead of 3.1e-6, of 4096 x 4096 3.8e-6
    // instead of 1.3e-6, so that single elements round to a neighbour (2.7e-4 and 1.1e-4
    // from the rounded definition instead of 1.2e-4 and 7e-5).  A whole sum of that length
    // in TMEM lets the epilogue work beside the next tile's products: 706 instead of 808 us,
    // 3.46 instead of 4.13 ms.  (Sums of 128: 7.3e-6 and 2.0e-6, 722 us and 3.72 ms.)
    g.chunk = (j.out.dtype == NMD_DT_FP32 ? 64 : 256) / depth_of(BN);
    return g;
  };
  for (int i = 0; i < steps; ++i) {
    // A = X X^T: 2^24 a in the sums, 2^12 a in the pieces
    Gemm g = product(r, r, M, plan.BN, true, plan.splits > 1 ? kPartial : kSymmetric);
    g.alpha = 1.f / kUnit;
    g.d = A;
    g.down = shift + i;
    g.times = 2;
    g.splits = (int)plan.splits;
    g.items *= g.splits;
    g.part = (float*)(w + l.part);
    st = wide ? launch<false, false>(plan.BN, X, X, g, s) : launch<true, true>(plan.BN, X, X, g, s);
    if (st != NMD_OK) return st;
    if (plan.splits > 1) {
      st = plan.splits > 16 ? start(join_kernel<true>, plan.tiles * kBM * (plan.BN / 32), kThreads, 0, s, g, plan.BN)
                            : start(join_kernel<false>, plan.tiles * (kBM / 32) * (plan.BN / 32), kThreads, 0, s, g, plan.BN);
      if (st != NMD_OK) return st;
    }
    // P = a I + b A + c A A
    g = product(r, r, r, bn_r, true, kSymmetric);
    g.alpha = (float)(k[2] / kUnit);
    g.beta = (float)k[1];
    g.diag = (float)(k[0] * kUnit);
    g.c = A;
    g.d = P;
    if ((st = launch<false, false>(bn_r, A, A, g, s)) != NMD_OK) return st;
    // X <- P X, or X P: P is symmetric
    const bool last = i + 1 == steps;
    g = product(j.R, j.C, r, bn_x, false, last ? kResult : kMatrix);
    g.alpha = last ? 1.f / (kUnit * kUnit) : 1.f / kUnit;
    g.up = last ? nullptr : shift + i + 1;
    g.down = shift + i;
    g.times = 1;
    g.d = Y;
    g.out = j;
    st = wide ? launch<false, true>(bn_x, P, X, g, s) : launch<false, false>(bn_x, X, P, g, s);
    if (st != NMD_OK) return st;
    std::swap(X, Y);
  }
  return NMD_OK;
}

// How far the elements of a matrix reach (a stride may be 0), and whether they lie apart; false where
// that is no distance in memory
constexpr int64_t kMostReach = (int64_t)1 << 44;   // elements
bool reach_of(int64_t rows, int64_t cols, int64_t rs, int64_t cs, int64_t* reach, bool* apart) {
  if (rs < 0 || cs < 0 || rs > kMostReach || cs > kMostReach) return false;
  int64_t n[2] = {rows, cols}, st[2] = {rs, cs};
  if (n[0] > 1 && n[1] > 1 && st[0] < st[1]) std::swap(n[0], n[1]), std::swap(st[0], st[1]);
  int64_t span = 1;
  *apart = true;
  for (int i = 1; i >= 0; --i) {
    if (n[i] <= 1) continue;
    if (st[i] > kMostReach / n[i]) return false;
    *apart &= st[i] >= span;
    span += (n[i] - 1) * st[i];
  }
  *reach = span;
  return true;
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
  bool apart = false;
  if (!reach_of(rows, cols, rs, cs, &reach, &apart) || (unique && !apart)) return false;
  *at = Range{(uintptr_t)x, (uintptr_t)x + (uintptr_t)(reach * size_of(dtype))};
  return true;
}
// whether the rows' elements lie further apart than the columns'
bool columns_apart(int64_t rows, int64_t cols, int64_t rs, int64_t cs) {
  return rows > 1 && (cols <= 1 || rs < cs);
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
  // either side may be the adjacent one
  *bytes = rows == 0 || cols == 0 ? 256 : std::max(layout_of(rows, cols).bytes, layout_of(cols, rows).bytes);
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
  j.R = rows;
  j.C = cols;
  j.grad = Matrix{(void*)d_update, dtype, row_stride, col_stride};
  j.out = Matrix{d_out, dtype, out_row_stride, out_col_stride};
  j.eps = eps;
  if (columns_apart(rows, cols, row_stride, col_stride)) turn(&j);
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
  j.R = rows;
  j.C = cols;
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
  if (columns_apart(rows, cols, weight->row_stride, weight->col_stride)) turn(&j);
  return run(j, steps, coefficients, d_workspace, (cudaStream_t)stream);
}

}  // extern "C"

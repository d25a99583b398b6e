// Log-probability of one column per row of softmax(A B^T / tau) without the
// T x n matrix of scores:  log p_t = a_t . b_y / tau - log sum_j exp(a_t . b_j / tau).
//
// The scores are formed tile by tile on the tcgen05 tensor cores (128 rows of A
// against chunks of 128 rows of B) in TMEM, and the epilogue warps reduce each
// row of a tile to a running maximum m and S = sum 2^(c (z - m)), c = log2(e) /
// tau, as the row kernels of the logits do.  Nothing of the scores is written.
//
// 16-bit factors are multiplied as they are.  fp32 factors are split into three
// bf16 pieces each (x = hi + lo + lo2 to 2^-24 of x), and the six products of
// pieces above 2^-24 are accumulated in fp32: hi hi, hi lo, lo hi, lo lo,
// hi lo2, lo2 hi.
//
// The tiles x chunks are dealt to one CTA per SM in equal contiguous runs, so
// that any T and n fill the GPU; a run that crosses into the next tile of rows
// writes its (m, S) and starts over, and the second kernel merges a row's
// partial results in the order of the chunks and takes the dot product a_t . b_y
// in fp32 on the CUDA cores.
//
// Warp roles (320 threads): warps 0-7 epilogue (two warpgroups on alternate
// chunks; thread t of each owns TMEM lane t = row t), warp 8 TMA and TMEM
// allocation, warp 9 issues the MMAs.  Waits are bounded (2 s): a CTA whose wait
// ran out flags its run, and the rows it would have counted become NaN.
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include "nmd_internal.cuh"
#include "tc_pipe.cuh"
#include "tc_ptx.cuh"

namespace nmd {
namespace {

using namespace tc;

constexpr int BM = 128, BN = 128;
constexpr int kEpiWarps = 8, kTmaWarp = 8, kMmaWarp = 9, kThreads = 320;
constexpr int kPanel = BM * 128;            // bytes of 128 rows x 64 16-bit columns
constexpr int kMaxCtas = 256;
constexpr int kMaxRank = 256;

// PIECES: bf16 pieces of each factor (1: 16-bit factors).  ARES: the tile of A
// stays in shared memory for the whole run; otherwise (fp32 at rank > 128,
// whose tile would take 192 KB) its panels are loaded beside those of B.
template <int PIECES, bool ARES>
struct Cfg {
  static constexpr int A_PANELS = ARES ? (PIECES == 1 ? 4 : 2) : 0;
  static constexpr int A_BYTES = PIECES * A_PANELS * kPanel;
  static constexpr int STAGE = PIECES * kPanel * (ARES ? 1 : 2);
  static constexpr int NST = PIECES == 1 ? 8 : 2;
  static constexpr int NB = 512 / BN;       // TMEM buffers
  static constexpr int NBAR = 2 * NST + 2 * NB + 3;
  static constexpr size_t SMEM = 1024 + A_BYTES + (size_t)NST * STAGE + NBAR * 8 + 64;
  static_assert(SMEM <= 227 * 1024, "shared memory per block");
  static_assert(SMEM > 114 * 1024, "one CTA (and its 512 TMEM columns) per SM");
};

struct Stat {
  float m, S;
};

struct Params {
  int64_t T, n, C, W;        // rows, columns, chunks per tile, tiles x chunks
  int r, npan;               // rank, panels of 64
  int slots;                 // partial results kept per tile (x 2 warpgroups)
  float c;
  uint32_t idesc;
  Stat* parts;               // [tile][slot][warpgroup][128]
  int* flags;                // 2 per CTA: nmd_status, detail
};

// CTA that works on unit u of W dealt to G CTAs, CTA b taking [b W / G, (b + 1) W / G)
__host__ __device__ __forceinline__ int64_t owner(int64_t u, int64_t W, int64_t G) { return ((u + 1) * G - 1) / W; }

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ Stat merge(const Stat& a, const Stat& b, float c) {
  const float m = fmaxf(a.m, b.m), z = base_of(m);
  return {m, a.S * ex2((a.m - z) * c) + b.S * ex2((b.m - z) * c)};
}

template <int PIECES, bool ARES>
__global__ void __launch_bounds__(kThreads, 1)
    score_kernel(const __grid_constant__ CUtensorMap ta0, const __grid_constant__ CUtensorMap ta1,
                 const __grid_constant__ CUtensorMap ta2, const __grid_constant__ CUtensorMap tb0,
                 const __grid_constant__ CUtensorMap tb1, const __grid_constant__ CUtensorMap tb2, const Params p) {
  using C = Cfg<PIECES, ARES>;
  constexpr int NST = C::NST, NB = C::NB;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  const uint32_t a_sm = smem_u32(smem), st_sm = a_sm + C::A_BYTES;
  uint64_t* bars = (uint64_t*)(smem + C::A_BYTES + (size_t)NST * C::STAGE);
  uint32_t* tmem_slot = (uint32_t*)(bars + C::NBAR);
  volatile int* abort_flag = (volatile int*)(tmem_slot + 1);
  const uint32_t b_full = smem_u32(bars), b_empty = b_full + 8 * NST, b_lfull = b_empty + 8 * NST,
                 b_lfree = b_lfull + 8 * NB, b_afull = b_lfree + 8 * NB, b_aempty = b_afull + 8,
                 b_drain = b_aempty + 8;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int* status = p.flags + 2 * blockIdx.x;
  if (threadIdx.x == 0) {
    for (int i = 0; i < NST; ++i) {
      mbar_init(b_full + 8 * i, 1);
      mbar_init(b_empty + 8 * i, 1);
    }
    for (int i = 0; i < NB; ++i) {
      mbar_init(b_lfull + 8 * i, 1);
      mbar_init(b_lfree + 8 * i, 4);
    }
    mbar_init(b_afull, 1);
    mbar_init(b_aempty, 1);
    mbar_init(b_drain, 1);
    *abort_flag = 0;
    status[0] = 0;
    status[1] = 0;
    fence_mbar_init();
  }
  if (warp == kTmaWarp) {
    tmem_alloc(smem_u32(tmem_slot), 512);
    tmem_relinquish();
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = *tmem_slot;

  const int64_t u0 = blockIdx.x * p.W / gridDim.x, u1 = (blockIdx.x + 1) * p.W / gridDim.x;
  const int64_t tile0 = u0 / p.C;

  if (warp == kTmaWarp) {
    if (lane == 0) {
      int s = 0;
      uint32_t ph = 1, aph = 1;
      int64_t loads = 0, aloads = 0;
      bool ok = true;
      int64_t tile = tile0, c = u0 - tile0 * p.C;
      bool first = true;
      for (int64_t u = u0; u < u1 && ok; ++u) {
        if (ARES && first) {
          if (!(ok = wait_bar(b_aempty, aph, abort_flag, status, 10))) break;
          aph ^= 1u;
          mbar_expect_tx(b_afull, PIECES * p.npan * kPanel);
          for (int k = 0; k < p.npan; ++k) {
            const uint32_t dst = a_sm + k * PIECES * kPanel;
            tma_load_2d(dst, &ta0, b_afull, 64 * k, (int)(tile * BM));
            if (PIECES > 1) tma_load_2d(dst + kPanel, &ta1, b_afull, 64 * k, (int)(tile * BM));
            if (PIECES > 1) tma_load_2d(dst + 2 * kPanel, &ta2, b_afull, 64 * k, (int)(tile * BM));
          }
          ++aloads;
          first = false;
        }
        for (int k = 0; k < p.npan; ++k) {
          if (!(ok = wait_bar(b_empty + 8 * s, ph, abort_flag, status, 1))) break;
          const uint32_t dst = st_sm + s * C::STAGE, bar = b_full + 8 * s;
          mbar_expect_tx(bar, C::STAGE);
          tma_load_2d(dst, &tb0, bar, 64 * k, (int)(c * BN));
          if (PIECES > 1) tma_load_2d(dst + kPanel, &tb1, bar, 64 * k, (int)(c * BN));
          if (PIECES > 1) tma_load_2d(dst + 2 * kPanel, &tb2, bar, 64 * k, (int)(c * BN));
          if (!ARES) {
            tma_load_2d(dst + PIECES * kPanel, &ta0, bar, 64 * k, (int)(tile * BM));
            if (PIECES > 1) tma_load_2d(dst + (PIECES + 1) * kPanel, &ta1, bar, 64 * k, (int)(tile * BM));
            if (PIECES > 1) tma_load_2d(dst + (PIECES + 2) * kPanel, &ta2, bar, 64 * k, (int)(tile * BM));
          }
          ++loads;
          if (++s == NST) {
            s = 0;
            ph ^= 1u;
          }
        }
        if (++c == p.C) {
          c = 0;
          ++tile;
          first = true;
        }
      }
      if (!ok) {   // wait for the copies in flight before shared memory goes away
        for (int64_t k = loads > NST ? loads - NST : 0; k < loads; ++k) {
          const uint64_t t0 = globaltimer_ns();
          while (!mbar_try_wait(b_full + 8 * (int)(k % NST), (uint32_t)((k / NST) & 1)) &&
                 globaltimer_ns() - t0 < 100000000ull) {
          }
        }
        if (aloads > 0) {
          const uint64_t t0 = globaltimer_ns();
          while (!mbar_try_wait(b_afull, (uint32_t)((aloads - 1) & 1)) && globaltimer_ns() - t0 < 100000000ull) {
          }
        }
      }
    }
  } else if (warp == kMmaWarp) {
    int s = 0, lb = 0;
    uint32_t ph = 0, lph = 1, aph = 0;
    bool ok = true, first = true;
    int64_t c = u0 - tile0 * p.C;
    for (int64_t u = u0; u < u1 && ok; ++u) {
      if (ARES && first) {
        if (!(ok = conv_wait(b_afull, aph, abort_flag, status, 2))) break;
        aph ^= 1u;
        first = false;
      }
      if (!(ok = conv_wait(b_lfree + 8 * lb, lph, abort_flag, status, 4))) break;
      const uint32_t d = tmem + lb * BN;
      for (int k = 0; k < p.npan; ++k) {
        if (!(ok = conv_wait(b_full + 8 * s, ph, abort_flag, status, 3))) break;
        fence_after();
        const uint32_t bs = st_sm + s * C::STAGE;
        const uint64_t db = sdesc(bs, 16, 1024, SWZ_128B);
        const uint64_t da = sdesc(ARES ? a_sm + k * PIECES * kPanel : bs + PIECES * kPanel, 16, 1024, SWZ_128B);
        const int steps = min(4, (p.r - 64 * k + 15) / 16);
        for (int q = 0; q < steps; ++q) {
          const uint32_t acc = (k | q) != 0;
          if (PIECES == 1) {
            mma_ss_elect(d, da + 2 * q, db + 2 * q, p.idesc, acc);
          } else {
            constexpr uint64_t P = kPanel >> 4;
            mma_ss_elect(d, da + 2 * q + P, db + 2 * q + P, p.idesc, acc);          // lo lo
            mma_ss_elect(d, da + 2 * q + 2 * P, db + 2 * q, p.idesc, 1);            // lo2 hi
            mma_ss_elect(d, da + 2 * q, db + 2 * q + 2 * P, p.idesc, 1);            // hi lo2
            mma_ss_elect(d, da + 2 * q + P, db + 2 * q, p.idesc, 1);                // lo hi
            mma_ss_elect(d, da + 2 * q, db + 2 * q + P, p.idesc, 1);                // hi lo
            mma_ss_elect(d, da + 2 * q, db + 2 * q, p.idesc, 1);                    // hi hi
          }
        }
        commit_elect(b_empty + 8 * s);
        if (++s == NST) {
          s = 0;
          ph ^= 1u;
        }
      }
      if (!ok) break;
      commit_elect(b_lfull + 8 * lb);
      if (++lb == NB) {
        lb = 0;
        lph ^= 1u;
      }
      if (++c == p.C) {
        c = 0;
        if (ARES) commit_elect(b_aempty);
        first = true;
      }
    }
    commit_elect(b_drain);   // every MMA issued has to be over before TMEM is freed
    if (lane == 0) {
      const uint64_t t0 = globaltimer_ns();
      while (!mbar_try_wait(b_drain, 0) && globaltimer_ns() - t0 < 200000000ull) {
      }
    }
    __syncwarp();
  } else {
    const int wg = warp >> 2, quarter = warp & 3;
    const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
    const float cc = p.c;
    Stat st{-INFINITY, 0.f};
    float lost = 0.f;   // what the additions to S have rounded away (compensated summation)
    bool ok = true;
    int64_t tile = tile0, c = u0 - tile0 * p.C;
    for (int64_t u = u0; u < u1 && ok; ++u) {
      const int64_t G = u - u0;
      if ((int)(G & 1) == wg) {
        const int lb = (int)(G % NB);
        if (!(ok = warp_wait(b_lfull + 8 * lb, (uint32_t)((G / NB) & 1), abort_flag, status, 7))) break;
        fence_after();
        if (tile * BM + quarter * 32 < p.T) {   // some row of this warp exists
          const int kv = (int)min((int64_t)BN, p.n - c * BN);
          const uint32_t col = tmem + lane_base + lb * BN;
#pragma unroll 1
          for (int j = 0; j < kv; j += 64) {
            uint32_t v[2][32];
            tmem_ld32(col + j, v[0]);
            tmem_ld32(col + j + 32, v[1]);
            tmem_wait_ld(v[0]);
            tmem_wait_ld(v[1]);
            if (kv < j + 64) {   // columns past the last count as -inf
#pragma unroll
              for (int i = 0; i < 64; ++i)
                if (j + i >= kv) v[i >> 5][i & 31] = 0xff800000u;
            }
            float m = -INFINITY;
#pragma unroll
            for (int i = 0; i < 64; ++i) m = fmaxf(m, __uint_as_float(v[i >> 5][i & 31]));
            if (m > st.m) {
              const float f = ex2((st.m - m) * cc);
              st.S *= f;
              lost *= f;
              st.m = m;
            }
            const float z = base_of(st.m);
            float t = 0.f;
#pragma unroll
            for (int i = 0; i < 64; ++i) t += ex2((__uint_as_float(v[i >> 5][i & 31]) - z) * cc);
            const float y = t - lost, sum = st.S + y;
            lost = (sum - st.S) - y;
            st.S = sum;
          }
        }
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(b_lfree + 8 * lb);
      }
      if (++c == p.C || u + 1 == u1) {   // the end of a tile, or of the run: hand over the row's partial result
        const int64_t slot = blockIdx.x - owner(tile * p.C, p.W, gridDim.x);
        p.parts[((tile * p.slots + slot) * 2 + wg) * BM + quarter * 32 + lane] = st;
        st = Stat{-INFINITY, 0.f};
        lost = 0.f;
        c = 0;
        ++tile;
      }
    }
  }
  fence_before();
  __syncthreads();
  fence_after();
  if (warp == kTmaWarp) tmem_dealloc(tmem, 512);
}

template <class T>
__device__ __forceinline__ float value(T x);
template <>
__device__ __forceinline__ float value(float x) { return x; }
template <>
__device__ __forceinline__ float value(bf16 x) { return __bfloat162float(x); }
template <>
__device__ __forceinline__ float value(__half x) { return __half2float(x); }

// One warp per row: its partial results merged, the target's score, the difference.
template <class T>
__global__ void __launch_bounds__(256)
    finish_kernel(const T* A, int64_t ar, int64_t ac, const T* B, int64_t br, int64_t bc, const int64_t* y,
                  float inv_temp, const Params p, int64_t G, float* logps) {
  const int64_t t = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (t >= p.T) return;
  const int64_t yt = y[t];
  if (yt < 0 || yt >= p.n) {
    if (lane == 0) logps[t] = yt < 0 ? 0.f : NAN;
    return;
  }
  const int64_t tile = t / BM, b0 = owner(tile * p.C, p.W, G), b1 = owner(tile * p.C + p.C - 1, p.W, G);
  Stat st{-INFINITY, 0.f};
  int bad = 0;
  for (int64_t k = lane; k < 2 * (b1 - b0 + 1); k += 32) {
    st = merge(st, p.parts[(tile * p.slots * 2 + k) * BM + t % BM], p.c);
    bad |= p.flags[2 * (b0 + k / 2)];
  }
  float z = 0.f;
  for (int k = lane; k < p.r; k += 32) z = fmaf(value(A[t * ar + k * ac]), value(B[yt * br + k * bc]), z);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const Stat other{__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.S, o)};
    st = merge(st, other, p.c);
    z += __shfl_xor_sync(0xffffffffu, z, o);
    bad |= __shfl_xor_sync(0xffffffffu, bad, o);
  }
  if (lane == 0) logps[t] = bad ? NAN : (z - st.m) * inv_temp - logf(st.S);
}

// Rows x columns of any strides into row-major 16-bit pieces with row stride rp
// (a multiple of 8 elements, as TMA asks), through tiles of 32 x 32 so that
// both sides are read and written along their rows.
template <class T, class D, int PIECES>
__global__ void __launch_bounds__(256)
    piece_kernel(const T* src, int64_t sr, int64_t sc, int64_t rows, int r, int rp, D* d0, D* d1, D* d2) {
  __shared__ T tile[32][33];
  const int64_t row0 = (int64_t)blockIdx.x * 32;
  const int col0 = blockIdx.y * 32;
  const int a = threadIdx.x & 31, b = threadIdx.x >> 5;
  for (int i = b; i < 32; i += 8) {   // lanes along the dimension whose stride is the smaller
    const int64_t row = row0 + (sc <= sr ? i : a);
    const int col = col0 + (sc <= sr ? a : i);
    if (row < rows && col < r) tile[row - row0][col - col0] = src[row * sr + col * sc];
  }
  __syncthreads();
  for (int i = b; i < 32; i += 8) {
    const int64_t row = row0 + i;
    const int col = col0 + a;
    if (row >= rows || col >= r) continue;
    if constexpr (PIECES == 1) {
      d0[row * rp + col] = tile[i][a];
    } else {
      const float x = tile[i][a];
      const bf16 h = __float2bfloat16_rn(x);
      const float e = x - __bfloat162float(h);
      const bf16 l = __float2bfloat16_rn(e);
      d0[row * rp + col] = h;
      d1[row * rp + col] = l;
      d2[row * rp + col] = __float2bfloat16_rn(e - __bfloat162float(l));
    }
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
// Where a factor's pieces lie: its own memory where TMA can read it, else packed.
struct Operand {
  bool packed;
  int64_t stride;       // elements between rows of the pieces
  size_t at, piece;     // offset in the workspace, bytes of one piece
};

struct Layout {
  Operand a, b;
  size_t parts, flags, total;
  int64_t tiles, C;
  int pieces, slots;
};

Operand operand(const void* base, int64_t row, int64_t col, int dtype, int64_t rows, int64_t r, size_t* off) {
  Operand o{};
  o.packed = dtype == NMD_DT_FP32 || (r > 1 && col != 1) || ((uintptr_t)base & 15) ||
             (rows > 1 && (row % 8 != 0 || row < r));
  o.stride = !o.packed && rows > 1 ? row : (r + 7) / 8 * 8;
  if (o.packed) {
    o.piece = ((size_t)rows * o.stride * 2 + 255) & ~size_t(255);
    o.at = *off;
    *off += o.piece * (dtype == NMD_DT_FP32 ? 3 : 1);
  }
  return o;
}

Layout layout(const void* A, int64_t ar, int64_t ac, const void* B, int64_t br, int64_t bc, int dtype, int64_t T,
              int64_t n, int64_t r) {
  Layout L{};
  size_t off = 0;
  L.pieces = dtype == NMD_DT_FP32 ? 3 : 1;
  L.a = operand(A, ar, ac, dtype, T, r, &off);
  L.b = operand(B, br, bc, dtype, n, r, &off);
  L.tiles = (T + BM - 1) / BM;
  L.C = (n + BN - 1) / BN;
  // a tile's chunks are spread over at most (CTAs / tiles) + 2 CTAs
  L.slots = (int)std::min<int64_t>(kMaxCtas, kMaxCtas / std::max<int64_t>(1, L.tiles) + 2);
  L.parts = off;
  off += ((size_t)L.tiles * L.slots * 2 * BM * sizeof(Stat) + 255) & ~size_t(255);
  L.flags = off;
  off += kMaxCtas * 2 * sizeof(int);
  L.total = off;
  return L;
}

bool bad_sizes(int64_t ar, int64_t ac, int64_t br, int64_t bc, int dtype, int64_t T, int64_t n, int64_t r) {
  return dtype < NMD_DT_FP32 || dtype > NMD_DT_FP16 || T < 0 || T > (int64_t(1) << 27) || n < 1 ||
         n >= (int64_t(1) << 31) || r < 1 || r > kMaxRank || ar < 0 || ac < 0 || br < 0 || bc < 0;
}

bool encode(const void* base, int64_t rows, int64_t r, int64_t stride, int dtype, CUtensorMap* m) {
  PFN_cuTensorMapEncodeTiled_v12000 fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {(cuuint64_t)r, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)stride * 2};
  cuuint32_t box[2] = {64, BM}, es[2] = {1, 1};
  return fn(m, dtype == NMD_DT_FP16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2,
            const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int PIECES, bool ARES>
nmd_status launch_scores(const CUtensorMap* ta, const CUtensorMap* tb, const Params& p, int grid, cudaStream_t s) {
  using C = Cfg<PIECES, ARES>;
  static std::atomic<int> attr[kMaxDevices];
  if (!per_device(attr, [] {
        return cudaFuncSetAttribute(score_kernel<PIECES, ARES>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    (int)C::SMEM) == cudaSuccess ? 1 : 0;
      }))
    return NMD_ERR_CUDA;
  constexpr int k1 = PIECES > 1 ? 1 : 0, k2 = PIECES > 1 ? 2 : 0;
  score_kernel<PIECES, ARES><<<grid, kThreads, C::SMEM, s>>>(ta[0], ta[k1], ta[k2], tb[0], tb[k1], tb[k2], p);
  return cudaGetLastError() == cudaSuccess ? NMD_OK : NMD_ERR_CUDA;
}

void pack(const void* src, int64_t sr, int64_t sc, int64_t rows, int64_t r, int dtype, const Operand& o, char* ws,
          cudaStream_t s) {
  const dim3 grid((unsigned)((rows + 31) / 32), (unsigned)((r + 31) / 32));
  char* d = ws + o.at;
  const int rp = (int)o.stride;
  if (dtype == NMD_DT_FP32)
    piece_kernel<float, bf16, 3><<<grid, 256, 0, s>>>((const float*)src, sr, sc, rows, (int)r, rp, (bf16*)d,
                                                      (bf16*)(d + o.piece), (bf16*)(d + 2 * o.piece));
  else   // 16-bit values are moved as they are
    piece_kernel<uint16_t, uint16_t, 1><<<grid, 256, 0, s>>>((const uint16_t*)src, sr, sc, rows, (int)r, rp,
                                                             (uint16_t*)d, nullptr, nullptr);
}

}  // namespace
}  // namespace nmd

using namespace nmd;

extern "C" {

nmd_status nmd_factor_workspace_bytes(const void* d_A, int64_t a_row, int64_t a_col, const void* d_B, int64_t b_row,
                                      int64_t b_col, int32_t dtype, int64_t T, int64_t n, int64_t r, size_t* bytes) {
  if (bad_sizes(a_row, a_col, b_row, b_col, dtype, T, n, r) || !bytes) return NMD_ERR_INVALID;
  *bytes = layout(d_A, a_row, a_col, d_B, b_row, b_col, dtype, T, n, r).total;
  return NMD_OK;
}

nmd_status nmd_factor_logprobs(const void* d_A, int64_t a_row, int64_t a_col, const void* d_B, int64_t b_row,
                               int64_t b_col, int32_t dtype, int64_t T, int64_t n, int64_t r, const int64_t* d_targets,
                               double temperature, float* d_logps, void* d_workspace, size_t ws_bytes, void* stream) {
  if (bad_sizes(a_row, a_col, b_row, b_col, dtype, T, n, r) || !(temperature > 0.0) || !std::isfinite(temperature))
    return NMD_ERR_INVALID;
  const float c = (float)(1.4426950408889634074 / temperature), it = (float)(1.0 / temperature);
  if (!(c > 0.f) || !std::isfinite(c) || !std::isfinite(it)) return NMD_ERR_INVALID;
  if (T == 0) return NMD_OK;
  const int es = dtype == NMD_DT_FP32 ? 4 : 2;
  if (!d_A || !d_B || !d_targets || !d_logps || (((uintptr_t)d_A | (uintptr_t)d_B) & (uintptr_t)(es - 1)))
    return NMD_ERR_INVALID;
  const Layout L = layout(d_A, a_row, a_col, d_B, b_row, b_col, dtype, T, n, r);
  if (!d_workspace || ws_bytes < L.total || ((uintptr_t)d_workspace & 255u)) return NMD_ERR_WORKSPACE;
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return NMD_ERR_CUDA;
  cudaStream_t s = (cudaStream_t)stream;
  char* ws = (char*)d_workspace;
  if (L.a.packed) pack(d_A, a_row, a_col, T, r, dtype, L.a, ws, s);
  if (L.b.packed) pack(d_B, b_row, b_col, n, r, dtype, L.b, ws, s);
  CUtensorMap ta[3], tb[3];
  const int kind = dtype == NMD_DT_FP16 ? NMD_DT_FP16 : NMD_DT_BF16;
  for (int k = 0; k < L.pieces; ++k) {
    if (!encode(L.a.packed ? ws + L.a.at + k * L.a.piece : d_A, T, r, L.a.stride, kind, &ta[k]) ||
        !encode(L.b.packed ? ws + L.b.at + k * L.b.piece : d_B, n, r, L.b.stride, kind, &tb[k]))
      return NMD_ERR_CUDA;
  }
  Params p{};
  p.T = T;
  p.n = n;
  p.C = L.C;
  p.W = L.tiles * L.C;
  p.r = (int)r;
  p.npan = (int)((r + 63) / 64);
  p.slots = L.slots;
  p.c = c;
  // kind::f16 with fp32 accumulation: A and B both bf16 (format 1) or both f16 (format 0)
  p.idesc = idesc_bf16(BM, BN, false) & (dtype == NMD_DT_FP16 ? ~((1u << 7) | (1u << 10)) : ~0u);
  p.parts = (Stat*)(ws + L.parts);
  p.flags = (int*)(ws + L.flags);
  const int grid = (int)std::min<int64_t>({(int64_t)sms, (int64_t)kMaxCtas, p.W});
  nmd_status st;
  if (L.pieces == 1) st = launch_scores<1, true>(ta, tb, p, grid, s);
  else if (r <= 128) st = launch_scores<3, true>(ta, tb, p, grid, s);
  else st = launch_scores<3, false>(ta, tb, p, grid, s);
  if (st != NMD_OK) return st;
  const unsigned fg = (unsigned)((T + 7) / 8);
  if (dtype == NMD_DT_FP32)
    finish_kernel<<<fg, 256, 0, s>>>((const float*)d_A, a_row, a_col, (const float*)d_B, b_row, b_col, d_targets, it, p,
                                     (int64_t)grid, d_logps);
  else if (dtype == NMD_DT_BF16)
    finish_kernel<<<fg, 256, 0, s>>>((const bf16*)d_A, a_row, a_col, (const bf16*)d_B, b_row, b_col, d_targets, it, p,
                                     (int64_t)grid, d_logps);
  else
    finish_kernel<<<fg, 256, 0, s>>>((const __half*)d_A, a_row, a_col, (const __half*)d_B, b_row, b_col, d_targets, it,
                                     p, (int64_t)grid, d_logps);
  return cudaGetLastError() == cudaSuccess ? NMD_OK : NMD_ERR_CUDA;
}

}  // extern "C"

// Log-probability of one column per row of softmax(A B^T / tau) without the
// T x n matrix of scores:  log p_t = a_t . b_y / tau - log sum_j exp(a_t . b_j / tau).
//
// The scores are formed tile by tile on the tcgen05 tensor cores (128 rows of A
// against chunks of 128 rows of B) in TMEM, and the epilogue warps reduce each
// row of a tile to a running maximum and sum, as the row kernels of the logits
// do.  Nothing of the scores is written.
//
// 16-bit factors are multiplied as they are.  fp32 factors are split into three
// bf16 pieces each (x = hi + lo + lo2 to 2^-24 of x), and the six products of
// pieces above 2^-24 are accumulated in fp32: lo lo, lo2 hi, hi lo2, lo hi and
// hi lo of all columns, and only then hi hi.  The tensor cores round every
// accumulation towards zero by up to a unit of the sum so far, so the five small
// products are taken while that is small (scores of 100 at r = 256 come out
// 1.25e-4 low on average in the order of the columns, 9e-6 in this one).  Past
// one panel of 64 columns the hi pieces are loaded again for it: 2047 rows of
// 20,000 columns at r = 128 take 60.5 us instead of 53.5, at r = 64 35.1 and 34.5.
//
// The tiles x chunks are dealt to one CTA per SM in equal contiguous runs, so
// that any T and n fill the GPU; a run that crosses into the next tile of rows
// writes its (m, S) and starts over, and the second kernel merges a row's
// partial results in the order of the chunks and takes the dot product a_t . b_y
// in fp32 on the CUDA cores.
//
// Bound by the round trip of a TMEM buffer (products, commit, epilogue, release;
// the SFUs work in half of the cycles): 4096 rows of 139,255 columns at r = 64 in
// bf16 take 116 us with the finish, 4.9e12 exponentials/s of the 9.2e12 that the
// SFUs make, 630 TFLOP/s; 2047 rows of 20,000 columns at r = 32 in fp32 27 us with
// packing and finish; 7 rows of 139,255 columns 13 us.  Chunks of 64 columns
// in eight buffers: 168 us, twice the products issued.
//
// Warp roles: warps 0-15 epilogue (four warpgroups taking chunks in turn; thread
// t of each owns TMEM lane t = row t), warp 16 TMA and TMEM allocation, and the
// warps after it issue the MMAs.  Waits are bounded (2 s): a CTA whose wait
// ran out flags its run, and the rows it would have counted become NaN.
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include "nmd_internal.cuh"
#include "softmax_sum.cuh"
#include "tc_pipe.cuh"
#include "tc_ptx.cuh"

namespace nmd {
namespace {

using namespace tc;

constexpr int BM = 128, BN = 128;
constexpr int kGroups = 4;                   // epilogue warpgroups
constexpr int kTmaWarp = 4 * kGroups, kMmaWarp = kTmaWarp + 1;
constexpr int kPanelA = BM * 128, kPanelB = BN * 128;   // bytes of a tile's or chunk's rows x 64 16-bit columns
constexpr int kMaxCtas = 256;
constexpr int kMaxRank = 256;

// PIECES: bf16 pieces of each factor (1: 16-bit factors).  ARES: the tile of A
// stays in shared memory for the whole run; otherwise (fp32 at rank > 128,
// whose tile would take 192 KB) its panels are loaded beside those of B.
template <int PIECES, bool ARES>
struct Cfg {
  static constexpr int A_PANELS = ARES ? (PIECES == 1 ? 4 : 2) : 0;
  static constexpr int A_BYTES = PIECES * A_PANELS * kPanelA;
  static constexpr int STAGE = PIECES * (kPanelB + (ARES ? 0 : kPanelA));   // the chunk's panels first
  // Warps that issue MMAs, chunks in turn, each with a ring of stages of its own.
  // (One issues a chunk of 16-bit factors in about 1100 cycles beside the
  // epilogue's sixteen warps, more than the products take: 4096 rows of 139,255
  // columns 169 us by one warp, 134 us by two at the time.  The 24 MMAs and more of an fp32
  // chunk cover that.)
  static constexpr int ISS = PIECES == 1 ? 2 : 1;
  static constexpr int THREADS = 32 * (kMmaWarp + ISS);
  static constexpr int RST = PIECES == 1 ? 8 / ISS : 2;   // stages of a ring: a power of two
  static constexpr int NST = ISS * RST;
  static constexpr int NB = 512 / BN;       // TMEM buffers
  // Stages that a chunk of `npan` panels passes through: of fp32 factors the hi pieces of
  // all panels but the last come again together, once the small products are there.
  static __device__ __forceinline__ int uses(int npan) { return PIECES > 1 && npan > 1 ? npan + 1 : npan; }
  static constexpr int NBAR = 2 * NST + 2 * NB + 2 + ISS;
  static constexpr size_t SMEM = 1024 + A_BYTES + (size_t)NST * STAGE + NBAR * 8 + 64;
  static_assert(SMEM <= 227 * 1024, "shared memory per block");
  static_assert(SMEM > 114 * 1024, "one CTA (and its 512 TMEM columns) per SM");
};

struct Params {
  int64_t T, n, C, W;        // rows, columns, chunks per tile, tiles x chunks
  int r, npan;               // rank, panels of 64
  int slots;                 // partial results kept per tile (x kGroups)
  Scale c;
  uint32_t idesc;
  Stat* parts;               // [tile][slot][warpgroup][128]
  int* flags;                // 2 per CTA: nmd_status, detail
};

// CTA that works on unit u of W dealt to G CTAs, CTA b taking [b W / G, (b + 1) W / G)
__host__ __device__ __forceinline__ int64_t owner(int64_t u, int64_t W, int64_t G) { return ((u + 1) * G - 1) / W; }

// 32 lanes x 32 columns of TMEM as 16 pairs of columns, waited for
__device__ __forceinline__ void tmem_pairs(uint32_t taddr, pair_t (&x)[16]) {
  asm volatile(
      "{\n\t.reg .b32 t<32>;\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {t0, t1, t2, t3, t4, t5, t6, t7, t8, t9, t10, t11, t12, t13, t14, t15, t16, t17, t18, t19, t20, t21, t22, t23, t24, t25, t26, t27, t28, t29, t30, t31}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;\n\t"
      "mov.b64 %0, {t0, t1};\n\t"
      "mov.b64 %1, {t2, t3};\n\t"
      "mov.b64 %2, {t4, t5};\n\t"
      "mov.b64 %3, {t6, t7};\n\t"
      "mov.b64 %4, {t8, t9};\n\t"
      "mov.b64 %5, {t10, t11};\n\t"
      "mov.b64 %6, {t12, t13};\n\t"
      "mov.b64 %7, {t14, t15};\n\t"
      "mov.b64 %8, {t16, t17};\n\t"
      "mov.b64 %9, {t18, t19};\n\t"
      "mov.b64 %10, {t20, t21};\n\t"
      "mov.b64 %11, {t22, t23};\n\t"
      "mov.b64 %12, {t24, t25};\n\t"
      "mov.b64 %13, {t26, t27};\n\t"
      "mov.b64 %14, {t28, t29};\n\t"
      "mov.b64 %15, {t30, t31};\n\t"
      "}"
      : "=l"(x[0]), "=l"(x[1]), "=l"(x[2]), "=l"(x[3]), "=l"(x[4]), "=l"(x[5]), "=l"(x[6]), "=l"(x[7]), "=l"(x[8]), "=l"(x[9]), "=l"(x[10]), "=l"(x[11]), "=l"(x[12]), "=l"(x[13]), "=l"(x[14]), "=l"(x[15])
      : "r"(taddr)
      : "memory");
}

// A row's running pair over its scores.
struct RowSum : RunningSum {
  float lost = 0.f;   // what the additions to S have rounded away: a row may have very many groups
  __device__ __forceinline__ void put(float group) {
    const float y = group - lost, sum = s.S + y;
    lost = (sum - s.S) - y;
    s.S = sum;
  }
  // `blocks` (at most four) times 32 scores; get(b, x) gives them as pairs, again
  // where they are not usual ones.  One vote and one compensated addition for all
  // (one for each 32 scores: 134 us instead of 119 for 4096 rows of 139,255
  // columns); the loops are rolled, or the code of seven rows would take longer
  // to arrive (16 us instead of 13) than it saves the 4096 (1.5 us).
  template <class G>
  __device__ __forceinline__ void add(int blocks, G get, Scale c) {
    pair_t x[16];
    if (__all_sync(0xffffffffu, usual)) {   // (TMEM is read by whole warps)
      float group = 0.f;
#pragma unroll 1
      for (int b = 0; b < blocks; ++b) {
        get(b, x);
        group += group_sum(x, c);
      }
      const bool fine = group < kHigh;
      if (fine) put(group);
      if (__all_sync(0xffffffffu, fine)) return;
#pragma unroll 1
      for (int b = 0; b < blocks; ++b) {
        get(b, x);
        if (!fine) slow(x, c);
      }
    } else {
#pragma unroll 1
      for (int b = 0; b < blocks; ++b) {
        get(b, x);
        slow(x, c);
      }
    }
  }

 private:
  // the first group, one with larger values, or one with NaN or infinities
  __device__ __forceinline__ void slow(const pair_t (&x)[16], Scale c) {
    float m = s.m;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float2 v = halves(x[i]);
      m = max_nan(m, max_nan(v.x, v.y));
    }
    if (m != s.m) lost = 0.f;
    raise(m, c);
    // against the reference where it is an integer, against m itself otherwise
    // (only -inf so far: the sum is 0 and stays 0)
    const float z = s.m == -INFINITY ? 0.f : s.m;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float2 e = halves(power2(x[i], z, c));
      sum += e.x + e.y;
    }
    put(sum * ex2(-above(s.m, c)));
  }
};

template <int PIECES, bool ARES>
__global__ void __launch_bounds__((Cfg<PIECES, ARES>::THREADS), 1)
    score_kernel(const __grid_constant__ CUtensorMap ta0, const __grid_constant__ CUtensorMap ta1,
                 const __grid_constant__ CUtensorMap ta2, const __grid_constant__ CUtensorMap tb0,
                 const __grid_constant__ CUtensorMap tb1, const __grid_constant__ CUtensorMap tb2, const Params p) {
  using C = Cfg<PIECES, ARES>;
  constexpr int NST = C::NST, RST = C::RST, NB = C::NB;
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
  asm volatile("griddepcontrol.launch_dependents;");
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
    mbar_init(b_aempty, C::ISS);
    for (int i = 0; i < C::ISS; ++i) mbar_init(b_drain + 8 * i, 1);
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
  const int uses = C::uses(p.npan);

  if (warp == kTmaWarp) {
    if (lane == 0) {
      uint32_t aph = 1;
      int64_t aloads = 0, done = 0;   // tiles of A, chunks asked for
      bool ok = true;
      int64_t tile = tile0, c = u0 - tile0 * p.C;
      bool first = true;
      for (int64_t u = u0; u < u1 && ok; ++u) {
        if (ARES && first) {
          if (!(ok = wait_bar(b_aempty, aph, abort_flag, status, 10))) break;
          aph ^= 1u;
          mbar_expect_tx(b_afull, PIECES * p.npan * kPanelA);
          for (int k = 0; k < p.npan; ++k) {
            const uint32_t dst = a_sm + k * PIECES * kPanelA;
            tma_load_2d(dst, &ta0, b_afull, 64 * k, (int)(tile * BM));
            if (PIECES > 1) tma_load_2d(dst + kPanelA, &ta1, b_afull, 64 * k, (int)(tile * BM));
            if (PIECES > 1) tma_load_2d(dst + 2 * kPanelA, &ta2, b_afull, 64 * k, (int)(tile * BM));
          }
          ++aloads;
          first = false;
        }
        const uint32_t G = (uint32_t)(u - u0), use = G / C::ISS * uses;
        for (int k = 0; k < uses; ++k) {
          const int s = (int)(G % C::ISS) * RST + (int)((use + k) % RST);
          if (!(ok = wait_bar(b_empty + 8 * s, (((use + k) / RST) & 1u) ^ 1u, abort_flag, status, 1))) break;
          const uint32_t dst = st_sm + s * C::STAGE, da = dst + PIECES * kPanelB, bar = b_full + 8 * s;
          if (PIECES > 1 && k == p.npan) {
            mbar_expect_tx(bar, (p.npan - 1) * (kPanelB + (ARES ? 0 : kPanelA)));
            for (int h = 0; h < p.npan - 1; ++h) {
              tma_load_2d(dst + h * kPanelB, &tb0, bar, 64 * h, (int)(c * BN));
              if (!ARES) tma_load_2d(da + h * kPanelA, &ta0, bar, 64 * h, (int)(tile * BM));
            }
            break;
          }
          mbar_expect_tx(bar, C::STAGE);
          tma_load_2d(dst, &tb0, bar, 64 * k, (int)(c * BN));
          if (PIECES > 1) tma_load_2d(dst + kPanelB, &tb1, bar, 64 * k, (int)(c * BN));
          if (PIECES > 1) tma_load_2d(dst + 2 * kPanelB, &tb2, bar, 64 * k, (int)(c * BN));
          if (!ARES) {
            tma_load_2d(da, &ta0, bar, 64 * k, (int)(tile * BM));
            if (PIECES > 1) tma_load_2d(da + kPanelA, &ta1, bar, 64 * k, (int)(tile * BM));
            if (PIECES > 1) tma_load_2d(da + 2 * kPanelA, &ta2, bar, 64 * k, (int)(tile * BM));
          }
        }
        ++done;
        if (++c == p.C) {
          c = 0;
          ++tile;
          first = true;
        }
      }
      if (!ok) {   // wait for the copies in flight before shared memory goes away
        for (int i = 0; i < NST; ++i) {   // (a stage that never gets its phase is given up after 0.1 s)
          const uint32_t ring = (uint32_t)(i / RST), chunks = (uint32_t)((done + C::ISS - 1 - ring) / C::ISS);
          const uint32_t total = chunks * uses;   // of this ring; the last use of its stage i % RST:
          if (total <= (uint32_t)(i % RST)) continue;
          const uint32_t last = (total - 1 - i % RST) / RST;
          const uint64_t t0 = globaltimer_ns();
          while (!mbar_try_wait(b_full + 8 * i, last & 1u) && globaltimer_ns() - t0 < 100000000ull) {
          }
        }
        if (aloads > 0) {
          const uint64_t t0 = globaltimer_ns();
          while (!mbar_try_wait(b_afull, (uint32_t)((aloads - 1) & 1)) && globaltimer_ns() - t0 < 100000000ull) {
          }
        }
      }
    }
  } else if (warp >= kMmaWarp) {
    const uint32_t me = warp - kMmaWarp;
    uint32_t aph = 0;
    bool ok = true;
    int64_t c0 = u0 - tile0 * p.C;
    for (int64_t u = u0; u < u1 && ok; c0 = 0) {   // the chunks of one tile of A after those of the other
      const uint32_t G0 = (uint32_t)(u - u0), seg = (uint32_t)min(p.C - c0, u1 - u);
      // by every issuer, so that none falls a phase behind
      if (ARES && !(ok = conv_wait(b_afull, aph, abort_flag, status, 2))) break;
      for (uint32_t i = (me - G0) % C::ISS; i < seg && ok; i += C::ISS) {
        const uint32_t G = G0 + i, lb = G % NB, use = G / C::ISS * uses;
        if (!(ok = conv_wait(b_lfree + 8 * lb, ((G / NB) & 1u) ^ 1u, abort_flag, status, 4))) break;
        const uint32_t d = tmem + lb * BN;
        for (int k = 0; k < uses; ++k) {
          const uint32_t s = me * RST + (use + k) % RST;
          if (!(ok = conv_wait(b_full + 8 * s, ((use + k) / RST) & 1u, abort_flag, status, 3))) break;
          fence_after();
          const uint32_t bs = st_sm + s * C::STAGE, as = bs + PIECES * kPanelB;
          const bool again = PIECES > 1 && k == p.npan;   // the hi pieces of the panels before the last
          if (!again) {
            const uint64_t db = sdesc(bs, 16, 1024, SWZ_128B);
            const uint64_t da = sdesc(ARES ? a_sm + k * PIECES * kPanelA : as, 16, 1024, SWZ_128B);
            const int steps = min(4, (p.r - 64 * k + 15) / 16);
            if (PIECES > 1) {
              constexpr uint64_t A = kPanelA >> 4, B = kPanelB >> 4;
              for (int q = 0; q < steps; ++q) {
                mma_ss_elect(d, da + 2 * q + A, db + 2 * q + B, p.idesc, (k | q) != 0);   // lo lo
                mma_ss_elect(d, da + 2 * q + 2 * A, db + 2 * q, p.idesc, 1);              // lo2 hi
                mma_ss_elect(d, da + 2 * q, db + 2 * q + 2 * B, p.idesc, 1);              // hi lo2
                mma_ss_elect(d, da + 2 * q + A, db + 2 * q, p.idesc, 1);                  // lo hi
                mma_ss_elect(d, da + 2 * q, db + 2 * q + B, p.idesc, 1);                  // hi lo
              }
            }
            if (PIECES == 1 || k == p.npan - 1)
              for (int q = 0; q < steps; ++q) mma_ss_elect(d, da + 2 * q, db + 2 * q, p.idesc, PIECES > 1 || (k | q) != 0);
          } else {
            for (int h = 0; h < p.npan - 1; ++h) {
              const uint64_t db = sdesc(bs + h * kPanelB, 16, 1024, SWZ_128B);
              const uint64_t da = sdesc(ARES ? a_sm + h * PIECES * kPanelA : as + h * kPanelA, 16, 1024, SWZ_128B);
              for (int q = 0; q < 4; ++q) mma_ss_elect(d, da + 2 * q, db + 2 * q, p.idesc, 1);
            }
          }
          commit_elect(b_empty + 8 * s);
        }
        if (!ok) break;
        commit_elect(b_lfull + 8 * lb);
      }
      if (c0 + seg == p.C) {   // done with this tile of A
        if (ARES) commit_elect(b_aempty);
        aph ^= 1u;
      }
      u += seg;
    }
    commit_elect(b_drain + 8 * me);   // every MMA issued has to be over before TMEM is freed
    if (lane == 0) {
      const uint64_t t0 = globaltimer_ns();
      while (!mbar_try_wait(b_drain + 8 * me, 0) && globaltimer_ns() - t0 < 200000000ull) {
      }
    }
    __syncwarp();
  } else {
    const int wg = warp >> 2, quarter = warp & 3;
    const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
    const Scale cc = p.c;
    RowSum run;
    // a warpgroup has a TMEM buffer of its own, so that it sees every phase of its barrier
    static_assert(NB == kGroups, "one TMEM buffer per epilogue warpgroup");
    const uint32_t col = tmem + lane_base + wg * BN;
    bool ok = true;
    int64_t tile = tile0, c0 = u0 - tile0 * p.C;
    for (int64_t u = u0; u < u1; ++tile, c0 = 0) {
      const uint32_t G0 = (uint32_t)(u - u0), seg = (uint32_t)min(p.C - c0, u1 - u);
      const bool some = tile * BM + quarter * 32 < p.T;   // some row of this warp exists
      for (uint32_t i = (wg - G0) % kGroups; i < seg; i += kGroups) {
        if (!(ok = conv_wait(b_lfull + 8 * wg, ((G0 + i) / NB) & 1u, abort_flag, status, 7))) break;
        fence_after();
        if (some) {
          const int kv = (int)min((int64_t)BN, p.n - (c0 + i) * BN);
          if (kv == BN) {
            run.add(BN / 32, [&](int b, pair_t(&x)[16]) { tmem_pairs(col + 32 * b, x); }, cc);
          } else {   // columns past the last count as -inf
            run.add(
                (kv + 31) / 32,
                [&](int b, pair_t(&x)[16]) {
                  tmem_pairs(col + 32 * b, x);
#pragma unroll
                  for (int i = 0; i < 16; ++i) {
                    const int k = 32 * b + 2 * i;
                    const float2 v = halves(x[i]);
                    x[i] = pair_of(k < kv ? v.x : -INFINITY, k + 1 < kv ? v.y : -INFINITY);
                  }
                },
                cc);
          }
        }
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(b_lfree + 8 * wg);
      }
      if (!ok) break;
      // the end of a tile, or of the run: hand over the row's partial result
      const int64_t slot = blockIdx.x - owner(tile * p.C, p.W, gridDim.x);
      p.parts[((tile * p.slots + slot) * kGroups + wg) * BM + quarter * 32 + lane] = run.s;
      run = RowSum();
      u += seg;
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

// A row's partial results merged, the target's score, the difference: by one
// warp, or by a CTA where few tiles spread over many CTAs leave many of them.
template <class T, bool CTA>
__global__ void __launch_bounds__(256)
    finish_kernel(const T* A, int64_t ar, int64_t ac, const T* B, int64_t br, int64_t bc, const int64_t* y,
                  float2 inv_temp, const Params p, int64_t G, float* logps) {
  __shared__ Stat red[8];
  __shared__ int bad_any;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t t = CTA ? blockIdx.x : (int64_t)blockIdx.x * 8 + warp;
  if (t >= p.T) return;
  if (CTA && threadIdx.x == 0) bad_any = 0;
  const int64_t yt = y[t];
  float z = 0.f;
  if (yt >= 0 && yt < p.n && (!CTA || warp == 0)) {   // before the scores are there
    for (int k = lane; k < p.r; k += 32) z = fmaf(value(A[t * ar + k * ac]), value(B[yt * br + k * bc]), z);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (yt < 0 || yt >= p.n) {
    if (CTA ? threadIdx.x == 0 : lane == 0) logps[t] = yt < 0 ? 0.f : NAN;
    return;
  }
  const int64_t tile = t / BM, b0 = owner(tile * p.C, p.W, G), b1 = owner(tile * p.C + p.C - 1, p.W, G);
  const int count = (int)(kGroups * (b1 - b0 + 1)), first = CTA ? threadIdx.x : lane, step = CTA ? 256 : 32;
  const Stat* parts = p.parts + tile * p.slots * kGroups * BM + t % BM;
  float m = -INFINITY;
  int bad = 0;
#pragma unroll 4
  for (int k = first; k < count; k += step) {
    m = max_nan(m, parts[(int64_t)k * BM].m);
    bad |= p.flags[2 * (b0 + k / kGroups)];
  }
  Stat st{m, 0.f};
#pragma unroll 4
  for (int k = first; k < count; k += step) {
    const Stat o = parts[(int64_t)k * BM];
    st.S += o.S * rescale(o.m, m, p.c);
  }
  st = merge_lanes<32>(st, p.c);
  bad = __any_sync(0xffffffffu, bad);
  if (CTA) {
    __syncthreads();
    if (lane == 0) {
      red[warp] = st;
      if (bad) bad_any = 1;
    }
    __syncthreads();
    st = merge_lanes<8>(lane < 8 ? red[lane] : Stat{-INFINITY, 0.f}, p.c);
    bad = bad_any;
  }
  if (CTA ? threadIdx.x == 0 : lane == 0)
    logps[t] = bad || st.m == INFINITY ? NAN : log_prob(z, st, above(st.m, p.c), inv_temp).value();
}

// A factor of any strides and the row-major 16-bit pieces that it is packed
// into, with row stride rp (a multiple of 8 elements, as TMA asks).
template <class T, class D>
struct PackJob {
  const T* src;
  int64_t sr, sc, rows;
  int rp;
  D* d[3];
  int64_t blocks;   // of 32 rows; 0: this factor is read where it is
};

// Both factors in one launch, through tiles of 32 x 32 so that both sides are
// read and written along their rows.
template <class T, class D, int PIECES>
__global__ void __launch_bounds__(256) piece_kernel(const PackJob<T, D> ja, const PackJob<T, D> jb, int r) {
  __shared__ T tile[32][33];
  const bool first = blockIdx.x < ja.blocks;
  const PackJob<T, D>& j = first ? ja : jb;
  const int64_t row0 = ((int64_t)blockIdx.x - (first ? 0 : ja.blocks)) * 32;
  const int col0 = blockIdx.y * 32;
  const int a = threadIdx.x & 31, b = threadIdx.x >> 5;
  for (int i = b; i < 32; i += 8) {   // lanes along the dimension whose stride is the smaller
    const int64_t row = row0 + (j.sc <= j.sr ? i : a);
    const int col = col0 + (j.sc <= j.sr ? a : i);
    if (row < j.rows && col < r) tile[row - row0][col - col0] = j.src[row * j.sr + col * j.sc];
  }
  __syncthreads();
  for (int i = b; i < 32; i += 8) {
    const int64_t row = row0 + i, at = row * j.rp + col0 + a;
    if (row >= j.rows || col0 + a >= r) continue;
    if constexpr (PIECES == 1) {
      j.d[0][at] = tile[i][a];
    } else {
      const float x = tile[i][a];
      const bf16 h = __float2bfloat16_rn(x);
      const float e = x - __bfloat162float(h);
      const bf16 l = __float2bfloat16_rn(e);
      j.d[0][at] = h;
      j.d[1][at] = l;
      j.d[2][at] = __float2bfloat16_rn(e - __bfloat162float(l));
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
  off += ((size_t)L.tiles * L.slots * kGroups * BM * sizeof(Stat) + 255) & ~size_t(255);
  L.flags = off;
  off += kMaxCtas * 2 * sizeof(int);
  L.total = off;
  return L;
}

bool bad_sizes(int64_t ar, int64_t ac, int64_t br, int64_t bc, int dtype, int64_t T, int64_t n, int64_t r) {
  return dtype < NMD_DT_FP32 || dtype > NMD_DT_FP16 || T < 0 || T > (int64_t(1) << 27) || n < 1 ||
         n >= (int64_t(1) << 31) || r < 1 || r > kMaxRank || ar < 0 || ac < 0 || br < 0 || bc < 0;
}

bool encode(const void* base, int64_t rows, int64_t r, int64_t stride, int dtype, int box_rows, CUtensorMap* m) {
  PFN_cuTensorMapEncodeTiled_v12000 fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {(cuuint64_t)r, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)stride * 2};
  cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, es[2] = {1, 1};
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
  score_kernel<PIECES, ARES><<<grid, C::THREADS, C::SMEM, s>>>(ta[0], ta[k1], ta[k2], tb[0], tb[k1], tb[k2], p);
  return cudaGetLastError() == cudaSuccess ? NMD_OK : NMD_ERR_CUDA;
}

// `overlap`: the kernel may start before the one ahead of it in the stream has
// finished (it waits for that one itself).
template <class... P, class... A>
cudaError_t launch(void (*kernel)(P...), int64_t grid, int block, size_t smem, bool overlap, cudaStream_t s,
                   const A&... args) {
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3((unsigned)block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = &attr;
  cfg.numAttrs = overlap ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <class T>
cudaError_t launch_finish(const void* const* f, const int64_t* st, const int64_t* y, float2 it, const Params& p,
                          int64_t grid, int64_t tiles, float* logps, cudaStream_t s) {
  // a CTA per row where a tile's partial results come from 32 CTAs or more
  if (tiles * 32 <= grid)
    return launch(finish_kernel<T, true>, p.T, 256, 0, true, s, (const T*)f[0], st[0], st[1], (const T*)f[1], st[2],
                  st[3], y, it, p, grid, logps);
  return launch(finish_kernel<T, false>, (p.T + 7) / 8, 256, 0, true, s, (const T*)f[0], st[0], st[1], (const T*)f[1],
                st[2], st[3], y, it, p, grid, logps);
}

template <class T, class D, int PIECES>
void pack(const void* A, const int64_t* sa, int64_t T_, const void* B, const int64_t* sb, int64_t n, int64_t r,
          const Layout& L, char* ws, cudaStream_t s) {
  auto job = [&](const void* src, const int64_t* st, int64_t rows, const Operand& o) {
    D* d = (D*)(ws + o.at);
    const size_t piece = o.piece / sizeof(D);
    return PackJob<T, D>{(const T*)src, st[0], st[1], rows, (int)o.stride, {d, d + piece, d + 2 * piece},
                         o.packed ? (rows + 31) / 32 : 0};
  };
  const PackJob<T, D> ja = job(A, sa, T_, L.a), jb = job(B, sb, n, L.b);
  const int64_t blocks = ja.blocks + jb.blocks;
  if (blocks > 0)
    piece_kernel<T, D, PIECES><<<dim3((unsigned)blocks, (unsigned)((r + 31) / 32)), 256, 0, s>>>(ja, jb, (int)r);
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
  Params p{};
  if (bad_sizes(a_row, a_col, b_row, b_col, dtype, T, n, r) || !scale_of(temperature, &p.c)) return NMD_ERR_INVALID;
  const float2 it = two_floats(1.0 / temperature);
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
  const int64_t sa[2] = {a_row, a_col}, sb[2] = {b_row, b_col};
  if (dtype == NMD_DT_FP32) pack<float, bf16, 3>(d_A, sa, T, d_B, sb, n, r, L, ws, s);
  else pack<uint16_t, uint16_t, 1>(d_A, sa, T, d_B, sb, n, r, L, ws, s);   // 16-bit values are moved as they are
  CUtensorMap ta[3], tb[3];
  const int kind = dtype == NMD_DT_FP16 ? NMD_DT_FP16 : NMD_DT_BF16;
  for (int k = 0; k < L.pieces; ++k) {
    if (!encode(L.a.packed ? ws + L.a.at + k * L.a.piece : d_A, T, r, L.a.stride, kind, BM, &ta[k]) ||
        !encode(L.b.packed ? ws + L.b.at + k * L.b.piece : d_B, n, r, L.b.stride, kind, BN, &tb[k]))
      return NMD_ERR_CUDA;
  }
  p.T = T;
  p.n = n;
  p.C = L.C;
  p.W = L.tiles * L.C;
  p.r = (int)r;
  p.npan = (int)((r + 63) / 64);
  p.slots = L.slots;
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
  const void* f[2] = {d_A, d_B};
  const int64_t strides[4] = {a_row, a_col, b_row, b_col};
  cudaError_t e;
  if (dtype == NMD_DT_FP32) e = launch_finish<float>(f, strides, d_targets, it, p, grid, L.tiles, d_logps, s);
  else if (dtype == NMD_DT_BF16) e = launch_finish<bf16>(f, strides, d_targets, it, p, grid, L.tiles, d_logps, s);
  else e = launch_finish<__half>(f, strides, d_targets, it, p, grid, L.tiles, d_logps, s);
  return e == cudaSuccess ? NMD_OK : NMD_ERR_CUDA;
}

}  // extern "C"

// All Newton-Schulz steps of an update with a short side of at most 64 in one kernel
// (mathematics, pieces and scales: muon.cu).
//
// X is M x 64, M the long side, in tiles of 128 rows; a CTA per SM holds its tiles on
// chip from the first step to the last: up to six in shared memory, or five there and up
// to three in TMEM, which pass through the sixth buffer on their way into Z.  A step is
// one pass over them,
//   X <- X P  (128 x 64 by 64 x 64),  Z += X^T X,
// and between passes the CTAs' sums Z are added up and every CTA forms
//   A = Z,  P = a I + b A + c A A
// for itself.  So nothing of X moves between steps, and a step costs two barriers of the
// grid (one among up to eight CTAs) instead of four launches.  139,255 x 64 in fp32 takes
// 85 us of the call's 115 (the rest is the norm and the pieces): a step 15 us, of which
// the pass over eight tiles is 6, the two barriers 4, A and P 2.  64 x 64 takes 26 us, a
// chain of latencies; a 32 x 20,000 step 62 us.  (As separate launches: 263, 92 and 164
// us a call; tiles that did not fit passed through global memory: 175 us instead of 85;
// 129 x 64 with the second barrier and each sum by one CTA at a time: 142 us, now 42.)
//
// Pieces are put side by side, so that one product of the tensor cores takes two:
//   X P:    columns [hi P_hi | hi P_lo + lo P_hi],  128 x 128;
//   X^T X:  rows [hi^T hi; lo^T hi], 128 x 64.  With Z = hi^T hi / 2 + lo^T hi the Gram
//           matrix is Z + Z^T, which is as symmetric in its bits as in the formula;
//   A A:    likewise.
// The small products have accumulators of their own, and Z leaves TMEM after every tile.
//
// Where the grid cannot run all at a time the launch is refused, and muon.cu's products
// take its place.
//
// A tile is stored as rows of 64 columns, 128 bytes in the 128-byte swizzle, hi and lo
// one after the other: K-major for X P, MN-major for X^T X.
#include <algorithm>

#include "muon.cuh"

namespace nmd {
namespace muon {
namespace {

using namespace tc;

constexpr int kThreads = 256, kSms = 152;                  // threads that work; one warp more issues the products
constexpr int kRows = 128, kSide = 64;
// CTAs that add up each other's Z without a second barrier (M x 64, five steps, one barrier
// and two: 2 CTAs 43 and 64 us, 4 46 and 64, 8 57 and 72, 12 62 and 78, 16 69 and 56, 24 81
// and 66; 9 to 15 share the elements unevenly and would gain from one)
constexpr int kFew = 8;
constexpr int kBuffers = 6;                                 // tiles in shared memory
constexpr int kPiece = kRows * kSide * 2, kTile = 2 * kPiece;   // bytes
constexpr int kSquare = 2 * kSide * kSide * 2;              // both pieces of a 64 x 64 matrix
// Z in shared memory: two halves of 32 columns, so placed that eight rows by columns 16
// apart, and the same transposed, lie in 32 banks
constexpr int kZ = 4248;
__device__ __forceinline__ int z_at(int i, int j) { return (j >> 5) * 2120 + i * 33 + (i >> 5) * 8 + (j & 31); }
constexpr size_t kOffP = (size_t)kBuffers * kTile, kOffZ = kOffP + kSquare,
                 kOffBars = kOffZ + (kZ * 4 + 255) / 256 * 256;
constexpr size_t kSmem = 1024 + kOffBars + 128;
static_assert(kSmem <= 227 * 1024 && kSms % 8 == 0, "shared memory");
// TMEM: two X P, Z, tiles (32 columns of hi, 32 of lo each)
constexpr uint32_t kColD = 0, kColZ = 256, kColX = 320, kTmem = 512;

struct Strip {
  Job j;
  Pieces x;            // X to start with
  int64_t M;
  int turned;          // the result's columns are X's rows
  int tiles, steps;
  float a, b, c;
  int* ints;
  float* part;         // the CTAs' Z, 64 x 64 each, of two steps
  float* sum;          // 64 x 64
};

// the 16-byte vector q (0 .. 7) of row m in a tile's piece
__device__ __forceinline__ uint32_t vector_at(int m, int q) { return (uint32_t)(m * 128 + ((q ^ (m & 7)) << 4)); }

__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// the working threads
__device__ __forceinline__ void sync_workers() { named_bar_sync(1, kThreads); }

// All CTAs' writes before are seen by all after.  `target`: arrivals of all barriers up to
// this one; the CTA that comes last raises the flag that the others look at, apart from
// the count.  A wait that runs out (2 s) raises the abort flag; the CTA then goes on
// without waiting.  Its status is there before what it adds up is: the result of every CTA
// that took part in sums from then on is NaN.
__device__ __forceinline__ void grid_barrier(int* ints, int target, volatile int* abort_flag, int* status) {
  sync_workers();
  if (threadIdx.x == 0) {
    int n;
    if (*abort_flag) record(status, NMD_ERR_TIMEOUT, 10);
    asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(n) : "l"(ints + kBarrier) : "memory");
    if (n + 1 == target) {
      asm volatile("st.release.gpu.global.s32 [%0], %1;" ::"l"(ints + kFlag), "r"(target) : "memory");
    } else {
      const uint64_t t0 = globaltimer_ns();
      for (;;) {
        asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(n) : "l"(ints + kFlag) : "memory");
        if (n >= target || *abort_flag) break;
        if (globaltimer_ns() - t0 > kTimeoutNs) {
          *abort_flag = 1;
          record(status, NMD_ERR_TIMEOUT, 10);
        }
      }
    }
  }
  sync_workers();
}

// fp32 rows of a tile in shared memory: groups of four columns, group g of row m where
// rows by eight lanes and groups by sixteen lie in different banks
__device__ __forceinline__ int group_at(int m, int g) { return m * kSide + ((g ^ (m & 15)) << 2); }

template <class T>
struct __align__(4 * sizeof(T)) Four {
  T x[4];
};
// A tile of the result.  Rows of the result that are X's rows: a thread takes four
// columns of every sixteenth row, in one store where the result's rows allow it.
// Rows that are X's columns: one row of X, adjacent to its neighbours' everywhere.
template <class T>
__device__ __forceinline__ void put_tile(const Strip& p, const float* stage, int64_t m0, float fill) {
  const int r = (int)p.x.cols, rows = (int)min((int64_t)kRows, p.M - m0), tid = threadIdx.x;
  auto mix = [&](float x, T w) { return p.j.step ? fmaf(-p.j.lr, x, p.j.keep * as_float(w)) : x; };
  if (!p.turned) {
    const int j = (tid & 15) * 4, first = tid >> 4;
    const int64_t rs = p.j.out.rs, cs = p.j.out.cs;
    T* at = &p.j.out.at<T>(m0 + first, j);
    const bool whole = cs == 1 && j + 4 <= r && (((uintptr_t)at | (uintptr_t)(rs * sizeof(T))) & (4 * sizeof(T) - 1)) == 0;
    if (whole) {
#pragma unroll 1
      for (int m = first; m < rows; m += 32, at += 32 * rs) {   // two at a time
        Four<T> w[2];
        const bool second = m + 16 < rows;
        if (p.j.step) {
          w[0] = *(const Four<T>*)at;
          if (second) w[1] = *(const Four<T>*)(at + 16 * rs);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          if (k == 1 && !second) break;
          const float4 x = *(const float4*)(stage + group_at(m + 16 * k, tid & 15));
          from_float(mix(x.x + fill, w[k].x[0]), &w[k].x[0]);
          from_float(mix(x.y + fill, w[k].x[1]), &w[k].x[1]);
          from_float(mix(x.z + fill, w[k].x[2]), &w[k].x[2]);
          from_float(mix(x.w + fill, w[k].x[3]), &w[k].x[3]);
          *(Four<T>*)(at + 16 * k * rs) = w[k];
        }
      }
      return;
    }
#pragma unroll 1
    for (int m = first; m < rows; m += 16, at += 16 * rs) {
      const float4 x = *(const float4*)(stage + group_at(m, tid & 15));
      T w[4];
      if (p.j.step) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (j + e < r) w[e] = at[e * cs];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (j + e < r) from_float(mix((e == 0 ? x.x : e == 1 ? x.y : e == 2 ? x.z : x.w) + fill, w[e]), at + e * cs);
    }
    return;
  }
  const int m = tid & (kRows - 1), j0 = tid / kRows;
  if (m >= rows) return;
  const int64_t rs = p.j.out.rs;
  T* at = &p.j.out.at<T>(j0, m0 + m);
#pragma unroll 1
  for (int j = j0; j < r; j += 8, at += 8 * rs) {   // every second row, four at a time
    T w[4];
    if (p.j.step) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (j + 2 * k < r) w[k] = at[2 * k * rs];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (j + 2 * k < r) from_float(mix(stage[group_at(m, (j + 2 * k) >> 2) + ((j + 2 * k) & 3)] + fill, w[k]), at + 2 * k * rs);
  }
}

__global__ void __launch_bounds__(kThreads + 32, 1) strip_kernel(const __grid_constant__ CUtensorMap tx, const __grid_constant__ Strip p) {
  extern __shared__ char smem_raw[];
  char* smem = (char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  float* Z = (float*)(smem + kOffZ);
  const uint32_t base = smem_u32(smem), sP = base + kOffP, bars = base + kOffBars;
  const uint32_t b_full = bars, b_xp = bars + 8 * kBuffers, b_z = b_xp + 16, b_done = b_z + 8, b_drain = b_done + 16;
  uint32_t* slot = (uint32_t*)(smem + kOffBars + 8 * (kBuffers + 6));
  volatile int* abort_flag = (volatile int*)(slot + 1);
  volatile int* others = (volatile int*)(slot + 2);   // another CTA's wait ran out
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int quad = warp & 3, half = warp >> 2;     // TMEM lanes and columns of this warp
  const int row = quad * 32 + lane;                // of a tile, or of [hi; lo]
  const uint32_t lanes = (uint32_t)(quad * 32) << 16;
  int* status = p.ints;
  const int* shift = p.ints + kShift;
  const int G = gridDim.x, T = (p.tiles - (int)blockIdx.x + G - 1) / G;
  auto tile_row = [&](int t) { return ((int64_t)blockIdx.x + (int64_t)t * G) * kRows; };
  // Of more than six tiles the second, fourth and sixth lie in TMEM, so that one in shared
  // memory comes between two that need the sixth buffer.
  const int away = max(0, T - kBuffers + (T > kBuffers ? 1 : 0));
  auto place_of = [&](int t) { return (t & 1) && t / 2 < away ? t / 2 : -1; };   // in TMEM
  auto buffer_of = [&](int t) { return place_of(t) >= 0 ? kBuffers - 1 : t - min(t / 2 + (t & 1), away); };

  if (tid == 0) {
    prefetch_tmap(&tx);
    for (int i = 0; i < kBuffers + 3; ++i) mbar_init(bars + 8 * i, 1);
    for (int i = 0; i < 2; ++i) mbar_init(b_done + 8 * i, kThreads / 32);
    mbar_init(b_drain, 1);
    fence_mbar_init();
    *abort_flag = 0;
    *others = 0;
  }
  if (warp == 0) {
    tmem_alloc(smem_u32(slot), kTmem);
    tmem_relinquish();
  }
  after_previous();
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = *(volatile uint32_t*)slot;

  uint32_t ph_full = 0, ph_xp = 0, ph_z = 0, turn = 0;   // parities of the next waits
  auto wait = [&](uint32_t bar, uint32_t& ph, int i, int where) {
    wait_bar(bar + 8 * i, ph >> i & 1u, abort_flag, status, where);
    ph ^= 1u << i;
  };
  // the rest of this block by the converged issuing warp: what is uniform stays in uniform registers
  auto load = [&](int t) {
    if (lane != 0) return;
    const int b = buffer_of(t);
    mbar_expect_tx(b_full + 8 * b, kTile);
    tma_load_3d(base + b * kTile, &tx, b_full + 8 * b, 0, (int)tile_row(t), 0);
  };
  // X P of a tile
  auto issue_xp = [&](int t) {
    constexpr uint32_t wide = idesc_fp16(128, 128, false, false), narrow = idesc_fp16(128, 64, false, false);
    const uint64_t P = sdesc(sP, 16, 1024, SWZ_128B);
    const uint32_t d = tmem + kColD + (t & 1) * 128;
    fence_after();
    if (place_of(t) >= 0) {
      const uint32_t x = tmem + kColX + place_of(t) * 64;
#pragma unroll
      for (int q = 0; q < kSide / 16; ++q) mma_ts_elect(d, x + q * 8, P + (q * 32 >> 4), wide, q > 0);
#pragma unroll
      for (int q = 0; q < kSide / 16; ++q) mma_ts_elect(d + 64, x + 32 + q * 8, P + (q * 32 >> 4), narrow, 1);
    } else {
      const uint64_t x = sdesc(base + buffer_of(t) * kTile, 16, 1024, SWZ_128B);
#pragma unroll
      for (int q = 0; q < kSide / 16; ++q) mma_ss_elect(d, x + (q * 32 >> 4), P + (q * 32 >> 4), wide, q > 0);
#pragma unroll
      for (int q = 0; q < kSide / 16; ++q) mma_ss_elect(d + 64, x + ((kPiece + q * 32) >> 4), P + (q * 32 >> 4), narrow, 1);
    }
    commit_elect(b_xp + 8 * (t & 1));
  };
  // X^T X of a tile
  auto issue_z = [&](int t) {
    constexpr uint32_t idesc = idesc_fp16(128, 64, true, true);
    const uint64_t x = sdesc(base + buffer_of(t) * kTile, kPiece, 1024, SWZ_128B);
    fence_after();
#pragma unroll
    for (int q = 0; q < kRows / 16; ++q) mma_ss_elect(tmem + kColZ, x + (q * 16 * 128 >> 4), x + (q * 16 * 128 >> 4), idesc, q > 0);
    commit_elect(b_z);
  };
  if (warp == kThreads / 32) {
    // ---- loads and products.  The workers say after each of their pieces of work that they
    // have done with it, on two barriers in turn: the next but one needs something that is
    // issued after this one.
    uint32_t n = 0;
    auto done = [&] {
      conv_wait(b_done + 8 * (n & 1), n >> 1 & 1u, abort_flag, status, 4);
      ++n;
    };
    for (int t = 0; t < T; ++t)
      if (place_of(t) <= 0) load(t);
    for (int t = 0; t < T; ++t) {
      const int b = buffer_of(t);
      conv_wait(b_full + 8 * b, ph_full >> b & 1u, abort_flag, status, 1);
      ph_full ^= 1u << b;
      issue_z(t);
      done();
      if (place_of(t) >= 0 && t + 2 < T && place_of(t + 2) >= 0) load(t + 2);
    }
    for (int step = 0; step < p.steps; ++step) {
      done();   // A is there
      constexpr uint32_t idesc = idesc_fp16(128, 64, false, false);
      const uint64_t a = sdesc(sP, 16, 1024, SWZ_128B);
      fence_after();
#pragma unroll
      for (int q = 0; q < kSide / 16; ++q) mma_ss_elect(tmem + kColD, a + (q * 32 >> 4), a + (q * 32 >> 4), idesc, q > 0);
      commit_elect(b_xp);
      done();   // P is there
      issue_xp(0);
      if (T > 1) issue_xp(1);
      for (int t = 0; t < T; ++t) {
        done();
        if (step + 1 < p.steps) issue_z(t);
        if (t + 2 < T) issue_xp(t + 2);
      }
    }
    __syncwarp();
    if (*abort_flag) {   // copies and products that nothing waited for land before this memory is given back
      commit_elect(b_drain);
      if (lane == 0) {
        const uint64_t t0 = globaltimer_ns();
        auto drain = [&](uint32_t bar, uint32_t parity) {
          while (!mbar_try_wait(bar, parity) && globaltimer_ns() - t0 < 200000000ull) {
          }
        };
        for (int t = 0; t < T; ++t) drain(b_full + 8 * buffer_of(t), (ph_full >> buffer_of(t) & 1u) ^ 1u);
        drain(b_drain, 0);
      }
      __syncwarp();
    }
    fence_before();
    __syncthreads();
    return;
  }
  auto done = [&] {   // what was written is there for the tensor cores, what was read may be overwritten
    fence_async();
    fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(b_done + 8 * (turn & 1));
    ++turn;
  };
  auto wait_warp = [&](uint32_t bar, uint32_t& ph, int i, int where) {
    wait(bar, ph, i, where);
    __syncwarp();
    fence_after();
  };
  float z[32];   // this thread's part of [hi^T hi; lo^T hi]: its row, 32 columns
  auto add_z = [&] {   // of the last tile that went into it
    wait_warp(b_z, ph_z, 0, 3);
    uint32_t v[32];
    tmem_ld32(tmem + lanes + kColZ + half * 32, v);
    tmem_wait_ld(v);
#pragma unroll
    for (int i = 0; i < 32; ++i) z[i] += __uint_as_float(v[i]);
  };
  // Z = top / 2 + bottom of 128 x 64 values, a row and 32 columns of a thread
  auto fold = [&](const float (&v)[32]) {
    if (quad < 2)
#pragma unroll
      for (int i = 0; i < 32; ++i) Z[z_at(row, half * 32 + i)] = 0.5f * v[i];
    sync_workers();
    if (quad >= 2) {
      float u[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) u[i] = Z[z_at(row - 64, half * 32 + i)];
#pragma unroll
      for (int i = 0; i < 32; ++i) Z[z_at(row - 64, half * 32 + i)] = u[i] + v[i];
    }
    sync_workers();
  };
  // a tile's row of this thread into TMEM, as the tensor cores take it
  auto keep = [&](int t, const uint4 (&h)[4], const uint4 (&l)[4]) {
    const uint32_t at = tmem + lanes + kColX + place_of(t) * 64 + half * 16;
    tmem_st16(at, (const uint32_t(&)[16])h);
    tmem_st16(at + 32, (const uint32_t(&)[16])l);
    tmem_wait_st();
  };

  // the first Z
#pragma unroll
  for (int i = 0; i < 32; ++i) z[i] = 0.f;
#pragma unroll 1
  for (int t = 0; t < T; ++t) {
    if (place_of(t) >= 0) {
      wait_warp(b_full, ph_full, buffer_of(t), 1);
      const char* tile = smem + buffer_of(t) * kTile;
      uint4 h[4], l[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        h[q] = *(const uint4*)(tile + vector_at(row, half * 4 + q));
        l[q] = *(const uint4*)(tile + kPiece + vector_at(row, half * 4 + q));
      }
      keep(t, h, l);
    }
    add_z();
    done();
  }

  int barriers = 0;
#pragma unroll 1
  for (int step = 0; step < p.steps; ++step) {
    const bool last = step + 1 == p.steps;
    // Z of all CTAs
    fold(z);
    if (G > 1) {
      // in two places in turn: a CTA may write the next step's while another still reads these
      const float* parts = p.part + (size_t)(step & 1) * G * kSide * kSide;
      float* mine = p.part + ((size_t)(step & 1) * G + blockIdx.x) * kSide * kSide;
#pragma unroll
      for (int i = 0; i < kSide * kSide / kThreads; ++i) {
        const int e = i * kThreads + tid;
        __stcg(mine + e, Z[z_at(e / kSide, e % kSide)]);
      }
      grid_barrier(p.ints, ++barriers * G, abort_flag, status);
      float v[kSide * kSide / kThreads];
      if (G <= kFew) {   // every CTA adds up all of them
#pragma unroll
        for (int i = 0; i < kSide * kSide / kThreads; ++i) v[i] = 0.f;
#pragma unroll 1
        for (int q = 0; q < G; ++q)
#pragma unroll
          for (int i = 0; i < kSide * kSide / kThreads; ++i) v[i] += __ldcg(parts + (size_t)q * kSide * kSide + i * kThreads + tid);
      } else {
        // 32 elements by a warp, or by eight (16 CTAs 56 and 72 us, 24 66 and 68, 32 58 and 64,
        // 47 76 and 64, 152 88 and 68)
        if (G <= 32) {
          for (int e0 = (blockIdx.x * 8 + warp) * 32; e0 < kSide * kSide; e0 += G * 8 * 32) {
            float s = 0.f;
#pragma unroll 16
            for (int q = 0; q < G; ++q) s += __ldcg(parts + (size_t)q * kSide * kSide + e0 + lane);
            __stcg(p.sum + e0 + lane, s);
          }
        } else {   // by eight warps, every eighth part each, in order
          for (int e0 = blockIdx.x * 32; e0 < kSide * kSide; e0 += G * 32) {
            float u[kSms / 8], s = 0.f;   // all loads under way together
#pragma unroll
            for (int q = 0; q < kSms / 8; ++q)
              u[q] = warp + 8 * q < G ? __ldcg(parts + (size_t)(warp + 8 * q) * kSide * kSide + e0 + lane) : 0.f;
#pragma unroll
            for (int q = 0; q < kSms / 8; ++q) s += u[q];
            Z[warp * 32 + lane] = s;
            sync_workers();
            if (warp == 0) {
#pragma unroll
              for (int q = 1; q < 8; ++q) s += Z[q * 32 + lane];
              __stcg(p.sum + e0 + lane, s);
            }
            sync_workers();
          }
        }
        grid_barrier(p.ints, ++barriers * G, abort_flag, status);
#pragma unroll
        for (int i = 0; i < kSide * kSide / kThreads; ++i) v[i] = __ldcg(p.sum + i * kThreads + tid);
      }
#pragma unroll
      for (int i = 0; i < kSide * kSide / kThreads; ++i) Z[z_at((i * kThreads + tid) / kSide, tid % kSide)] = v[i];
      if (last && tid == 0) *others = *(volatile int*)status;
      sync_workers();
    }
    // A in pieces, [hi; lo]; a thread has 16 columns of a row
    const int i = tid >> 2, j0 = (tid & 3) * 16, t0 = shift[step], t1 = shift[step + 1];
    auto put_square = [&](const float (&v)[16]) {   // A, and later P, side by side in the same place
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        uint4 h, l;
        split2(v[8 * q], v[8 * q + 1], h.x, l.x);
        split2(v[8 * q + 2], v[8 * q + 3], h.y, l.y);
        split2(v[8 * q + 4], v[8 * q + 5], h.z, l.z);
        split2(v[8 * q + 6], v[8 * q + 7], h.w, l.w);
        char* to = smem + kOffP + vector_at(i, (tid & 3) * 2 + q);
        *(uint4*)to = h;
        *(uint4*)(to + kSquare / 2) = l;
      }
    };
    float A[16];
    const float to_a = ldexpf(1.f / kUnit, -2 * t0);
#pragma unroll
    for (int e = 0; e < 16; ++e) A[e] = to_a * (Z[z_at(i, j0 + e)] + Z[z_at(j0 + e, i)]);
    put_square(A);
    done();
    wait_warp(b_xp, ph_xp, 0, 2);
    {
      uint32_t v[32];
      tmem_ld32(tmem + lanes + kColD + half * 32, v);
      tmem_wait_ld(v);
#pragma unroll
      for (int e = 0; e < 32; ++e) z[e] = __uint_as_float(v[e]);
    }
    fold(z);
    // P = a I + b A + c A A
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float aa = Z[z_at(i, j0 + e)] + Z[z_at(j0 + e, i)];
      A[e] = fmaf(p.b, A[e], p.c / kUnit * aa) + (i == j0 + e ? p.a * kUnit : 0.f);
    }
    put_square(A);
    done();

    // X <- X P and its Z
    const float to_x = last ? ldexpf(1.f / (kUnit * kUnit), -t0) : ldexpf(1.f / kUnit, t1 - t0);
#pragma unroll
    for (int e = 0; e < 32; ++e) z[e] = 0.f;
#pragma unroll 1
    for (int t = 0; t < T; ++t) {
      wait_warp(b_xp, ph_xp, t & 1, 2);
      float y[32];
      {
        uint32_t v[32], w[32];
        tmem_ld32(tmem + lanes + kColD + (t & 1) * 128 + half * 32, v);
        tmem_ld32(tmem + lanes + kColD + (t & 1) * 128 + 64 + half * 32, w);
        tmem_wait_ld(v);
        tmem_wait_ld(w);
#pragma unroll
        for (int e = 0; e < 32; ++e) y[e] = to_x * (__uint_as_float(v[e]) + __uint_as_float(w[e]));
      }
      char* tile = smem + buffer_of(t) * kTile;
      const int64_t m0 = tile_row(t);
      if (!last) {   // in its place: the product that read it has ended
        uint4 h[4], l[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          split2(y[8 * q], y[8 * q + 1], h[q].x, l[q].x);
          split2(y[8 * q + 2], y[8 * q + 3], h[q].y, l[q].y);
          split2(y[8 * q + 4], y[8 * q + 5], h[q].z, l[q].z);
          split2(y[8 * q + 6], y[8 * q + 7], h[q].w, l[q].w);
          char* to = tile + vector_at(row, half * 4 + q);
          *(uint4*)to = h[q];
          *(uint4*)(to + kPiece) = l[q];
        }
        if (place_of(t) >= 0) keep(t, h, l);
        if (t > 0) add_z();
        done();
      } else {
        float* stage = (float*)tile;
#pragma unroll
        for (int q = 0; q < 8; ++q)
          *(float4*)(stage + group_at(row, half * 8 + q)) = make_float4(y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]);
        sync_workers();
        const float fill = *abort_flag || *others ? NAN : 0.f;   // the result of a wait that ran out shows
        if (p.j.out.dtype == NMD_DT_FP32) put_tile<float>(p, stage, m0, fill);
        else if (p.j.out.dtype == NMD_DT_BF16) put_tile<bf16>(p, stage, m0, fill);
        else put_tile<__half>(p, stage, m0, fill);
        done();
      }
    }
    if (!last) add_z();
  }
  fence_after();
  fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, kTmem);
}

int grid_of(int64_t tiles) {   // the fewest CTAs with the fewest tiles each
  const int64_t each = (tiles + kSms - 1) / kSms;
  return (int)((tiles + each - 1) / each);
}

}  // namespace

size_t strip_bytes(int64_t M) {
  const int G = grid_of((M + kRows - 1) / kRows);
  return G > 1 ? (size_t)(2 * G + 1) * kSide * kSide * 4 : 0;
}

nmd_status strip_run(const Job& j, const Pieces& X, int steps, const double* k, int* ints, void* ws, cudaStream_t s) {
  static std::atomic<int> ready[kMaxDevices];
  if (!per_device(ready, [] {
        return cudaFuncSetAttribute(strip_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem) == cudaSuccess;
      }))
    return NMD_ERR_CUDA;
  Strip p{};
  p.j = j;
  p.x = X;
  p.M = X.rows;
  p.turned = j.R <= j.C;
  p.tiles = (int)((X.rows + kRows - 1) / kRows);
  p.steps = steps;
  p.a = (float)k[0];
  p.b = (float)k[1];
  p.c = (float)k[2];
  p.ints = ints;
  const int G = grid_of(p.tiles);
  p.part = (float*)ws;
  p.sum = p.part + (size_t)2 * G * kSide * kSide;
  CUtensorMap tx;
  if (!map_of(X, kRows, &tx)) return NMD_ERR_CUDA;
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr{};
  if (G > 1) {   // its CTAs wait for one another
    attr.id = cudaLaunchAttributeCooperative;
    attr.val.cooperative = 1;
  } else {
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
  }
  cfg.gridDim = dim3((unsigned)G);
  cfg.blockDim = dim3(kThreads + 32);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = s;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, strip_kernel, tx, p) == cudaSuccess ? NMD_OK : NMD_ERR_CUDA;
}

}  // namespace muon
}  // namespace nmd

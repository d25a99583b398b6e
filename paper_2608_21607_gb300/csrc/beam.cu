// One step of beam search over the rows of a logits matrix, and the beams'
// states in the order of their parents (formulas in include/nmd.h).
//
// A cluster of CTAs per group reads the rows of the beams that are in use once.  The
// rows' columns are dealt to its CTAs in equal contiguous runs, whatever the number
// of beams; a run that ends one row and begins the next is two segments.  Of a
// segment a CTA keeps the running sum of the softmax and the `width` largest logits:
// within a row the logits' order is that of the offers, so that nothing has to wait
// for the row's sum.  The segments' lists go to the cluster's first CTA, which adds up
// the sums and merges the lists by the offers' values, each kept as two fp32 values.
//
// What is largest is found on the way at the cost of one comparison per four vectors:
// a group of elements whose sum of powers is below the power of the width-th largest
// so far (where that is not too small for a sum in fp32) holds nothing that could
// displace it.  Of the groups that pass, all of them where a row is flat, the largest
// element is compared; the elements themselves are looked at in the few that still pass.
#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "row_vec.cuh"
#include "tc_ptx.cuh"

namespace nmd {
namespace {

constexpr int kThreads = 256;
constexpr int kMostBeams = 64, kMostWidth = 128, kMostCluster = 8;
constexpr int kSmallRow = 1024;   // columns of a row that a warp takes
constexpr int kDepth = 2;   // groups of four vectors under way

struct Select {
  const void* x;
  int64_t V, ld;
  int K, width;
  Scale c;
  float2 inv_temp;   // 1 / tau as the sum of two
  const float* scores;
  const uint8_t* finished;
  int64_t end;
  float* out_scores;
  int64_t* parents;
  int64_t* tokens;
  uint8_t* out_finished;
};

// A logit and its column as one number: larger logits first, of equal ones (0 and -0
// are equal) the lower column.
typedef unsigned long long entry_t;
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return (int)b < 0 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ entry_t entry_of(float x, int64_t col) { return (entry_t)order_of(x) << 32 | (0xffffffffu - (uint32_t)col); }
__device__ __forceinline__ float value_of(entry_t e) {
  const uint32_t o = (uint32_t)(e >> 32);
  return __uint_as_float((int)o < 0 ? o & 0x7fffffffu : ~o);
}
// A value hi + lo, hi rounded to nearest, as one number above 0 (finite hi)
__device__ __forceinline__ entry_t order_of(float hi, float lo) { return (entry_t)order_of(hi) << 32 | order_of(lo); }
__device__ __forceinline__ float score_of(entry_t o) {
  const uint32_t h = (uint32_t)(o >> 32);
  return __uint_as_float((int)h < 0 ? h & 0x7fffffffu : ~h);
}
// score + lp in two fp32 values: offers are compared to 2^-40 of them, not as the rounded
// sums; 0 if it is not finite
__device__ __forceinline__ entry_t sum_of(float score, LogProb lp) {
  const float s = score + lp.hi, t = s - score, rest = (score - (s - t)) + (lp.hi - t) + lp.lo;
  const float hi = s + rest;
  return fabsf(hi) < INFINITY ? order_of(hi, rest - (hi - s)) : 0;
}
__device__ __forceinline__ uint32_t column_of(entry_t e) { return 0xffffffffu - (uint32_t)e; }

// The largest entries so far, by a CTA.
struct Best {
  entry_t* list;       // room
  entry_t* sorted;     // width
  int* count;          // offered; those past the room are lost
  int* lost;
  entry_t* least;      // what an entry has to be above; at least `width` entries are at or above it
  int width, limit, room;

  __device__ __forceinline__ void clear() {   // by one thread
    *count = 0;
    *lost = 0;
    *least = entry_of(-INFINITY, 0);   // a banned column is not among them
  }
  __device__ __forceinline__ void offer(entry_t e, entry_t bar) {
    if (e <= bar) return;
    const int p = atomicAdd(count, 1);
    if (p < room) list[p] = e;
  }
  __device__ __forceinline__ void offer_warp(entry_t e, entry_t bar) {
    const unsigned some = __ballot_sync(0xffffffffu, e > bar);
    if (some == 0) return;
    const int lane = threadIdx.x & 31;
    int p = 0;
    if (lane == 0) p = atomicAdd(count, __popc(some));
    p = __shfl_sync(0xffffffffu, p, 0) + __popc(some & ((1u << lane) - 1));
    if (e > bar && p < room) list[p] = e;
  }
  // The width largest of the list, in order.  By the whole CTA, between barriers.
  __device__ __forceinline__ void cut() {
    const int n = min(*count, room);
    if (threadIdx.x == 0 && *count > room) *lost = 1;
    __syncthreads();
    if (n <= 32) {   // a warp per entry: its rank among the others by a vote
      const int lane = threadIdx.x & 31;
      const entry_t mine = lane < n ? list[lane] : 0;
      for (int i = threadIdx.x >> 5; i < n; i += kThreads / 32) {
        const entry_t e = list[i];
        const int rank = __popc(__ballot_sync(0xffffffffu, mine > e));
        if (lane == 0 && rank < width) sorted[rank] = e;
      }
    } else {   // a thread per entry, two others at a time
      for (int i = threadIdx.x; i < n; i += kThreads) {
        const entry_t e = list[i];
        int rank = 0, k = 0;
#pragma unroll 4
        for (; k + 1 < n; k += 2) {
          const ulonglong2 u = *(const ulonglong2*)(list + k);
          rank += (u.x > e) + (u.y > e);
        }
        if (k < n) rank += list[k] > e;
        if (rank < width) sorted[rank] = e;
      }
    }
    __syncthreads();
    const int kept = min(n, width);
    for (int i = threadIdx.x; i < kept; i += kThreads) list[i] = sorted[i];
    if (threadIdx.x == 0) {
      *count = kept;
      if (kept == width) *least = max(*least, sorted[width - 1]);
    }
    __syncthreads();
  }
};

// A first bar: the width-th largest of the maxima of groups of elements that threads
// have in hand, as at least that many elements are not below it.  A maximum's column is
// taken to be the last of the vector that has it, so that rows of equal values offer few.
// Where there are as many of 32 groups of threads, every warp ranks them; otherwise they
// are those of single threads.  `vectors`: of the segment, from column `col0` on.
template <class T, class G>
__device__ __forceinline__ entry_t first_bar(G get, int64_t col0, int vectors, const Best& best, entry_t* bests) {
  float m = Vec<T>::top(get(0));
  int at = 0;
#pragma unroll
  for (int q = 1; q < 4; ++q) {
    const float f = Vec<T>::top(get(q));
    if (f > m) at = q;
    m = max_nan(m, f);
  }
  entry_t o = entry_of(m, col0 + (int64_t)(at * kThreads + threadIdx.x + 1) * Vec<T>::N - 1);   // no two are equal
  const int lane = threadIdx.x & 31;
  entry_t bar = *best.least;
  constexpr int kGroup = kThreads / 32;
  if (kGroup * best.width <= min(vectors, kThreads)) {
#pragma unroll
    for (int d = 1; d < kGroup; d *= 2) o = max(o, __shfl_xor_sync(0xffffffffu, o, d));
    if (lane % kGroup == 0) bests[threadIdx.x / kGroup] = o;
    __syncthreads();
    o = bests[lane];
    int rank = 0;
#pragma unroll 4
    for (int k = 0; k < 16; ++k) {
      const ulonglong2 u = ((const ulonglong2*)bests)[k];
      rank += (u.x > o) + (u.y > o);
    }
    o = __shfl_sync(0xffffffffu, o, __ffs(__ballot_sync(0xffffffffu, rank == best.width - 1)) - 1);
    bar = max(bar, o - 1);
    if (lane == 0) *best.least = bar;   // every warp the same
    __syncwarp();
  } else {
    if (vectors < best.width) return bar;   // the same for all
    bests[threadIdx.x] = o;
    __syncthreads();
    int rank = 0;
    const int some = min((vectors + 1) & ~1, kThreads);   // (of the others o is that of -inf)
#pragma unroll 4
    for (int k = 0; k < some; k += 2) {
      const ulonglong2 u = *(const ulonglong2*)(bests + k);
      rank += (u.x > o) + (u.y > o);
    }
    if (threadIdx.x < some && rank == best.width - 1) *best.least = max(bar, o - 1);
    __syncthreads();
    bar = *best.least;
  }
  return bar;
}

// A segment's largest entries again, where there were more offers than room: one
// vector of a thread at a time, and where more than `width` threads have something to
// offer, the width-th of their largest entries is the bar first.  A round adds at most
// 8 width entries.  Rows that rise from column to column.
template <class T>
__device__ __noinline__ void again(Best best, entry_t* bests, const uint4* xv, int n, int64_t col0, T xs, int64_t scalar) {
  constexpr int N = Vec<T>::N;
  if (threadIdx.x == 0) best.clear();
  __syncthreads();
  const int rounds = (n + kThreads - 1) / kThreads;
  for (int i = 0; i <= rounds; ++i) {
    const int v = i * kThreads + threadIdx.x;
    const entry_t bar = *best.least;
    entry_t mine[N], top = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) mine[e] = 0;
    if (i == rounds) {
      if (scalar >= 0) mine[0] = entry_of(Vec<T>::get(xs), scalar);
    } else if (v < n) {
      const uint4 w = xv[v];
#pragma unroll
      for (int e = 0; e < N; ++e) mine[e] = entry_of(Vec<T>::get(((const T*)&w)[e]), col0 + (int64_t)v * N + e);
    }
#pragma unroll
    for (int e = 0; e < N; ++e) top = max(top, mine[e]);
    const int some = __syncthreads_count(top > bar);
    if (some == 0) continue;
    entry_t over = bar;
    if (some > best.width) {
      bests[threadIdx.x] = top;
      __syncthreads();
      int rank = 0;
      for (int k = 0; k < kThreads; ++k) rank += bests[k] > top;
      if (top > bar && rank == best.width - 1) *best.least = top - 1;
      __syncthreads();
      over = *best.least;
    }
#pragma unroll
    for (int e = 0; e < N; ++e) best.offer(mine[e], over);
    __syncthreads();
    if (*(volatile int*)best.count >= best.limit) best.cut();
    else __syncthreads();
  }
}

// Dynamic shared memory: slots, then the lists
struct Shape {
  int cluster, limit, room, small;
  size_t off_list, off_sorted, off_all, off_places, bytes;
};
Shape shape_of(int64_t K, int width, int cluster, bool small = false) {
  Shape s;
  s.small = small;
  s.cluster = cluster;
  s.limit = 2 * width;
  s.room = s.limit + (width <= 32 ? 64 : 36) * width;   // (in rows of equal values a first round offers eight vectors for each)
  s.off_list = (size_t)kDepth * 4 * kThreads * 16;   // (16-byte aligned, as the pairs that are read of it)
  s.off_sorted = s.off_list + (size_t)s.room * 8;
  s.off_all = s.off_sorted + (size_t)width * 8;
  const size_t offers = ((size_t)(K + cluster) * width + K) * 8;   // the segments' lists and finished beams, in the first CTA
  s.off_places = s.off_all + offers;
  s.bytes = s.off_places + offers;
  return s;
}

__device__ __forceinline__ uint32_t first_cta(const void* p) {   // the address in the cluster's first CTA
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"(tc::smem_u32(p)));
  return a;
}
__device__ __forceinline__ void put_remote(uint32_t at, entry_t v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(at), "l"(v) : "memory");
}

// Bound by HBM where there is much to read: 128 groups of four rows of 139,255 bf16
// columns (a tenth of the beams finished) take 40 us, of which 20 are the rows at 6.4
// TB/s and the rest the start, the last cut and the merge, which nothing covers as all
// CTAs run at a time (twice as many CTAs: 49 us).  64 groups of eight rows of 50,001 fp16
// columns 30 us; one group of four rows of 139,255 18 us, eight CTAs' latency.  A bar that
// needs every element compared, or a list per warp, cost as much again as the sums.  The
// 128 groups with logits of standard deviation one take 42 us (108 without the groups'
// maxima), and with all logits equal 51 (205 with a first bar that is a value alone, whose
// offers run over).
template <class T>
__global__ void __launch_bounds__(kThreads, 4) select_kernel(const __grid_constant__ Select a, const __grid_constant__ Shape shape) {
  constexpr int N = Vec<T>::N;
  constexpr int kSegments = kMostBeams + kMostCluster;
  extern __shared__ uint4 slots[];
  __shared__ Stat red[kThreads / 32], stats[kSegments];
  __shared__ int counts[kSegments], row_beam[kMostBeams], done_beam[kMostBeams], count, lost, rows_in_use, finished_in_use;
  __shared__ float row_score[kMostBeams], done_score[kMostBeams];
  __shared__ Stat row_stat[kMostBeams];
  __shared__ float row_over[kMostBeams];
  __shared__ int row_first[kMostBeams], row_last[kMostBeams], seg_row[kSegments], next[kSegments + kMostBeams];   // CTAs of a row, row of a segment
  __shared__ entry_t least;
  __shared__ __align__(16) entry_t bests[kThreads];
  char* raw = (char*)slots;
  Best best{(entry_t*)(raw + shape.off_list), (entry_t*)(raw + shape.off_sorted), &count, &lost, &least, a.width, shape.limit,
            shape.room};
  entry_t* all = (entry_t*)(raw + shape.off_all);
  entry_t* places = (entry_t*)(raw + shape.off_places);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  unsigned csize, rank;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(csize));
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const int log_cluster = __ffs(csize) - 1;
  if (csize > 1) cluster_arrive();   // waited for before the first CTA's shared memory is written
  const int64_t b = blockIdx.x / csize;

  // the beams whose rows are read, and the finished ones
  if (warp == 0) {
    int rows = 0, done = 0;
    for (int k0 = 0; k0 < a.K; k0 += 32) {
      const int k = k0 + lane;
      const float s = k < a.K ? a.scores[b * a.K + k] : -INFINITY;
      const uint8_t ended = k < a.K && a.finished != nullptr ? a.finished[b * a.K + k] : 0;
      const bool used = fabsf(s) < INFINITY, fin = used && ended != 0;
      const unsigned m = __ballot_sync(0xffffffffu, used && !fin), f = __ballot_sync(0xffffffffu, fin);
      const int before = __popc(m & ((1u << lane) - 1)), fbefore = __popc(f & ((1u << lane) - 1));
      if (used && !fin) {
        row_beam[rows + before] = k;
        row_score[rows + before] = s;
      }
      if (fin) {
        done_beam[done + fbefore] = k;
        done_score[done + fbefore] = s;
      }
      rows += __popc(m);
      done += __popc(f);
    }
    if (lane == 0) {
      rows_in_use = rows;
      finished_in_use = done;
    }
  }
  __syncthreads();
  const int R = rows_in_use;
  // The rows' columns one after another, cut into as many runs as there are CTAs.
  // Segment row + q is what CTA q has of the row: no two have one number, as each step
  // along the runs raises the row, the CTA or both.
  const int64_t total = R * a.V;
  auto border = [&](unsigned q) { return (int64_t)((unsigned long long)(total * q) >> log_cluster); };   // (csize is a power of two)
  const int64_t from = border(rank), to = border(rank + 1);
  if (rank == 0) {
    for (int row = tid; row < R; row += kThreads) {
      unsigned q = 0;
      while (q + 1 < csize && border(q + 1) <= row * a.V) ++q;
      row_first[row] = q;
      while (q + 1 < csize && border(q + 1) < (row + 1) * a.V) ++q;
      row_last[row] = q;
    }
    for (int i = tid; i < kSegments; i += kThreads) seg_row[i] = -1;
  }
  const uint4* mine = slots + tid;
  bool waited = csize == 1;

  // Short rows: a warp each, in fp32 in its part of the slots; the largest is taken `width`
  // times, a lane keeping the largest of its own columns l, l + 32, ...
  if (shape.small) {
    float* x = (float*)slots + warp * kSmallRow;
    const int V = (int)a.V;
#pragma unroll 1
    for (int r = warp; r < R; r += kThreads / 32) {
      const T* from_row = (const T*)a.x + (b * a.K + row_beam[r]) * a.ld;
      float m = -INFINITY;
#pragma unroll 8
      for (int v = lane; v < V; v += 32) {
        const float f = Vec<T>::get(from_row[v]);
        x[v] = f;
        m = max_nan(m, f);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
      const bool near = is_near(m, a.c), some = m > -INFINITY && m < INFINITY;
      const float ref = near ? ref_of(m, a.c) : 0.f;
      float S = 0.f;
      entry_t top = 0;
      if (some) {
#pragma unroll 4
        for (int v = lane; v < V; v += 32) {
          const float f = x[v];
          S += near ? ex2(fmaf(f, a.c.hi, -ref) + f * a.c.lo) : power(f, m, a.c);
          top = max(top, entry_of(f, v));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) S += __shfl_xor_sync(0xffffffffu, S, o);
      }
      const entry_t bar = entry_of(-INFINITY, 0);
      int n = 0;
#pragma unroll 1
      for (; some && n < a.width; ++n) {
        const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(top >> 32));
        const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(top >> 32) == hi ? (uint32_t)top : 0u);
        const entry_t e = (entry_t)hi << 32 | lo;
        if (e <= bar) break;
        if (top == e) {   // one lane: its next
          all[r * a.width + n] = e;
          x[column_of(e)] = -INFINITY;
          top = 0;
#pragma unroll 4
          for (int v = lane; v < V; v += 32) top = max(top, entry_of(x[v], v));
        }
        __syncwarp();
      }
      if (lane == 0) {
        stats[r] = Stat{m, S};
        counts[r] = n;
      }
      __syncwarp();
    }
  }
  // A segment: its row, its vectors, and the element before or after the row's vectors that
  // this thread has.  What comes first of it is under way before the one before is finished.
  int row = 0, n = 0, ahead = 0;
  int64_t at = shape.small ? to : from, col0 = 0, scalar = -1;   // col0: of its first vector
  const uint4* xv = nullptr;
  T xs = Vec<T>::put(0.f);
  auto load = [&](int slot) {
#pragma unroll
    for (int q = 0; q < 4; ++q, ahead += kThreads)
      if (ahead < n) copy_async(tc::smem_u32(mine + (slot * 4 + q) * kThreads), xv + ahead);
      else slots[(slot * 4 + q) * kThreads + tid] = Vec<T>::none();   // -inf past the segment's end
    copy_commit();
  };
  auto begin = [&] {   // the segment at `at`
    while (at >= (row + 1) * a.V) ++row;
    const int64_t e0 = at - row * a.V, e1 = min(a.V, to - row * a.V);
    at = row * a.V + e1;
    const T* x = (const T*)a.x + (b * a.K + row_beam[row]) * a.ld;
    const Span sp = span_of(x, a.V);
    // the cut between two CTAs falls on the same vector for both
    auto vector_at = [&](int64_t e) { return e == 0 ? (int64_t)0 : e == a.V ? sp.nvec : min(sp.nvec, max((int64_t)0, (e - sp.head) / N)); };
    const int64_t v0 = vector_at(e0);
    n = (int)(vector_at(e1) - v0);
    xv = (const uint4*)(x + sp.head) + v0;
    col0 = sp.head + v0 * N;
    scalar = -1;
    if (e0 == 0 && tid < sp.head) scalar = tid;
    if (e1 == a.V && tid >= 32 && tid - 32 < sp.tail) scalar = sp.head + sp.nvec * N + tid - 32;
    ahead = tid;
#pragma unroll
    for (int d = 0; d < kDepth; ++d) load(d);
    if (scalar >= 0) xs = x[scalar];
  };
  bool more = at < to;
  if (more) begin();
  while (more) {
    if (tid == 0) best.clear();
    __syncthreads();

    Running<T> run;
    const int rounds = (n + 4 * kThreads - 1) / (4 * kThreads);
    int d = 0;
    for (int i = 0; i < rounds; ++i) {
      auto get = [&](int q) { return mine[(d * 4 + q) * kThreads]; };
      copy_wait<kDepth - 1>();
      const float group = run.add(get, a.c);
      // What has to be passed only rises; an older value lets more through, not less
      const entry_t bar = i == 0 ? first_bar<T>(get, col0, n, best, bests) : *(volatile entry_t*)&least;
      const float bar_x = value_of(bar);
      const float power = ex2(fmaf(bar_x, a.c.hi, -run.r) + bar_x * a.c.lo);
      // (0.99: far more than the sum's rounding.  Below 2^-124 a sum has lost half of its
      // elements, which are taken 2^-2 smaller: beside a dominating column it says nothing,
      // and everything passes well before that.)  In flat rows most sums pass; there the
      // largest element says whether there is something (for four threads that costs more
      // than it saves).  The warp looks at a thread's elements together, one or none a lane.
      unsigned look = __ballot_sync(0xffffffffu, !(power >= 0x1p-120f && group < 0.99f * power));
      if (__popc(look) > 4) {
        float m = Vec<T>::top(get(0));
#pragma unroll
        for (int q = 1; q < 4; ++q) m = max_nan(m, Vec<T>::top(get(q)));
        // (after the first round what is equal to the bar comes after it)
        look &= __ballot_sync(0xffffffffu, i == 0 ? !(m < bar_x) : !(m <= bar_x));
      }
      if (look != 0) {
        __syncwarp();   // the copies of all lanes have landed
        do {
          const int from = __ffs(look) - 1;
          look &= look - 1;
          const int q = lane / N, vec = i * 4 * kThreads + warp * 32 + from + q * kThreads;
          entry_t e = 0;
          if (q < 4) {   // (-inf past the segment's end is below every bar)
            const T* its = (const T*)(slots + (d * 4 + q) * kThreads + warp * 32 + from);
            e = entry_of(Vec<T>::get(its[lane % N]), col0 + (int64_t)vec * N + lane % N);
          }
          best.offer_warp(e, bar);
        } while (look != 0);
        __syncwarp();   // before the slots are filled again
      }
      load(d);
      if (++d == kDepth) d = 0;
      // a higher bar after 2, 4, 8 and every 16 rounds
      if ((i & 15) == 15 || i == 1 || i == 3 || i == 7) {
        __syncthreads();
        if (*(volatile int*)&count >= shape.limit) best.cut();   // the same for all: the next offers come after a barrier
        else __syncthreads();
      }
    }
    if (scalar >= 0) {
      run.add(Vec<T>::get(xs), a.c);
      best.offer(entry_of(Vec<T>::get(xs), scalar), *(volatile entry_t*)&least);
    }
    copy_wait<0>();
    // the segment's sum and list
    const Stat st = merge_lanes<32>(run.s, a.c);
    if (lane == 0) red[warp] = st;
    __syncthreads();
    if (*(volatile int*)&count > shape.room || lost) {   // more offers than there is room for (rising rows)
      __syncthreads();
      again<T>(best, bests, xv, n, col0, xs, scalar);
    }
    const int seg = row + (int)rank;
    more = at < to;
    if (more) begin();
    best.cut();
    if (!waited) {
      cluster_wait();
      waited = true;
    }
    const int kept = count;
    const uint32_t to_list = first_cta(all + (int64_t)seg * a.width);
    for (int i = tid; i < kept; i += kThreads) put_remote(to_list + i * 8, best.sorted[i]);
    if (warp == 0) {
      const Stat s = merge_lanes<32>(lane < kThreads / 32 ? red[lane] : Stat{-INFINITY, 0.f}, a.c);
      if (lane == 0) {
        put_remote(first_cta(stats + seg), (entry_t)__float_as_uint(s.m) | (entry_t)__float_as_uint(s.S) << 32);
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(first_cta(counts + seg)), "r"(kept) : "memory");
      }
    }
    __syncthreads();
  }
  if (csize > 1) {
    if (!waited) cluster_wait();
    cluster_arrive();
    cluster_wait();
    if (rank != 0) return;
  } else {
    __syncthreads();
  }

  // The values of all offers, as whole numbers in their order.  Places: beam, column.
#pragma unroll 1
  for (int row = tid; row < R; row += kThreads) {
    const int q0 = row_first[row], q1 = row_last[row];
    float m = -INFINITY, S = 0.f;
    for (int q = q0; q <= q1; ++q) m = max_nan(m, stats[row + q].m);
    for (int q = q0; q <= q1; ++q) S += stats[row + q].S * rescale(stats[row + q].m, m, a.c);
    row_stat[row] = Stat{m < INFINITY ? m : NAN, S};   // +inf: no distribution
    row_over[row] = above(m, a.c);
    for (int q = q0; q <= q1; ++q) seg_row[row + q] = row;
  }
  const int segments = R == 0 ? 0 : R + (int)csize - 1, listed = segments * a.width, offers = listed + finished_in_use;
  for (int i = tid; i < finished_in_use; i += kThreads) {
    all[listed + i] = order_of(done_score[i], 0.f);
    places[listed + i] = (entry_t)done_beam[i] << 32 | (uint32_t)a.end;
  }
  __syncthreads();
#pragma unroll 1
  for (int i = tid; i < listed; i += kThreads) {
    const int seg = i / a.width, row = seg_row[seg];
    entry_t v = 0;
    if (row >= 0 && i - seg * a.width < counts[seg]) {
      const entry_t e = all[i];
      places[i] = (entry_t)row_beam[row] << 32 | column_of(e);
      const LogProb lp = log_prob(value_of(e), row_stat[row], row_over[row], a.inv_temp);
      v = sum_of(row_score[row], lp);
    }
    all[i] = v;
  }
  __syncthreads();

  // The order of two offers: the larger value, then the lower beam, then its lower column
  auto put = [&](int i, entry_t value, entry_t place) {
    const int64_t at = b * a.width + i;
    const bool offered = value != 0;
    const int64_t column = offered ? (int64_t)(uint32_t)place : -1;
    a.out_scores[at] = offered ? score_of(value) : -INFINITY;
    a.parents[at] = offered ? (int64_t)(place >> 32) : 0;
    a.tokens[at] = column;
    if (a.out_finished != nullptr) a.out_finished[at] = offered && column == a.end;
  };
  if (offers <= kThreads) {   // a thread per offer: its rank among all
    const entry_t v = tid < offers ? all[tid] : 0, place = v != 0 ? places[tid] : 0;
    const int there = __syncthreads_count(v != 0);
    if (v != 0) {
      int rank = 0;
#pragma unroll 8
      for (int k = 0; k < offers; ++k) {
        const entry_t u = all[k];
        rank += u > v;
        if (u == v && k != tid) rank += places[k] < place;
      }
      if (rank < a.width) put(rank, v, place);
    }
    if (tid >= there && tid < a.width) put(tid, 0, 0);
    return;
  }
  // More offers: only those not below the width-th largest of the threads' largest ones
  {
    entry_t mine_top = 0;
    for (int i = tid; i < offers; i += kThreads) mine_top = max(mine_top, all[i]);
    bests[tid] = mine_top;
    if (tid == 0) count = 0, least = 1;
    __syncthreads();
    int rank = 0;
#pragma unroll 4
    for (int k = 0; k < kThreads; k += 2) {
      const ulonglong2 u = *(const ulonglong2*)(bests + k);
      rank += (u.x > mine_top || (u.x == mine_top && k < tid)) + (u.y > mine_top || (u.y == mine_top && k + 1 < tid));
    }
    if (rank == a.width - 1 && mine_top != 0) least = mine_top;
    __syncthreads();
    const entry_t bar = least;
    int* which = (int*)best.list;
    for (int i = tid; i < offers; i += kThreads)
      if (all[i] >= bar) {
        const int q = atomicAdd(&count, 1);
        if (q < shape.room) which[q] = i;
      }
    __syncthreads();
    const int n = count;
    if (n <= min(shape.room, 2 * kThreads)) {
      for (int i = tid; i < n; i += kThreads) {
        const entry_t v = all[which[i]], place = places[which[i]];
        int better = 0;
#pragma unroll 4
        for (int k = 0; k < n; ++k) {
          const entry_t u = all[which[k]];
          better += u > v;
          if (u == v && k != i) better += places[which[k]] < place;
        }
        if (better < a.width) put(better, v, place);
      }
      for (int i = n + tid; i < a.width; i += kThreads) put(i, 0, 0);
      return;
    }
  }
  if (warp != 0) return;

  // Lists are in order: the best of their heads is the next offer.  Lane l has lists l,
  // l + 32, ...: the segments', then the finished beams.
  const int lists = segments + finished_in_use;
  for (int l = lane; l < lists; l += 32) next[l] = 0;
  entry_t value = 0, place = 0;   // of this lane's best head
  int from_list = 0;
  auto look = [&] {
    value = 0;
#pragma unroll 1
    for (int l = lane; l < lists; l += 32) {
      const int at = next[l], i = l < segments ? l * a.width + at : listed + l - segments;
      const entry_t v = at < (l < segments ? a.width : 1) ? all[i] : 0;
      if (v == 0) continue;
      if (v > value || (v == value && places[i] < place)) {
        value = v;
        place = places[i];
        from_list = l;
      }
    }
  };
  look();
  for (int i = 0; i < a.width; ++i) {
    // the warp's reductions take 32 bits
    const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(value >> 32));
    bool best_is = (uint32_t)(value >> 32) == hi;
    const uint32_t lo = __reduce_max_sync(0xffffffffu, best_is ? (uint32_t)value : 0u);
    best_is = best_is && (uint32_t)value == lo;
    const uint32_t k = __reduce_min_sync(0xffffffffu, best_is ? (uint32_t)(place >> 32) : 0xffffffffu);
    best_is = best_is && (uint32_t)(place >> 32) == k;
    const uint32_t col = __reduce_min_sync(0xffffffffu, best_is ? (uint32_t)place : 0xffffffffu);
    best_is = best_is && (uint32_t)place == col;
    if (hi == 0) {   // (the order of a number starts above 0)
      if (lane == 0) put(i, 0, 0);
    } else if (best_is) {   // one lane: no two offers have one place
      put(i, value, place);
      ++next[from_list];   // this lane's own
      look();
    }
    __syncwarp();
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
  int K, width, per;      // per: bytes of a row in a CTA's memory, a power of two
  int64_t B, work;
  const int64_t* parents;
};

// A piece of all K rows of a group: `rows` of them at a time, `across` threads to a row.
template <class U>
__device__ __forceinline__ void move(const State& s, int64_t slice, int64_t b, int64_t o, const States& a, char* smem,
                                     const int* parent, unsigned long long needed) {
  const int per = a.per / (int)sizeof(U), across = min(per, kThreads), rows = kThreads / across;
  const int u0 = threadIdx.x & (across - 1), k0 = threadIdx.x / across;
  const int n = (int)min((int64_t)per, s.units - slice * per);
  const char* in = s.in + o * s.in_outer + b * a.K * s.in_row + slice * a.per;
  char* out = s.out + o * s.out_outer + b * a.width * s.out_row + slice * a.per;
  U* buf = (U*)smem;
  if constexpr (sizeof(U) >= 4) {
    for (int u = u0; u < n; u += across) {
#pragma unroll 4
      for (int k = k0; k < a.K; k += rows)
        if (needed >> k & 1) copy_async<sizeof(U)>(tc::smem_u32(buf + k * per + u), (const U*)(in + k * s.in_row) + u);
    }
    copy_commit();
    copy_wait<0>();
  } else {   // loads of a thread eight at a time
    for (int k = k0; k < a.K; k += rows) {
      if (!(needed >> k & 1)) continue;
      const U* from = (const U*)(in + k * s.in_row);
      for (int u = u0; u < n; u += 8 * across) {
        U v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (u + i * across < n) v[i] = from[u + i * across];
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (u + i * across < n) buf[k * per + u + i * across] = v[i];
      }
    }
  }
  __syncthreads();
  for (int u = u0; u < n; u += across) {
#pragma unroll 4
    for (int k = k0; k < a.width; k += rows) {
      const int p = parent[k];
      if (p >= 0) ((U*)(out + k * s.out_row))[u] = buf[p * per + u];
    }
  }
}

// The same for rows that start at any multiple of two bytes: whole words are loaded as
// they lie, and stored as they are to lie, each out of the two words that hold it.
__device__ __forceinline__ void move_halves(const State& s, int64_t slice, int64_t b, int64_t o, const States& a, char* smem,
                                            const int* parent, unsigned long long needed) {
  const int stride = a.per / 4 + 1;   // words of a row here
  const int n = (int)min((int64_t)a.per, s.units * 2 - slice * a.per);   // bytes
  const char* in = s.in + o * s.in_outer + b * a.K * s.in_row + slice * a.per;
  char* out = s.out + o * s.out_outer + b * a.width * s.out_row + slice * a.per;
  uint32_t* buf = (uint32_t*)smem;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int across = min(stride, kThreads) > 128 ? kThreads / 32 : 1;   // warps to a row
  for (int k = warp / across; k < a.K; k += kThreads / 32 / across) {
    if (!(needed >> k & 1)) continue;
    const char* from = in + k * s.in_row;
    const int odd = (int)((uintptr_t)from & 2), words = (odd + n + 3) / 4;
    const char* base = from - odd;
    for (int i = warp % across * 32 + lane; i < words; i += 32 * across) {
      const int at = 4 * i - odd;   // of the row's bytes
      if (at >= 0 && at + 4 <= n) {
        copy_async<4>(tc::smem_u32(buf + k * stride + i), base + 4 * i);
      } else {   // a word that the row has half of
        uint16_t* half = (uint16_t*)(buf + k * stride + i);
        if (at >= 0 && at < n) half[0] = *(const uint16_t*)(from + at);
        if (at + 2 >= 0 && at + 2 < n) half[1] = *(const uint16_t*)(from + at + 2);
      }
    }
  }
  copy_commit();
  copy_wait<0>();
  __syncthreads();
  for (int k = warp / across; k < a.width; k += kThreads / 32 / across) {
    const int p = parent[k];
    if (p < 0) continue;
    char* to = out + k * s.out_row;
    const int odd = (int)((uintptr_t)to & 2), from_odd = (int)((uintptr_t)(in + p * s.in_row) & 2), words = (odd + n + 3) / 4;
    const uint32_t* row = buf + p * stride;
    for (int i = warp % across * 32 + lane; i < words; i += 32 * across) {
      const int at = 4 * i - odd, w = (at + from_odd) >> 2;   // the word that holds byte `at`
      if (at >= 0 && at + 4 <= n) {
        *(uint32_t*)(to + at) = (at + from_odd) & 2 ? __funnelshift_r(row[w], row[w + 1], 16) : row[w];
      } else {
        const uint16_t* half = (const uint16_t*)row;
        if (at >= 0 && at < n) *(uint16_t*)(to + at) = half[(at + from_odd) >> 1];
        if (at + 2 >= 0 && at + 2 < n) *(uint16_t*)(to + at + 2) = half[(at + 2 + from_odd) >> 1];
      }
    }
  }
}

// A CTA takes a piece of all K rows of a group at a time: what is needed of it is in
// shared memory before any row is written, so that rows may change places.  In place,
// rows that stay are not written, and those that nothing goes on from not read.  Bound by
// HBM: 16 tensors of 512 rows of 64 KB (groups of eight, parents at random) take 138 us,
// 5.8 TB/s over what moves; with four CTAs an SM 154 us, and 179 us where the grid is
// larger than what fits at a time.
__global__ void __launch_bounds__(kThreads, 6) reorder_kernel(const __grid_constant__ States a) {
  extern __shared__ __align__(16) char smem[];
  __shared__ int parent[kMostWidth];
  __shared__ unsigned long long needed;
  for (int64_t w = blockIdx.x; w < a.work; w += gridDim.x) {
    int e = 0;
    while (e + 1 < a.count && a.s[e + 1].first <= w) ++e;
    const State& s = a.s[e];
    const int64_t mine = w - s.first, g = mine / s.slices, slice = mine - g * s.slices, o = g / a.B, b = g - o * a.B;
    __syncthreads();
    if (threadIdx.x == 0) needed = 0;
    __syncthreads();
    for (int k = threadIdx.x; k < a.width; k += kThreads) {
      const int64_t p = a.parents[b * a.width + k];
      const bool moves = p >= 0 && p < a.K && !(s.in == s.out && p == k);
      parent[k] = moves ? (int)p : -1;
      if (moves) atomicOr(&needed, 1ull << p);
    }
    __syncthreads();
    switch (s.unit) {
      case 16: move<uint4>(s, slice, b, o, a, smem, parent, needed); break;
      case 8: move<uint2>(s, slice, b, o, a, smem, parent, needed); break;
      case 4: move<uint32_t>(s, slice, b, o, a, smem, parent, needed); break;
      case 2: move_halves(s, slice, b, o, a, smem, parent, needed); break;
      default: move<uint8_t>(s, slice, b, o, a, smem, parent, needed);
    }
  }
}

// CTAs of a group: enough that the groups give every SM three, and none with less than
// a round of its own.  (Groups of 4 rows of 50,000 bf16 columns with at least 1.5, 3 and 6
// CTAs an SM: 57 groups 18.5, 20.5 and 20.5 us, 100 20.7, 29.9 and 30.2, 128 28.9, 24.6 and
// 33.0, 200 33, 36 and 47, 228 47, 33 and 37, 456 60, 60 and 64; of 8 rows of 8192 fp32
// columns 57 20.7, 20.5 and 20.5, 128 32.8, 26.9 and 29.9, 228 55, 37 and 43.)
template <class T>
nmd_status launch_select(const Select& a, int64_t B, cudaStream_t s) {
  int cluster = 1;
  // Short rows go to warps, unless very many of their columns are wanted one by one
  const bool small = a.V <= kSmallRow && std::min<int64_t>(a.width, a.V) <= 48;
  while (!small && cluster < kMostCluster && B * cluster < 456 && a.K * a.V > (int64_t)cluster * 4 * kThreads * Vec<T>::N) cluster *= 2;
  const Shape shape = shape_of(a.K, a.width, cluster, small);
  static std::atomic<int> ready[kMaxDevices];
  auto kernel = select_kernel<T>;
  if (!per_device(ready, [&] {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    (int)shape_of(kMostBeams, kMostWidth, kMostCluster).bytes) == cudaSuccess;
      }))
    return NMD_ERR_CUDA;
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)cluster;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)(B * cluster));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = shape.bytes;
  cfg.stream = s;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, a, shape) == cudaSuccess ? NMD_OK : NMD_ERR_CUDA;
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
  const Select a{d_logits, V, ld, (int)K, (int)width, c, two_floats(1.0 / temperature), d_scores, d_finished, end,
                 d_out_scores, d_parents, d_tokens, d_out_finished};
  cudaStream_t s = (cudaStream_t)stream;
  if (dtype == NMD_DT_FP32) return launch_select<float>(a, B, s);
  return dtype == NMD_DT_BF16 ? launch_select<bf16>(a, B, s) : launch_select<__half>(a, B, s);
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
  *end++ = Range{(uintptr_t)d_parents, (uintptr_t)d_parents + (uintptr_t)(B * width * 8), kRead};
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
    Range taken[kStates];
    a.B = B;
    a.K = (int)K;
    a.width = (int)width;
    a.parents = d_parents;
    a.per = 16384;
    while (a.per > 512 && a.per * K > 32768) a.per /= 2;
    for (; k < count && a.count < kStates; ++k) {
      const nmd_beam_state& s = states[k];
      if (s.outer == 0 || s.bytes == 0 || B == 0) continue;
      // in place, states between each other's bytes go one after another
      int64_t reach = 0;
      rows_apart(s.outer, s.out_outer, B * width, s.out_row, s.bytes, &reach);
      const Range r{(uintptr_t)s.out, (uintptr_t)s.out + (uintptr_t)reach, kPlace};
      bool meets = false;
      for (int i = 0; i < a.count; ++i) meets |= r.from < taken[i].to && taken[i].from < r.to;
      if (meets) break;
      taken[a.count] = r;
      uintptr_t all = (uintptr_t)s.in | (uintptr_t)s.out | (uintptr_t)s.bytes | 16;
      if (B * K > 1) all |= (uintptr_t)s.in_row;
      if (B * width > 1) all |= (uintptr_t)s.out_row;
      if (s.outer > 1) all |= (uintptr_t)s.in_outer | (uintptr_t)s.out_outer;
      State& t = a.s[a.count++];
      t = State{(const char*)s.in, (char*)s.out, s.in_outer, s.out_outer, s.in_row, s.out_row, 0, 0, a.work,
                (int)(all & (~all + 1))};
      t.units = s.bytes / t.unit;
      t.slices = (s.bytes + a.per - 1) / a.per;
      a.work += t.slices * B * s.outer;
    }
    if (a.count == 0) break;
    reorder_kernel<<<(unsigned)std::min<int64_t>(a.work, 152 * 12), kThreads, (a.per + 4) * K, (cudaStream_t)stream>>>(a);
    if (cudaGetLastError() != cudaSuccess) return NMD_ERR_CUDA;
  }
  return NMD_OK;
}

}  // extern "C"

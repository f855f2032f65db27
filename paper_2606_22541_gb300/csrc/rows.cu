// Tokens sorted by expert and back, on plain tensors: the place of every (token,
// slot) in its expert's segment, rows to their places, weighted sums of rows back
// to the tokens, and the gradients of both.
#include "common.cuh"
#include "elem.cuh"
#include "rows.h"

#include <cuda_fp8.h>

#include <algorithm>
#include <atomic>

namespace asap {

namespace {

constexpr unsigned kFull = 0xffffffffu;

// ------------------------------------------------------------ sort
// place(i) = offsets[e_i] + #{i' < i : e_i' = e_i}.  A CTA ranks a chunk of up to 8
// entries a thread: a warp takes up to 256 that follow one another, 32 at a time; the
// lanes with one expert find each other (a vote per bit of its number: a match
// instruction takes about 40 clocks of the SM, nine votes 12), the lowest of them
// adds their number to the warp's counter, and the counter before it plus the
// lanes below is an entry's rank in its warp.  Counters are then summed over the
// warps.  No atomics, so a rank does not depend on any order of execution.
constexpr int kSortRounds = 8;  // at most

template <int THREADS>
struct SortShared {
  static constexpr int kWarps = THREADS / 32;
  uint16_t* before;  // [kWarps][pitch]: entries of an expert in the chunk's earlier warps
  int* total;        // [E] of an expert in the chunk
  int* first;        // [E] first place of the chunk's entries of an expert
  int* warp_sum;     // [kWarps]
  int pitch;
  static size_t bytes(int E) { return kWarps * 2 * ((E + 1) & ~1) + 8 * E + 4 * kWarps; }
  __device__ __forceinline__ SortShared(void* smem, int E) {
    pitch = (E + 1) & ~1;
    before = static_cast<uint16_t*>(smem);
    total = reinterpret_cast<int*>(before + kWarps * pitch);
    first = total + E;
    warp_sum = first + E;
  }
};

template <int THREADS>
__device__ __forceinline__ void rank_chunk(SortShared<THREADS>& s, const int32_t* idx, long long from, long long entries,
                                           int rounds, int E, int (&e)[kSortRounds], int (&rank)[kSortRounds]) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long at = from + warp * 32 * rounds + lane;
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    e[r] = r < rounds && at + 32 * r < entries ? ld_dep(idx + at + 32 * r) : -1;
    if (e[r] >= E || e[r] < 0) e[r] = -1;
  }
  uint16_t* mine = s.before + warp * s.pitch;
  for (int i = lane; i < s.pitch / 2; i += 32) reinterpret_cast<uint32_t*>(mine)[i] = 0;
  unsigned same[kSortRounds];  // lanes with this one's expert
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) same[r] = __ballot_sync(kFull, e[r] >= 0);
  for (int b = 1; b < E; b <<= 1) {
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
      if (r >= rounds) break;
      const unsigned set = __ballot_sync(kFull, e[r] & b);
      same[r] &= e[r] & b ? set : ~set;
    }
  }
  __syncwarp();
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    if (r >= rounds) break;
    const int below = __popc(same[r] & ((1u << lane) - 1));
    int had = 0;
    if (e[r] >= 0) had = mine[e[r]];
    __syncwarp();
    if (e[r] >= 0 && below == 0) mine[e[r]] = static_cast<uint16_t>(had + __popc(same[r]));
    __syncwarp();
    rank[r] = had + below;
  }
  __syncthreads();
  for (int x = threadIdx.x; x < E; x += THREADS) {
    int sum = 0;
#pragma unroll
    for (int w = 0; w < SortShared<THREADS>::kWarps; ++w) {
      const int c = s.before[w * s.pitch + x];
      s.before[w * s.pitch + x] = static_cast<uint16_t>(sum);
      sum += c;
    }
    s.total[x] = sum;
  }
  __syncthreads();
}

// s.first[x] = sum of all(x') over x' < x, plus lower(x), for x < E; offsets (nullable): the sums without lower, and the
// sum over all experts behind them.
template <int THREADS, typename F>
__device__ __forceinline__ void scan_experts(SortShared<THREADS>& s, int E, int32_t* offsets, F counts) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int carry = 0;
  for (int x0 = 0; x0 < E; x0 += THREADS) {
    const int x = x0 + threadIdx.x;
    const int2 c = x < E ? counts(x) : make_int2(0, 0);  // of all chunks, of lower ones
    int sum = c.x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(kFull, sum, o);
      if (lane >= o) sum += v;
    }
    if (lane == 31) s.warp_sum[warp] = sum;
    __syncthreads();
    int lower = carry, all = carry;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
      const int v = s.warp_sum[w];
      if (w < warp) lower += v;
      all += v;
    }
    if (x < E) {
      s.first[x] = lower + sum - c.x + c.y;
      if (offsets) offsets[x] = lower + sum - c.x;
    }
    carry = all;
    __syncthreads();
  }
  if (offsets && threadIdx.x == 0) offsets[E] = carry;
}

template <int THREADS>
__device__ __forceinline__ void write_places(const SortShared<THREADS>& s, long long from, long long entries,
                                             int rounds, int k, const int (&e)[kSortRounds],
                                             const int (&rank)[kSortRounds], int32_t* perm_dst, int32_t* perm_src) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const long long i = from + (warp * rounds + r) * 32 + lane;
    if (r >= rounds || i >= entries) continue;
    const int place = e[r] < 0 ? -1 : s.first[e[r]] + s.before[warp * s.pitch + e[r]] + rank[r];
    perm_dst[i] = place;
    if (perm_src && place >= 0) perm_src[place] = static_cast<int32_t>(i / k);
  }
}

// The whole sort in one cluster, a chunk a CTA; the chunks' counts are read from the CTAs' shared memory.
template <int THREADS>
__global__ void __launch_bounds__(THREADS)
    sort_cluster_kernel(const int32_t* idx, int entries, int rounds, int k, int E, int32_t* offsets, int32_t* perm_dst,
                        int32_t* perm_src) {
  extern __shared__ __align__(16) uint8_t smem[];
  SortShared<THREADS> s(smem, E);
  pdl_wait();
  pdl_launch();
  const int ranks = gridDim.x, rank_of = blockIdx.x;  // (one cluster)
  const long long from = static_cast<long long>(rank_of) * THREADS * rounds;
  int e[kSortRounds], rank[kSortRounds];
  rank_chunk(s, idx, from, entries, rounds, E, e, rank);
  if (ranks > 1) {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  }
  scan_experts(s, E, rank_of == 0 ? offsets : nullptr, [&](int x) {
    if (ranks == 1) return make_int2(s.total[x], 0);
    int v[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      v[r] = 0;
      if (r < ranks) {
        uint32_t peer;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(peer) : "r"(smem_u32(s.total + x)), "r"(r));
        asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v[r]) : "r"(peer) : "memory");
      }
    }
    int2 c = make_int2(0, 0);
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      c.x += v[r];
      if (r < rank_of) c.y += v[r];
    }
    return c;
  });
  if (ranks > 1) asm volatile("barrier.cluster.arrive.release;" ::: "memory");  // this CTA has read the others' counts
  write_places(s, from, entries, rounds, k, e, rank, perm_dst, perm_src);
  if (ranks > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}

// Many chunks: each one's counts (hist [chunk][E]); per expert, sums over the
// earlier chunks (in place) and over all (total [E]); places.  (Chunks of 4096: 0.6 to 0.8 us more up to 131072 entries, 6 less
// for 8.4 million.)
constexpr int kManyThreads = 256, kManyChunk = kManyThreads * kSortRounds;

__global__ void __launch_bounds__(kManyThreads)
    sort_count_kernel(const int32_t* idx, long long entries, int E, int32_t* hist) {
  __shared__ int count[kSortMaxExperts];
  pdl_wait();
  pdl_launch();
  for (int x = threadIdx.x; x < E; x += kManyThreads) count[x] = 0;
  __syncthreads();
  const long long from = static_cast<long long>(blockIdx.x) * kManyChunk;
  int e[kSortRounds];
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const long long i = from + r * kManyThreads + threadIdx.x;
    e[r] = i < entries ? ld_dep(idx + i) : -1;
  }
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r)
    if (e[r] >= 0 && e[r] < E) atomicAdd(&count[e[r]], 1);  // (a count: any order gives it)
  __syncthreads();
  for (int x = threadIdx.x; x < E; x += kManyThreads) hist[static_cast<long long>(blockIdx.x) * E + x] = count[x];
}

__global__ void __launch_bounds__(1024) sort_scan_kernel(int32_t* hist, int chunks, int E, int32_t* total) {
  __shared__ int part[32][33];
  pdl_wait();
  pdl_launch();
  const int x = blockIdx.x * 32 + (threadIdx.x & 31), w = threadIdx.x >> 5;
  const int c0 = static_cast<int>(static_cast<long long>(chunks) * w / 32);
  const int c1 = static_cast<int>(static_cast<long long>(chunks) * (w + 1) / 32);
  int sum = 0;
  if (x < E)
    for (int c = c0; c < c1; ++c) sum += ld_dep(hist + static_cast<long long>(c) * E + x);
  part[w][threadIdx.x & 31] = sum;
  __syncthreads();
  if (x >= E) return;
  int run = 0;
  for (int v = 0; v < w; ++v) run += part[v][threadIdx.x & 31];
  if (w == 31) total[x] = run + sum;
  for (int c = c0; c < c1; ++c) {
    int32_t* p = hist + static_cast<long long>(c) * E + x;
    const int v = *p;
    *p = run;
    run += v;
  }
}

__global__ void __launch_bounds__(kManyThreads)
    sort_place_kernel(const int32_t* idx, long long entries, int k, int E, const int32_t* hist, const int32_t* total,
                      int32_t* offsets, int32_t* perm_dst, int32_t* perm_src) {
  extern __shared__ __align__(16) uint8_t smem[];
  SortShared<kManyThreads> s(smem, E);
  pdl_wait();
  pdl_launch();
  const long long from = static_cast<long long>(blockIdx.x) * kManyChunk;
  int e[kSortRounds], rank[kSortRounds];
  rank_chunk(s, idx, from, entries, kSortRounds, E, e, rank);
  const int32_t* lower = hist + static_cast<long long>(blockIdx.x) * E;
  scan_experts(s, E, blockIdx.x == 0 ? offsets : nullptr,
               [&](int x) { return make_int2(ld_dep(total + x), ld_dep(lower + x)); });
  write_places(s, from, entries, kSortRounds, k, e, rank, perm_dst, perm_src);
}

// Entries of one cluster at most; below which one small CTA ranks them all; entries for each CTA of a cluster.  Measured
// with 256 experts, us: one CTA / a cluster / three kernels for 2048 entries 3.9 / 5.0 / -, 4096 5.2 / 6.0 / 6.2, 16384
// - / 6.2 / 6.7, 32768 - / 7.0 / 6.7 (one launch on the host instead of three), 65536 - / 9.0 / 6.7: bound by latency.
// Millions of entries are bound by the kernels' own work: 8.4 million take 62 us, the 101 MB that the three kernels move
// would take 15.  Alone they take 10 (count), 25 (scan: E / 32 CTAs, which read the counts twice) and 36 (votes and places).
constexpr long long kClusterEntries = 32768, kSmallEntries = 4096, kCtaEntries = 1024;
static_assert(kClusterEntries <= 8 * 1024 * kSortRounds && kSmallEntries <= 512 * kSortRounds, "entries of the launches");

// ------------------------------------------------------------ rows
// A row is taken by blockDim.x threads (8, 16 or whole warps), blockDim.y rows by a
// CTA; a thread has every blockDim.x-th unit (16 bytes) of its row.  With few rows the
// columns are spread over gridDim.y CTAs as well; with many a CTA takes rows in turn
// and has the next one's places on their way (the chain from a place to its row's
// loads is what these kernels wait for most).  A call of many wide rows is bound by
// HBM and moves its bytes at 0.94 to 0.97 of the copy rate:
//   permute 8045 tokens of 7168 bf16, k 8: 157 us, its bytes at the copy rate 152.7
//   unpermute 5185 of 7168 bf16, k 8: 104 (98.5)
//   gradients 4096 of 7168 bf16, k 8: 156 (147)
//   e4m3 rows of 4096 x 7168 read back, k 8: 77.5 (73.6)
// Calls of 10 to 50 us are at about 0.8, held up by that chain and the launch's ends:
//   unpermute 3584 of 4096 fp16, k 2: 15.5 (12.1); gradients 3584 of 4096, k 2: 26.7 (21.6)
// The gradients of narrow rows, whose next row has only its places ahead, at 0.34 to 0.67:
//   4431 of 1152 bf16, k 4: 20.3 (13.6); 4044 of 272, k 3: 6.2 (2.3); 5994 of 144, k 5: 8.3 (2.9)
// 16-bit rows that do not start on 8 bytes are shifted into place (struct Any), with two
// loads for every 16 bytes, 0.45 to 0.55 for sums and gradients:
//   unpermute 3780 of 4401 bf16, k 7: 73 us (39), with 2-byte accesses 155, in 4-byte words 268;
//   14762 of 2254, k 7: 142 (78); gradients of those: 268 (147); 3406 of 1909, k 7: 63 (29)
// fp32 rows, which need no shifts, go by 4 bytes with more of them on their way: 3780 of
// 4401, k 7: 107 (78), shifted 16 bytes 155.
constexpr int kRowThreads = 256;
constexpr int kSms = 152;
constexpr int kFewCtas = kSms * 4;  // below this many CTAs a call is short of work
// Of a CTA of the kernels that wait for several rows: more CTAs an SM, so that some
// always have loads out (256, 128 and 64 threads, us: unpermute 12900 of 1792, k 6 56,
// 54, 56; gradients 3584 of 4096, k 2 30, 27, 28).
constexpr int kSumThreads = 128;
// CTAs of a grid at most, in waves of as many as the SMs hold.  A part of a wave more
// costs most (unpermute 3584 of 4096, k 2: 16.2 us in one wave, 17.0 in two, 19.2 in one
// and a half); copies, whose CTAs differ more in their pace, gain from more waves
// (permute 8045 of 7168, k 8 with 1, 2, 4, 8: 178, 166, 161, 157; gradients 4096 of 7168
// with 1, 2, 4: 164, 165, 155).
constexpr int kCopyWaves = 8, kSumWaves = 1, kAnySumWaves = 2, kGradWaves = 4;

// Rows of a CTA: first_row() + threadIdx.y, and gridDim.x blockDim.y further on.
__device__ __forceinline__ long long first_row() { return static_cast<long long>(blockIdx.x) * blockDim.y; }
// Lanes of a warp that share a row.
__device__ __forceinline__ int team_width() { return min(32, static_cast<int>(blockDim.x)); }

// The place of entry (t, j) for the team's lane j, -1 where there is none (a place
// that is no row of y is recorded).  All lanes of a warp call it.
__device__ __forceinline__ int place_of(const RowsArgs& a, long long t, int j, bool wanted) {
  if (!wanted || t >= a.n || j >= a.k) return -1;
  int p = ld_dep(a.perm + t * a.k + j);
  if (p < 0 || p >= a.rows) {
    if (p != -1 && threadIdx.x < 32 && blockIdx.y == 0) record_status(a.status, ST_BAD_POSITION);
    p = -1;
  }
  return p;
}

__device__ __forceinline__ uint4 load_unit(const uint4* p) { return ld_dep(p); }
template <typename U>
__device__ __forceinline__ U load_unit(const U* p) {
  return *const_cast<const volatile U*>(p);
}

// x_perm[place] = x[t]: rows that start on 16 bytes, in units of 16, the last few bytes of a row one by one.
// A thread has its next units (and the next row's places) on their way while it stores those it has.
constexpr int kCopyUnits = 4;
__global__ void __launch_bounds__(kRowThreads)
    permute_kernel(const char* x, long long ldx, char* __restrict__ y, long long ldy, long long row_bytes,
                   const RowsArgs a) {
  pdl_wait();
  pdl_launch();
  const int width = team_width(), lane = threadIdx.x & (width - 1);
  using U = uint4;
  const int units = static_cast<int>(row_bytes / static_cast<int>(sizeof(U)));
  const int rest = static_cast<int>(row_bytes - static_cast<long long>(units) * sizeof(U));
  const int start = blockIdx.y * blockDim.x * kCopyUnits;
  const int step = gridDim.y * blockDim.x * kCopyUnits, rows = gridDim.x * blockDim.y;
  long long base = first_row();
  int v0 = start;  // (both the same in the CTA)
  U next[kCopyUnits];
  int next_place;
  auto fetch = [&]() {
    const long long t = base + threadIdx.y;
    if (v0 == start) next_place = place_of(a, t, lane, true);
    const U* row = reinterpret_cast<const U*>(x + t * ldx);
#pragma unroll
    for (int i = 0; i < kCopyUnits; ++i) {
      const int v = v0 + static_cast<int>(i * blockDim.x + threadIdx.x);
      if (t < a.n && v < units) next[i] = load_unit(row + v);
    }
  };
  auto put = [&](int mine, int places, int at, const U (&u)[kCopyUnits]) {
    for (int j = 0; j < places; ++j) {
      const int p = __shfl_sync(kFull, mine, j, width);
      if (p < 0) continue;
      U* to = reinterpret_cast<U*>(y + p * ldy);
#pragma unroll
      for (int i = 0; i < kCopyUnits; ++i) {
        const int v = at + static_cast<int>(i * blockDim.x + threadIdx.x);
        if (v < units) to[v] = u[i];
      }
    }
  };
  auto put_rest = [&](long long t, int mine, int places) {
    for (int j = 0; j < places; ++j) {
      const int p = __shfl_sync(kFull, mine, j, width);
      if (p < 0) continue;
      for (int b = threadIdx.x; b < rest; b += blockDim.x) {
        const long long at = static_cast<long long>(units) * sizeof(U) + b;
        y[p * ldy + at] = load_unit(x + t * ldx + at);
      }
    }
  };
  int mine = -1;
  if (base < a.n) fetch();
  while (base < a.n) {
    U u[kCopyUnits];
#pragma unroll
    for (int i = 0; i < kCopyUnits; ++i) u[i] = next[i];
    const long long t = base + threadIdx.y;
    const int at = v0;
    if (at == start) mine = next_place;
    v0 += step;
    if (v0 >= units) v0 = start, base += rows;
    if (base < a.n) fetch();
    put(mine, min(width, a.k), at, u);
    const bool last = rest > 0 && at == start && blockIdx.y == 0;
    if (last) put_rest(t, mine, min(width, a.k));
    for (int j0 = width; j0 < a.k; j0 += width) {  // more places than lanes
      const int more = place_of(a, t, j0 + lane, true), places = min(width, a.k - j0);
      put(more, places, at, u);
      if (last) put_rest(t, more, places);
    }
  }
}

// The same for rows at any address.  T: an element.  A thread has the aligned 16 bytes of x and those before them; a
// place's row takes 16 of these 32 for an aligned store.
constexpr int kAnyUnits = 2;  // of a thread on their way
template <typename T>
__global__ void __launch_bounds__(kRowThreads)
    permute_any_kernel(const T* x, long long ldx, T* __restrict__ y, long long ldy, const RowsArgs a) {
  using A = Any<T>;
  constexpr int C = kAnyUnits;
  pdl_wait();
  pdl_launch();
  const int width = team_width(), lane = threadIdx.x & (width - 1);
  const int start = blockIdx.y * blockDim.x * C * A::N;
  const int step = gridDim.y * blockDim.x * C * A::N, rows = gridDim.x * blockDim.y;
  for (long long base = first_row(); base < a.n; base += rows) {
    const long long t = base + threadIdx.y;
    const T* row = x + t * ldx;
    const int from = A::past(row);
    for (int j0 = 0; j0 < a.k; j0 += width) {
      const int mine = place_of(a, t, j0 + lane, true), places = min(width, a.k - j0);
      for (int c0 = start; c0 < a.cols + 2 * A::N; c0 += step) {
        typename A::V lo[C], hi[C];
#pragma unroll
        for (int i = 0; i < C; ++i) {
          if (t >= a.n) continue;
          const int c = c0 + static_cast<int>((i * blockDim.x + threadIdx.x) * A::N) - from;
          const typename A::Raw r = A::fetch(row, c - A::N, a.cols);
          lo[i] = r.lo, hi[i] = r.hi;
        }
        for (int j = 0; j < places; ++j) {
          const int p = __shfl_sync(kFull, mine, j, width);
          if (p < 0) continue;
          T* to = y + p * ldy;
          // the byte of the 32 that comes to a boundary: 1 .. 16
          const int o = (((from - A::past(to)) * A::kSize - 1) & 15) + 1;
#pragma unroll
          for (int i = 0; i < C; ++i) {
            const int c = c0 + static_cast<int>((i * blockDim.x + threadIdx.x) * A::N) - from - A::N + o / A::kSize;
            if (c + A::N > 0 && c < a.cols) A::store(to, c, a.cols, A::shifted(lo[i], hi[i], o));
          }
        }
      }
    }
  }
}

constexpr int kSumCtas = 4;  // CTAs of kRowThreads an SM that the registers are kept to
// out[t] = sum_j w[t][j] y[place], fp32 in slot order; J places and C units of N
// columns at a time.
// ANY: rows at any address, N columns as out's row has them on 16 bytes.
template <typename T, int N, int J, int C, bool ANY>
__global__ void __launch_bounds__(kRowThreads, ANY ? 3 : kSumCtas)
    unpermute_kernel(const T* y, long long ldy, T* __restrict__ out, long long ldo, const RowsArgs a) {
  pdl_wait();
  pdl_launch();
  const int width = team_width(), lane = threadIdx.x & (width - 1);
  const int start = blockIdx.y * blockDim.x * C * N;
  const int step = gridDim.y * blockDim.x * C * N, rows = gridDim.x * blockDim.y;
  int next_place;
  float next_w;
  auto fetch = [&](long long t, int j0) {  // places and weights, by lane
    next_place = place_of(a, t, j0 + lane, lane < J);
    next_w = a.w && next_place >= 0 ? ld_dep(a.w + t * a.k + j0 + lane) : 1.f;
  };
  long long base = first_row();
  if (base < a.n) fetch(base + threadIdx.y, 0);
  for (; base < a.n; base += rows) {
    const long long t = base + threadIdx.y;
    int mine = next_place;
    float wt = next_w;
    if (base + rows < a.n) fetch(t + rows, 0);
    const int pre = ANY ? Any<T>::past(out + t * ldo) : 0;
    for (int c0 = start; c0 < a.cols + (ANY ? N : 0); c0 += step) {
      float acc[C][N];
#pragma unroll
      for (int i = 0; i < C; ++i)
#pragma unroll
        for (int q = 0; q < N; ++q) acc[i][q] = 0.f;
      for (int j0 = 0; j0 < a.k; j0 += J) {
        if (a.k > J) {  // more places than are handled together
          const int keep_place = next_place;
          const float keep_w = next_w;
          fetch(t, j0);
          mine = next_place, wt = next_w;
          next_place = keep_place, next_w = keep_w;
        }
        std::conditional_t<ANY, typename Any<T>::Raw, Cols<T, N>> v[J][C];
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const int p = __shfl_sync(kFull, mine, j, width);
          const T* from = y + p * ldy;
#pragma unroll
          for (int i = 0; i < C; ++i) {
            const int c = c0 + static_cast<int>((i * blockDim.x + threadIdx.x) * N) - pre;
            if (p < 0 || c >= a.cols) continue;
            if constexpr (ANY)
              v[j][i] = Any<T>::fetch(from, c, a.cols);
            else
              v[j][i].load(from + c, a.cols - c);
          }
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const int p = __shfl_sync(kFull, mine, j, width);
          const float w = __shfl_sync(kFull, wt, j, width);
          if (p >= 0) {
#pragma unroll
            for (int i = 0; i < C; ++i) {
              float f[N];
              if constexpr (ANY)
                Any<T>::columns(v[j][i], y + p * ldy, c0 + static_cast<int>((i * blockDim.x + threadIdx.x) * N) - pre).to(f);
              else
                v[j][i].to(f);
#pragma unroll
              for (int q = 0; q < N; ++q) acc[i][q] = fmaf(w, f[q], acc[i][q]);
            }
          }
        }
      }
#pragma unroll
      for (int i = 0; i < C; ++i) {
        const int c = c0 + static_cast<int>((i * blockDim.x + threadIdx.x) * N) - pre;
        if (t >= a.n || c >= a.cols) continue;
        Cols<T, N> o;
        o.from(acc[i]);
        if constexpr (ANY)
          Any<T>::store(out + t * ldo, c, a.cols, o);
        else
          o.store(out + t * ldo + c, a.cols - c);
      }
    }
  }
}

// Threads of a CTA of the gradients at most.  (Few rows have their laps side by side, 8 tokens of 7168 6.2 us instead of
// 10.4; 1024 threads limit the kernel to 64 registers, and where these are too few CTAs stay small.)
constexpr int kGradThreads = 1024;
template <typename T, int J, bool ANY>
constexpr int grad_threads = ANY || (J == 8 && std::is_same_v<T, __half>) ? kRowThreads : kGradThreads;
// d_y[place] = w d_out[t], d_w[t][j] = <d_out[t], y[place]> (fp32: per thread, then
// over the lanes and the row's warps in a fixed tree).
// ANY: rows at any address, N columns as each row of d_y (of y without it) has them on 16 bytes.
template <typename T, int N, int J, bool ANY>
__global__ void __launch_bounds__(grad_threads<T, J, ANY>, grad_threads<T, J, ANY> == kRowThreads ? 3 : 1)
    unpermute_backward_kernel(const T* d_out, long long ldo, const T* y, long long ldy, T* __restrict__ d_y, long long ldd,
                              float* __restrict__ d_w, const RowsArgs a) {
  __shared__ float part[2][kGradThreads / 32][J];
  pdl_wait();
  pdl_launch();
  const int width = team_width(), lane = threadIdx.x & (width - 1);
  const int warps = blockDim.x / 32, warp = (threadIdx.y * blockDim.x + threadIdx.x) / 32;
  const unsigned rows = gridDim.x * blockDim.y;
  int next_place, turn = 0;
  float next_w;
  long long base = first_row();
  int j0 = 0;
  auto fetch = [&](long long t) {
    next_place = place_of(a, t, j0 + lane, lane < J);
    next_w = a.w && next_place >= 0 ? ld_dep(a.w + t * a.k + j0 + lane) : 1.f;
  };
  if (base < a.n) fetch(base + threadIdx.y);
  while (base < a.n) {
    const long long t = base + threadIdx.y;
    const bool live = t < a.n;
    const int mine = next_place, jt = j0;
    const float wt = next_w;
    j0 += J;
    if (j0 >= a.k) j0 = 0, base += rows;
    if (base < a.n) fetch(base + threadIdx.y);
    float s[J];
#pragma unroll
    for (int j = 0; j < J; ++j) s[j] = 0.f;
    const T* d_row = d_out + t * ldo;
    // (whole warps: they exchange places in the loop)
    for (int c0 = 0; c0 < a.cols + (ANY ? N : 0); c0 += blockDim.x * N) {
      const int ct = c0 + static_cast<int>(threadIdx.x) * N;
      std::conditional_t<ANY, typename Any<T>::Raw, Cols<T, N>> v[J];
      Cols<T, N> d, d_lo;  // (d_lo: the N columns before d's)
      if constexpr (ANY) {
        if (live) {
          const auto hi = Any<T>::fetch(d_row, ct, a.cols), lo = Any<T>::fetch(d_row, ct - N, a.cols);
          d = Any<T>::columns(hi, d_row, ct);
          d_lo = Any<T>::columns(lo, d_row, ct - N);
        }
      } else if (live && ct < a.cols) {
        d.load(d_row + ct, a.cols - ct);
      }
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int p = __shfl_sync(kFull, mine, j, width);
        if (!d_w || p < 0) continue;
        const T* from = y + p * ldy;
        if constexpr (ANY)
          v[j] = Any<T>::fetch(from, ct - Any<T>::past(d_y ? d_y + p * ldd : from), a.cols);
        else if (ct < a.cols)
          v[j].load(from + ct, a.cols - ct);
      }
      float g[N];
      if (!ANY) d.to(g);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int p = __shfl_sync(kFull, mine, j, width);
        const float w = __shfl_sync(kFull, wt, j, width);
        if (p < 0) continue;  // (as are all of a row that is not there)
        T* to = d_y + p * ldd;
        int pre = 0;
        if constexpr (ANY) {
          pre = Any<T>::past(d_y ? to : y + p * ldy);
          Any<T>::before(d_lo, d, pre).to(g);
        }
        const int c = ct - pre;
        if (c >= a.cols) continue;
        float f[N];
        if (d_y) {
#pragma unroll
          for (int i = 0; i < N; ++i) f[i] = w * g[i];
          Cols<T, N> o;
          o.from(f);
          if constexpr (ANY)
            Any<T>::store(to, c, a.cols, o);
          else
            o.store(to + c, a.cols - c);
        }
        if (d_w) {
          if constexpr (ANY)
            Any<T>::columns(v[j], y + p * ldy, c).to(f);
          else
            v[j].to(f);
          if (ANY && (c < 0 || c + N > a.cols)) {  // (beside the row there may be anything)
#pragma unroll
            for (int i = 0; i < N; ++i)
              if (c + i < 0 || c + i >= a.cols) f[i] = 0.f, g[i] = 0.f;
          }
#pragma unroll
          for (int i = 0; i < N; ++i) s[j] = fmaf(g[i], f[i], s[j]);
        }
      }
    }
    if (!d_w) continue;
#pragma unroll
    for (int j = 0; j < J; ++j)
      for (int o = width / 2; o > 0; o >>= 1) s[j] += __shfl_xor_sync(kFull, s[j], o);
    if (warps > 1) {
      // (two copies in turn: a warp that writes one again has passed the barrier after which the other was read)
      if (lane == 0) {
#pragma unroll
        for (int j = 0; j < J; ++j) part[turn][warp][j] = s[j];
      }
      __syncthreads();
      if (live && threadIdx.x < J && jt + static_cast<int>(threadIdx.x) < a.k) {
        float sum = 0.f;
        for (int v = 0; v < warps; ++v) sum += part[turn][warp + v][threadIdx.x];
        d_w[t * a.k + jt + threadIdx.x] = sum;
      }
      turn ^= 1;
    } else if (live) {
#pragma unroll
      for (int j = 0; j < J; ++j)
        if (lane == j && jt + j < a.k) d_w[t * a.k + jt + j] = s[j];
    }
  }
}

// y[place] = scale q[t], N columns at a time (a scale per 128).
constexpr int kDecodeUnits = 2;  // of a thread
template <typename T, int N>
__global__ void __launch_bounds__(kRowThreads)
    dequantize_kernel(const uint8_t* q, long long ldq, const float* scales, long long lds, T* __restrict__ y, long long ldy,
                      const RowsArgs a) {
  pdl_wait();
  pdl_launch();
  const int width = team_width(), lane = threadIdx.x & (width - 1);
  const int start = blockIdx.y * blockDim.x * kDecodeUnits * N;
  const int step = gridDim.y * blockDim.x * kDecodeUnits * N, rows = gridDim.x * blockDim.y;
  long long base = first_row();
  int c0 = start;  // (both the same in the CTA)
  // the next units and their scales, the next row's places
  uint32_t b[kDecodeUnits][(N + 3) / 4];
  float s[kDecodeUnits];
  int next_place;
  auto fetch = [&]() {
    const long long t = base + threadIdx.y;
    if (c0 == start)
      next_place = a.perm ? place_of(a, t, lane, true) : lane == 0 && t < a.n ? static_cast<int>(t) : -1;
#pragma unroll
    for (int i = 0; i < kDecodeUnits; ++i) {
      const int c = c0 + static_cast<int>((i * blockDim.x + threadIdx.x) * N);
      s[i] = 0.f;
#pragma unroll
      for (int k = 0; k < (N + 3) / 4; ++k) b[i][k] = 0;
      if (t >= a.n || c >= a.cols) continue;
      const int left = a.cols - c;
      const uint8_t* from = q + t * ldq + c;
      s[i] = ld_dep(scales + t * lds + (c >> 7));
      if (N >= 4 && left >= N) {
        if constexpr (N == 8)
          asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(b[i][0]), "=r"(b[i][1]) : "l"(from));
        else
          asm volatile("ld.global.b32 %0, [%1];" : "=r"(b[i][0]) : "l"(from));
      } else {
#pragma unroll
        for (int k = 0; k < N; ++k)
          if (k < left) b[i][k / 4] |= static_cast<uint32_t>(load_unit(from + k)) << (8 * (k & 3));
      }
    }
  };
  auto put = [&](int mine, int places, int at, const Cols<T, N> (&o)[kDecodeUnits]) {
    for (int j = 0; j < places; ++j) {
      const int p = __shfl_sync(kFull, mine, j, width);
      if (p < 0) continue;
#pragma unroll
      for (int i = 0; i < kDecodeUnits; ++i) {
        const int c = at + static_cast<int>((i * blockDim.x + threadIdx.x) * N);
        if (c < a.cols) o[i].store(y + p * ldy + c, a.cols - c);
      }
    }
  };
  int mine = -1;
  if (base < a.n) fetch();
  while (base < a.n) {
    Cols<T, N> o[kDecodeUnits];
#pragma unroll
    for (int i = 0; i < kDecodeUnits; ++i) {
      float f[N];
#pragma unroll
      for (int k = 0; k < N; ++k)
        f[k] = s[i] * __half2float(__half(__nv_cvt_fp8_to_halfraw(static_cast<uint8_t>(b[i][k / 4] >> (8 * (k & 3))),
                                                                 __NV_E4M3)));
      o[i].from(f);
    }
    const long long t = base + threadIdx.y;
    const int at = c0;
    if (at == start) mine = next_place;
    c0 += step;
    if (c0 >= a.cols) c0 = start, base += rows;
    if (base < a.n) fetch();
    put(mine, min(width, a.k), at, o);
    for (int j0 = width; j0 < a.k; j0 += width)  // more places than lanes
      put(place_of(a, t, j0 + lane, true), min(width, a.k - j0), at, o);
  }
}

// N e4m3 values and their scales as columns c .. c + N - 1 of y's type, zeros outside the row.
template <typename T>
__device__ __forceinline__ Cols<T, Any<T>::N> decode_any(const uint8_t* q, const float* scales, int c, int cols) {
  constexpr int N = Any<T>::N;
  float f[N];
  if (c >= 0 && c + N <= cols) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(q + c), first = at & ~static_cast<uintptr_t>(7);
    const int o = static_cast<int>(at & 7);
    uint64_t b, next = 0;
    asm volatile("ld.global.b64 %0, [%1];" : "=l"(b) : "l"(first));
    if (o + N > 8) asm volatile("ld.global.b64 %0, [%1];" : "=l"(next) : "l"(first + 8));
    if (o) b = b >> (8 * o) | next << (64 - 8 * o);
    const float s = ld_dep(scales + (c >> 7));  // (c is a multiple of N: one scale)
#pragma unroll
    for (int i = 0; i < N; ++i)
      f[i] = s * __half2float(__half(__nv_cvt_fp8_to_halfraw(static_cast<uint8_t>(b >> (8 * i)), __NV_E4M3)));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      f[i] = 0.f;
      if (c + i >= 0 && c + i < cols)
        f[i] = ld_dep(scales + ((c + i) >> 7)) * __half2float(__half(__nv_cvt_fp8_to_halfraw(load_unit(q + c + i), __NV_E4M3)));
    }
  }
  Cols<T, N> v;
  v.from(f);
  return v;
}

// The same for rows at any address: a thread has N columns and the N before them; a place's row takes N of these for an
// aligned store.
template <typename T>
__global__ void __launch_bounds__(kRowThreads)
    dequantize_any_kernel(const uint8_t* q, long long ldq, const float* scales, long long lds, T* __restrict__ y,
                          long long ldy, const RowsArgs a) {
  using A = Any<T>;
  constexpr int C = kAnyUnits;
  pdl_wait();
  pdl_launch();
  const int width = team_width(), lane = threadIdx.x & (width - 1);
  const int start = blockIdx.y * blockDim.x * C * A::N;
  const int step = gridDim.y * blockDim.x * C * A::N, rows = gridDim.x * blockDim.y;
  for (long long base = first_row(); base < a.n; base += rows) {
    const long long t = base + threadIdx.y;
    for (int j0 = 0; j0 < a.k; j0 += width) {
      const int mine = a.perm ? place_of(a, t, j0 + lane, true) : lane == 0 && t < a.n ? static_cast<int>(t) : -1;
      const int places = min(width, a.k - j0);
      for (int c0 = start; c0 < a.cols + A::N; c0 += step) {
        typename A::V lo[C], hi[C];
#pragma unroll
        for (int i = 0; i < C; ++i) {
          const int c = c0 + static_cast<int>((i * blockDim.x + threadIdx.x) * A::N), cols = t < a.n ? a.cols : 0;
          hi[i] = decode_any<T>(q + t * ldq, scales + t * lds, c, cols);
          lo[i] = decode_any<T>(q + t * ldq, scales + t * lds, c - A::N, cols);
        }
        for (int j = 0; j < places; ++j) {
          const int p = __shfl_sync(kFull, mine, j, width);
          if (p < 0) continue;
          T* to = y + p * ldy;
          const int pre = A::past(to);
#pragma unroll
          for (int i = 0; i < C; ++i) {
            const int c = c0 + static_cast<int>((i * blockDim.x + threadIdx.x) * A::N) - pre;
            if (c < a.cols) A::store(to, c, a.cols, A::before(lo[i], hi[i], pre));
          }
        }
      }
    }
  }
}

// CTAs of this many threads that an SM holds (asked once: the library runs on one kind of GPU).
template <auto KERNEL>
int resident(int threads) {
  static std::atomic<int> known[kGradThreads / 32 + 1];
  std::atomic<int>& k = known[threads / 32];
  int v = k.load(std::memory_order_relaxed);
  if (v == 0) {
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&v, KERNEL, threads, 0) != cudaSuccess || v < 1) {
      cudaGetLastError();
      return 1;
    }
    k.store(v, std::memory_order_relaxed);
  }
  return v;
}

// Threads and CTAs for n rows of ``units`` units, C of them a thread at a time: as
// few threads as a row needs, in equal laps where it needs more than a CTA has;
// laps side by side (split) while the rows alone would leave SMs without work.  CTAs of
// ``waves`` full waves at most, which then take more rows in turn.
struct RowLaunch {
  dim3 grid, block;
};
template <auto KERNEL>
RowLaunch row_launch(long long n, long long units, int C, bool split, int most, int waves) {
  const long long need = std::max<long long>(1, (units + C - 1) / C);
  const long long laps = (need + most - 1) / most;
  const long long per = (need + laps - 1) / laps;
  const int x = per <= 8 ? 8 : per <= 16 ? 16 : static_cast<int>((per + 31) / 32 * 32);
  const int y = std::max(1, std::min(most, kRowThreads) / x);
  const long long ctas = (n + y - 1) / y;
  dim3 grid(static_cast<unsigned>(ctas), 1);
  if (split && ctas < kFewCtas) grid.y = static_cast<unsigned>(std::min<long long>(laps, 64));
  if (ctas > kFewCtas) grid.x = static_cast<unsigned>(std::min<long long>(ctas, 1ll * kSms * resident<KERNEL>(x * y) * waves));
  return {grid, dim3(x, y)};
}

template <typename F>
cudaError_t by_type(int type, F f) {
  switch (type) {
    case kElemBf16: return f(__nv_bfloat16{});
    case kElemF16: return f(__half{});
    case kElemF32: return f(0.f);
    default: return cudaErrorInvalidValue;
  }
}
// Bytes an access where every row of T starts on as many (at: addresses and strides in bytes): 16, 8, or those of a word;
// else 0.
template <typename T, typename F>
cudaError_t by_alignment(uintptr_t at, F f) {
  if (at % 16 == 0) return f(std::integral_constant<int, 16>{});
  if (at % 8 == 0) return f(std::integral_constant<int, 8>{});
  return f(std::integral_constant<int, sizeof(T) == 4 ? 4 : 0>{});
}
// Units of a thread for accesses of this many bytes and J places: as many bytes on their way.
constexpr int units_of(int access, int J) {
  return access == 0 ? 1 : access == 16 ? (J >= 4 ? 1 : 2) : access == 8 ? (J >= 8 ? 1 : 2) : (J >= 8 ? 2 : 4);
}

// Places handled together.
template <typename F>
cudaError_t by_places(int k, F f) {
  if (k == 1) return f(std::integral_constant<int, 1>{});
  if (k == 2) return f(std::integral_constant<int, 2>{});
  if (k <= 4) return f(std::integral_constant<int, 4>{});
  return f(std::integral_constant<int, 8>{});
}

uintptr_t bits(const void* p) { return reinterpret_cast<uintptr_t>(p); }

}  // namespace

size_t sort_workspace(long long entries, int experts) {
  if (entries <= kClusterEntries) return 0;
  return static_cast<size_t>(ceil_div(entries, kManyChunk) + 1) * experts * 4;
}

namespace {
template <int THREADS>
cudaError_t sort_cluster(int ctas, const int32_t* idx, int entries, int k, int E, int32_t* offsets, int32_t* perm_dst,
                         int32_t* perm_src, cudaStream_t s) {
  const size_t smem = SortShared<THREADS>::bytes(E);
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(sort_cluster_kernel<THREADS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               static_cast<int>(smem));
    if (e != cudaSuccess) return e;
  }
  const int rounds = std::max(1, ceil_div(entries, ctas * THREADS));
  return launch_pdl(sort_cluster_kernel<THREADS>, ctas, THREADS, smem, s, ctas, idx, entries, rounds, k, E, offsets, perm_dst,
                    perm_src);
}
}  // namespace

cudaError_t launch_sort(const int32_t* idx, long long entries, int k, int E, int32_t* offsets, int32_t* perm_dst,
                        int32_t* perm_src, void* ws, cudaStream_t s) {
  if (entries <= kSmallEntries)
    return sort_cluster<512>(1, idx, static_cast<int>(entries), k, E, offsets, perm_dst, perm_src, s);
  if (entries <= kClusterEntries) {
    const int ctas = std::min(8, ceil_div(entries, kCtaEntries));
    return sort_cluster<1024>(ctas, idx, static_cast<int>(entries), k, E, offsets, perm_dst, perm_src, s);
  }
  const int chunks = ceil_div(entries, kManyChunk);
  int32_t* total = static_cast<int32_t*>(ws);
  int32_t* hist = total + E;
  cudaError_t e = launch_pdl(sort_count_kernel, chunks, kManyThreads, 0, s, 1, idx, entries, E, hist);
  if (e == cudaSuccess) e = launch_pdl(sort_scan_kernel, ceil_div(E, 32), 1024, 0, s, 1, hist, chunks, E, total);
  if (e == cudaSuccess)
    e = launch_pdl(sort_place_kernel, chunks, kManyThreads, SortShared<kManyThreads>::bytes(E), s, 1, idx, entries, k, E, hist,
                   total, offsets, perm_dst, perm_src);
  return e;
}

cudaError_t launch_permute(int elem_bytes, const void* x, long long ldx, void* y, long long ldy, const RowsArgs& a,
                           cudaStream_t s) {
  const uintptr_t at = bits(x) | bits(y) | static_cast<uintptr_t>((ldx | ldy) * elem_bytes);
  const long long bytes = static_cast<long long>(a.cols) * elem_bytes;
  if (at % 16 == 0 && bytes >= 16) {
    const RowLaunch r = row_launch<permute_kernel>(a.n, bytes / 16, kCopyUnits, true, kRowThreads, kCopyWaves);
    return launch_pdl(permute_kernel, r.grid, r.block, 0, s, 1, static_cast<const char*>(x), ldx * elem_bytes,
                      static_cast<char*>(y), ldy * elem_bytes, bytes, a);
  }
  auto any = [&](auto elem) {
    using T = decltype(elem);
    const RowLaunch r = row_launch<permute_any_kernel<T>>(a.n, bytes / 16 + 2, kAnyUnits, true, kRowThreads, kCopyWaves);
    return launch_pdl(permute_any_kernel<T>, r.grid, r.block, 0, s, 1, static_cast<const T*>(x), ldx, static_cast<T*>(y), ldy,
                      a);
  };
  return elem_bytes == 4 ? any(uint32_t{}) : elem_bytes == 2 ? any(uint16_t{}) : any(uint8_t{});
}

cudaError_t launch_unpermute(int type, const void* y, long long ldy, void* out, long long ldo, const RowsArgs& a,
                             cudaStream_t s) {
  return by_type(type, [&](auto t) {
    using T = decltype(t);
    return by_alignment<T>(bits(y) | bits(out) | static_cast<uintptr_t>((ldy | ldo) * sizeof(T)), [&](auto access) {
      return by_places(a.k, [&](auto places) {
        constexpr bool ANY = decltype(access)::value == 0;
        constexpr int N = (ANY ? 16 : decltype(access)::value) / static_cast<int>(sizeof(T));
        constexpr int J = ANY ? std::min(4, decltype(places)::value) : decltype(places)::value;  // (registers)
        constexpr int C = units_of(decltype(access)::value, J);
        const RowLaunch r = row_launch<unpermute_kernel<T, N, J, C, ANY>>(
            a.n, ceil_div(a.cols, N) + ANY, C, true, ANY ? kRowThreads : kSumThreads, ANY ? kAnySumWaves : kSumWaves);
        return launch_pdl(unpermute_kernel<T, N, J, C, ANY>, r.grid, r.block, 0, s, 1, static_cast<const T*>(y), ldy,
                          static_cast<T*>(out), ldo, a);
      });
    });
  });
}

cudaError_t launch_unpermute_backward(int type, const void* d_out, long long ldo, const void* y, long long ldy, void* d_y,
                                      long long ldd, float* d_w, const RowsArgs& a, cudaStream_t s) {
  return by_type(type, [&](auto t) {
    using T = decltype(t);
    uintptr_t at = bits(d_out) | bits(y) | bits(d_y) | static_cast<uintptr_t>(ldo * sizeof(T));
    if (d_w) at |= static_cast<uintptr_t>(ldy * sizeof(T));
    if (d_y) at |= static_cast<uintptr_t>(ldd * sizeof(T));
    if (a.cols == 0) at = 0;  // (sums of nothing: no row is touched)
    return by_alignment<T>(at, [&](auto access) {
      return by_places(a.k, [&](auto places) {
        constexpr bool ANY = decltype(access)::value == 0;
        constexpr int N = (ANY ? 16 : decltype(access)::value) / static_cast<int>(sizeof(T));
        constexpr int J = ANY ? std::min(4, decltype(places)::value) : decltype(places)::value;  // (registers)
        // (a row's sums meet in its CTA: few rows have wide ones)
        const int threads = a.n <= kSms ? grad_threads<T, J, ANY> : a.n <= kFewCtas ? kRowThreads : kSumThreads;
        const RowLaunch r = row_launch<unpermute_backward_kernel<T, N, J, ANY>>(a.n, ceil_div(a.cols, N) + ANY, 1, false,
                                                                                threads, kGradWaves);
        return launch_pdl(unpermute_backward_kernel<T, N, J, ANY>, r.grid, r.block, 0, s, 1, static_cast<const T*>(d_out),
                          ldo, static_cast<const T*>(y), ldy, static_cast<T*>(d_y), ldd, d_w, a);
      });
    });
  });
}

cudaError_t launch_dequantize(int type, const void* q, long long ldq, const float* scales, long long lds, void* y,
                              long long ldy, const RowsArgs& a, cudaStream_t s) {
  return by_type(type, [&](auto t) {
    using T = decltype(t);
    // (rows of q start on N bytes where rows of y start on 16)
    const uintptr_t at =
        bits(y) | static_cast<uintptr_t>(ldy * sizeof(T)) | (bits(q) | static_cast<uintptr_t>(ldq)) * sizeof(T);
    return by_alignment<T>(at, [&](auto access) {
      constexpr bool ANY = decltype(access)::value == 0;
      constexpr int N = (ANY ? 16 : decltype(access)::value) / static_cast<int>(sizeof(T));
      const int units = ceil_div(a.cols, N) + ANY;
      if constexpr (ANY) {
        const RowLaunch r = row_launch<dequantize_any_kernel<T>>(a.n, units, kAnyUnits, true, kRowThreads, kCopyWaves);
        return launch_pdl(dequantize_any_kernel<T>, r.grid, r.block, 0, s, 1, static_cast<const uint8_t*>(q), ldq, scales, lds,
                          static_cast<T*>(y), ldy, a);
      } else {
        const RowLaunch r = row_launch<dequantize_kernel<T, N>>(a.n, units, kDecodeUnits, true, kRowThreads, kCopyWaves);
        return launch_pdl(dequantize_kernel<T, N>, r.grid, r.block, 0, s, 1, static_cast<const uint8_t*>(q), ldq, scales, lds,
                          static_cast<T*>(y), ldy, a);
      }
    });
  });
}

}  // namespace asap

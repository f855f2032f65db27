// Tokens sorted by expert and back, on plain tensors: the place of every (token,
// slot) in its expert's segment, rows to their places, weighted sums of rows back
// to the tokens, and the gradients of both.
#include "common.cuh"
#include "elem.cuh"
#include "rows.h"

#include <cuda_fp8.h>

#include <algorithm>

namespace asap {

namespace {

constexpr unsigned kFull = 0xffffffffu;

// ------------------------------------------------------------ sort
// place(i) = offsets[e_i] + #{i' < i : e_i' = e_i}.  A CTA ranks a chunk of
// kSortChunk entries: a warp takes 256 that follow one another, 32 at a time; the
// lanes with one expert find each other (match), the lowest of them adds their
// number to the warp's counter, and the counter before it plus the lanes below is
// an entry's rank in its warp.  Counters are then summed over the warps.  No
// atomics, so a rank does not depend on any order of execution.
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortRounds = kSortChunk / kSortThreads;
constexpr int kWarpEntries = kSortChunk / kSortWarps;

struct SortShared {
  uint16_t before[kSortWarps][kSortMaxExperts];  // entries of an expert in the chunk's earlier warps
  int total[kSortMaxExperts];                    // of an expert in the chunk; then its first place
  int warp_sum[kSortWarps];
};

__device__ __forceinline__ void rank_chunk(SortShared& s, const int32_t* idx, long long first, long long entries, int E,
                                           int (&e)[kSortRounds], int (&rank)[kSortRounds]) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long at = first + warp * kWarpEntries + lane;
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    e[r] = at + 32 * r < entries ? ld_dep(idx + at + 32 * r) : -1;
    if (e[r] >= E) e[r] = -1;
    if (e[r] < 0) e[r] = -1;
  }
  for (int i = lane; i < E; i += 32) s.before[warp][i] = 0;
  __syncwarp();
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const unsigned same = __match_any_sync(kFull, e[r]);
    const int below = __popc(same & ((1u << lane) - 1));
    int had = 0;
    if (e[r] >= 0) had = s.before[warp][e[r]];
    __syncwarp();
    if (e[r] >= 0 && below == 0) s.before[warp][e[r]] = static_cast<uint16_t>(had + __popc(same));
    __syncwarp();
    rank[r] = had + below;
  }
  __syncthreads();
  for (int x = threadIdx.x; x < E; x += kSortThreads) {
    int sum = 0;
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) {
      const int c = s.before[w][x];
      s.before[w][x] = static_cast<uint16_t>(sum);
      sum += c;
    }
    s.total[x] = sum;
  }
  __syncthreads();
}

// first[x] = sum of count(x') over x' < x, for x < E; returns the sum over all.
template <typename F>
__device__ __forceinline__ int scan_experts(SortShared& s, int E, int* first, F count) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int carry = 0;
  for (int x0 = 0; x0 < E; x0 += kSortThreads) {
    const int x = x0 + threadIdx.x;
    const int c = x < E ? count(x) : 0;
    int sum = c;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(kFull, sum, o);
      if (lane >= o) sum += v;
    }
    if (lane == 31) s.warp_sum[warp] = sum;
    __syncthreads();
    int lower = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) {
      const int v = s.warp_sum[w];
      if (w < warp) lower += v;
      all += v;
    }
    if (x < E) first[x] = carry + lower + sum - c;
    carry += all;
    __syncthreads();
  }
  return carry;
}

__device__ __forceinline__ void write_places(const SortShared& s, long long first, long long entries, int k,
                                             const int (&e)[kSortRounds], const int (&rank)[kSortRounds],
                                             int32_t* perm_dst, int32_t* perm_src) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const long long i = first + warp * kWarpEntries + 32 * r + lane;
    if (i >= entries) continue;
    const int place = e[r] < 0 ? -1 : s.total[e[r]] + s.before[warp][e[r]] + rank[r];
    perm_dst[i] = place;
    if (perm_src && place >= 0) perm_src[place] = static_cast<int32_t>(i / k);
  }
}

// One chunk: the whole sort.
__global__ void __launch_bounds__(kSortThreads)
    sort_small_kernel(const int32_t* idx, int entries, int k, int E, int32_t* offsets, int32_t* perm_dst,
                      int32_t* perm_src) {
  __shared__ SortShared s;
  pdl_wait();
  pdl_launch();
  int e[kSortRounds], rank[kSortRounds];
  rank_chunk(s, idx, 0, entries, E, e, rank);
  const int all = scan_experts(s, E, s.total, [&](int x) { return s.total[x]; });
  for (int x = threadIdx.x; x < E; x += kSortThreads) offsets[x] = s.total[x];
  if (threadIdx.x == 0) offsets[E] = all;
  write_places(s, 0, entries, k, e, rank, perm_dst, perm_src);
}

// Many chunks: each one's counts (hist [chunk][E]); per expert, sums over the
// earlier chunks (in place) and over all (total [E]); places.
__global__ void __launch_bounds__(kSortThreads)
    sort_count_kernel(const int32_t* idx, long long entries, int E, int32_t* hist) {
  __shared__ int count[kSortMaxExperts];
  pdl_wait();
  pdl_launch();
  for (int x = threadIdx.x; x < E; x += kSortThreads) count[x] = 0;
  __syncthreads();
  const long long first = static_cast<long long>(blockIdx.x) * kSortChunk;
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const long long i = first + r * kSortThreads + threadIdx.x;
    const int e = i < entries ? ld_dep(idx + i) : -1;
    if (e >= 0 && e < E) atomicAdd(&count[e], 1);  // (a count: any order gives it)
  }
  __syncthreads();
  for (int x = threadIdx.x; x < E; x += kSortThreads) hist[static_cast<long long>(blockIdx.x) * E + x] = count[x];
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

__global__ void __launch_bounds__(kSortThreads)
    sort_place_kernel(const int32_t* idx, long long entries, int k, int E, const int32_t* hist, const int32_t* total,
                      int32_t* offsets, int32_t* perm_dst, int32_t* perm_src) {
  __shared__ SortShared s;
  pdl_wait();
  pdl_launch();
  const long long first = static_cast<long long>(blockIdx.x) * kSortChunk;
  int e[kSortRounds], rank[kSortRounds];
  rank_chunk(s, idx, first, entries, E, e, rank);
  const int all = scan_experts(s, E, s.total, [&](int x) { return ld_dep(total + x); });
  if (blockIdx.x == 0) {
    for (int x = threadIdx.x; x < E; x += kSortThreads) offsets[x] = s.total[x];
    if (threadIdx.x == 0) offsets[E] = all;
    __syncthreads();
  }
  for (int x = threadIdx.x; x < E; x += kSortThreads)
    s.total[x] += ld_dep(hist + static_cast<long long>(blockIdx.x) * E + x);
  __syncthreads();
  write_places(s, first, entries, k, e, rank, perm_dst, perm_src);
}

// ------------------------------------------------------------ rows
// Threads per token: a CTA takes 256 / PER tokens.
constexpr int kRowThreads = 256;
constexpr int kGroup = 8;  // places of a token handled together

// The j0-th to j0 + 7-th places of token t, -1 where there is none.
__device__ __forceinline__ void load_places(const RowsArgs& a, long long t, int j0, bool report, int (&p)[kGroup]) {
#pragma unroll
  for (int j = 0; j < kGroup; ++j) {
    p[j] = -1;
    if (j0 + j < a.k) {
      p[j] = ld_dep(a.perm + t * a.k + j0 + j);
      if (p[j] < 0 || p[j] >= a.rows) {
        if (report && p[j] != -1) record_status(a.status, ST_BAD_POSITION);
        p[j] = -1;
      }
    }
  }
}

__device__ __forceinline__ uint4 load_unit(const uint4* p) { return ld_dep(p); }
__device__ __forceinline__ uint2 load_unit(const uint2* p) {
  uint2 v;
  asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}
template <typename U>
__device__ __forceinline__ U load_unit(const U* p) {
  return *const_cast<const volatile U*>(p);
}

// x_perm[place] = x[t]: bytes in units of U, the last few of a row one by one.
template <typename U, int PER>
__global__ void __launch_bounds__(kRowThreads)
    permute_kernel(const char* x, long long ldx, char* __restrict__ y, long long ldy, long long row_bytes,
                   const RowsArgs a) {
  pdl_wait();
  pdl_launch();
  const long long t = static_cast<long long>(blockIdx.x) * (kRowThreads / PER) + threadIdx.x / PER;
  if (t >= a.n) return;
  const int vt = threadIdx.x % PER;
  const long long units = row_bytes / static_cast<int>(sizeof(U));
  const char* row = x + t * ldx;
  for (int j0 = 0; j0 < a.k; j0 += kGroup) {
    int p[kGroup];
    load_places(a, t, j0, vt == 0, p);
    for (long long v = vt; v < units; v += PER) {
      const U u = load_unit(reinterpret_cast<const U*>(row + v * sizeof(U)));
#pragma unroll
      for (int j = 0; j < kGroup; ++j)
        if (p[j] >= 0) *reinterpret_cast<U*>(y + p[j] * ldy + v * sizeof(U)) = u;
    }
    for (long long b = units * sizeof(U) + vt; b < row_bytes; b += PER) {
      const char u = load_unit(row + b);
#pragma unroll
      for (int j = 0; j < kGroup; ++j)
        if (p[j] >= 0) y[p[j] * ldy + b] = u;
    }
  }
}

// out[t] = sum_j w[t][j] y[place], fp32 in slot order.
template <typename T, int N, int PER>
__global__ void __launch_bounds__(kRowThreads)
    unpermute_kernel(const T* y, long long ldy, T* __restrict__ out, long long ldo, const RowsArgs a) {
  pdl_wait();
  pdl_launch();
  const long long t = static_cast<long long>(blockIdx.x) * (kRowThreads / PER) + threadIdx.x / PER;
  if (t >= a.n) return;
  const int vt = threadIdx.x % PER;
  int p[kGroup];
  load_places(a, t, 0, vt == 0, p);
  for (long long c = static_cast<long long>(vt) * N; c < a.cols; c += PER * N) {
    const int left = static_cast<int>(a.cols - c);
    float acc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] = 0.f;
    for (int j0 = 0; j0 < a.k; j0 += kGroup) {
      if (a.k > kGroup) load_places(a, t, j0, c == 0, p);
      Cols<T, N> v[kGroup];
#pragma unroll
      for (int j = 0; j < kGroup; ++j)
        if (p[j] >= 0) v[j].load(y + p[j] * ldy + c, left);
#pragma unroll
      for (int j = 0; j < kGroup; ++j)
        if (p[j] >= 0) {
          const float w = a.w ? ld_dep(a.w + t * a.k + j0 + j) : 1.f;
          float f[N];
          v[j].to(f);
#pragma unroll
          for (int i = 0; i < N; ++i) acc[i] = fmaf(w, f[i], acc[i]);
        }
    }
    Cols<T, N> o;
    o.from(acc);
    o.store(out + t * ldo + c, left);
  }
}

// d_y[place] = w d_out[t], d_w[t][j] = <d_out[t], y[place]> (fp32: per thread, then over the threads in a fixed tree).
template <typename T, int N, int PER>
__global__ void __launch_bounds__(kRowThreads)
    unpermute_backward_kernel(const T* d_out, long long ldo, const T* y, long long ldy, T* __restrict__ d_y, long long ldd,
                              float* __restrict__ d_w, const RowsArgs a) {
  __shared__ float part[kRowThreads / 32][kGroup];
  pdl_wait();
  pdl_launch();
  const long long t = static_cast<long long>(blockIdx.x) * (kRowThreads / PER) + threadIdx.x / PER;
  const int vt = threadIdx.x % PER, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool live = t < a.n;
  for (int j0 = 0; j0 < a.k; j0 += kGroup) {
    int p[kGroup];
    float w[kGroup], s[kGroup];
#pragma unroll
    for (int j = 0; j < kGroup; ++j) {
      p[j] = -1;
      s[j] = 0.f;
      w[j] = 1.f;
    }
    if (live) {
      load_places(a, t, j0, vt == 0, p);
#pragma unroll
      for (int j = 0; j < kGroup; ++j)
        if (a.w && p[j] >= 0) w[j] = ld_dep(a.w + t * a.k + j0 + j);
      for (long long c = static_cast<long long>(vt) * N; c < a.cols; c += PER * N) {
        const int left = static_cast<int>(a.cols - c);
        Cols<T, N> v[kGroup], d;
        d.load(d_out + t * ldo + c, left);
        if (d_w) {
#pragma unroll
          for (int j = 0; j < kGroup; ++j)
            if (p[j] >= 0) v[j].load(y + p[j] * ldy + c, left);
        }
        float g[N];
        d.to(g);
#pragma unroll
        for (int j = 0; j < kGroup; ++j)
          if (p[j] >= 0) {
            float f[N];
            if (d_w) {
              v[j].to(f);
#pragma unroll
              for (int i = 0; i < N; ++i) s[j] = fmaf(g[i], f[i], s[j]);
            }
            if (d_y) {
#pragma unroll
              for (int i = 0; i < N; ++i) f[i] = w[j] * g[i];
              Cols<T, N> o;
              o.from(f);
              o.store(d_y + p[j] * ldd + c, left);
            }
          }
      }
    }
    if (!d_w) continue;
#pragma unroll
    for (int j = 0; j < kGroup; ++j)
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s[j] += __shfl_xor_sync(kFull, s[j], o);
    if constexpr (PER > 32) {
      if (lane == 0) {
#pragma unroll
        for (int j = 0; j < kGroup; ++j) part[warp][j] = s[j];
      }
      __syncthreads();
      if (live && vt < kGroup && j0 + vt < a.k) {
        float sum = 0.f;
#pragma unroll
        for (int v = 0; v < PER / 32; ++v) sum += part[warp + v][vt];
        d_w[t * a.k + j0 + vt] = sum;
      }
      __syncthreads();
    } else if (live) {
#pragma unroll
      for (int j = 0; j < kGroup; ++j)
        if (lane == j && j0 + j < a.k) d_w[t * a.k + j0 + j] = s[j];
    }
  }
}

// y[place] = scale q[t], N columns at a time (a scale per 128).
template <typename T, int N, int PER>
__global__ void __launch_bounds__(kRowThreads)
    dequantize_kernel(const uint8_t* q, long long ldq, const float* scales, long long lds, T* __restrict__ y, long long ldy,
                      const RowsArgs a) {
  pdl_wait();
  pdl_launch();
  const long long t = static_cast<long long>(blockIdx.x) * (kRowThreads / PER) + threadIdx.x / PER;
  if (t >= a.n) return;
  const int vt = threadIdx.x % PER;
  for (int j0 = 0; j0 < a.k; j0 += kGroup) {
    int p[kGroup];
    if (a.perm) {
      load_places(a, t, j0, vt == 0, p);
    } else {
#pragma unroll
      for (int j = 0; j < kGroup; ++j) p[j] = j == 0 && t < a.rows ? static_cast<int>(t) : -1;
    }
    for (long long c = static_cast<long long>(vt) * N; c < a.cols; c += PER * N) {
      const int left = static_cast<int>(a.cols - c);
      const uint8_t* from = q + t * ldq + c;
      uint8_t b[N];
      if (N == 8 && left >= 8) {
        uint32_t v[2];
        asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(v[0]), "=r"(v[1]) : "l"(from));
#pragma unroll
        for (int i = 0; i < N; ++i) b[i] = static_cast<uint8_t>(v[(i >> 2) & 1] >> (8 * (i & 3)));
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) b[i] = i < left ? *reinterpret_cast<const volatile uint8_t*>(from + i) : 0;
      }
      const float s = ld_dep(scales + t * lds + (c >> 7));
      float f[N];
#pragma unroll
      for (int i = 0; i < N; ++i)
        f[i] = s * __half2float(__half(__nv_cvt_fp8_to_halfraw(b[i], __NV_E4M3)));
      Cols<T, N> o;
      o.from(f);
#pragma unroll
      for (int j = 0; j < kGroup; ++j)
        if (p[j] >= 0) o.store(y + p[j] * ldy + c, left);
    }
  }
}

// Threads per token for rows of this many units.
int threads_per_row(long long units) { return units <= 32 ? 32 : units <= 128 ? 64 : 256; }

template <typename F>
cudaError_t by_threads(long long units, F f) {
  switch (threads_per_row(units)) {
    case 32: return f(std::integral_constant<int, 32>{});
    case 64: return f(std::integral_constant<int, 64>{});
    default: return f(std::integral_constant<int, 256>{});
  }
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
// Columns per access: 8 where every row starts on 16 bytes, 4 on 8, 2 on 4, else one.  at: addresses and strides in bytes.
template <typename F>
cudaError_t by_alignment(uintptr_t at, int elem, F f) {
  if (at % 16 == 0) return f(std::integral_constant<int, 8>{});
  if (at % (4 * elem) == 0) return f(std::integral_constant<int, 4>{});
  if (at % (2 * elem) == 0) return f(std::integral_constant<int, 2>{});
  return f(std::integral_constant<int, 1>{});
}

uintptr_t bits(const void* p) { return reinterpret_cast<uintptr_t>(p); }
unsigned row_grid(const RowsArgs& a, int per) { return static_cast<unsigned>(ceil_div(a.n, kRowThreads / per)); }

}  // namespace

size_t sort_workspace(long long entries, int experts) {
  const long long chunks = ceil_div(entries, kSortChunk);
  return chunks <= 1 ? 0 : static_cast<size_t>(chunks + 1) * experts * 4;
}

cudaError_t launch_sort(const int32_t* idx, long long entries, int k, int E, int32_t* offsets, int32_t* perm_dst,
                        int32_t* perm_src, void* ws, cudaStream_t s) {
  const long long chunks = ceil_div(entries, kSortChunk);
  if (chunks <= 1)
    return launch_pdl(sort_small_kernel, 1, kSortThreads, 0, s, 1, idx, static_cast<int>(entries), k, E, offsets, perm_dst,
                      perm_src);
  int32_t* total = static_cast<int32_t*>(ws);
  int32_t* hist = total + E;
  const unsigned grid = static_cast<unsigned>(chunks);
  cudaError_t e = launch_pdl(sort_count_kernel, grid, kSortThreads, 0, s, 1, idx, entries, E, hist);
  if (e == cudaSuccess)
    e = launch_pdl(sort_scan_kernel, ceil_div(E, 32), 1024, 0, s, 1, hist, static_cast<int>(chunks), E, total);
  if (e == cudaSuccess)
    e = launch_pdl(sort_place_kernel, grid, kSortThreads, 0, s, 1, idx, entries, k, E, hist, total, offsets, perm_dst,
                   perm_src);
  return e;
}

cudaError_t launch_permute(int elem_bytes, const void* x, long long ldx, void* y, long long ldy, const RowsArgs& a,
                           cudaStream_t s) {
  const long long bytes = static_cast<long long>(a.cols) * elem_bytes;
  ldx *= elem_bytes;
  ldy *= elem_bytes;
  const uintptr_t at = bits(x) | bits(y) | static_cast<uintptr_t>(ldx) | static_cast<uintptr_t>(ldy);
  auto go = [&](auto unit) {
    using U = decltype(unit);
    return by_threads(bytes / static_cast<int>(sizeof(U)), [&](auto per) {
      constexpr int PER = decltype(per)::value;
      return launch_pdl(permute_kernel<U, PER>, row_grid(a, PER), kRowThreads, 0, s, 1, static_cast<const char*>(x), ldx,
                        static_cast<char*>(y), ldy, bytes, a);
    });
  };
  if (at % 16 == 0) return go(uint4{});
  if (at % 8 == 0) return go(uint2{});
  if (at % 4 == 0) return go(0u);
  if (at % 2 == 0) return go(uint16_t{});
  return go(uint8_t{});
}

cudaError_t launch_unpermute(int type, const void* y, long long ldy, void* out, long long ldo, const RowsArgs& a,
                             cudaStream_t s) {
  return by_type(type, [&](auto t) {
    using T = decltype(t);
    const uintptr_t at = bits(y) | bits(out) | static_cast<uintptr_t>((ldy | ldo) * sizeof(T));
    return by_alignment(at, sizeof(T), [&](auto cols) {
      constexpr int N = decltype(cols)::value;
      return by_threads(ceil_div(a.cols, N), [&](auto per) {
        constexpr int PER = decltype(per)::value;
        return launch_pdl(unpermute_kernel<T, N, PER>, row_grid(a, PER), kRowThreads, 0, s, 1, static_cast<const T*>(y),
                          ldy, static_cast<T*>(out), ldo, a);
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
    return by_alignment(at, sizeof(T), [&](auto cols) {
      constexpr int N = decltype(cols)::value;
      return by_threads(ceil_div(a.cols, N), [&](auto per) {
        constexpr int PER = decltype(per)::value;
        return launch_pdl(unpermute_backward_kernel<T, N, PER>, row_grid(a, PER), kRowThreads, 0, s, 1,
                          static_cast<const T*>(d_out), ldo, static_cast<const T*>(y), ldy, static_cast<T*>(d_y), ldd, d_w,
                          a);
      });
    });
  });
}

cudaError_t launch_dequantize(int type, const void* q, long long ldq, const float* scales, long long lds, void* y,
                              long long ldy, const RowsArgs& a, cudaStream_t s) {
  return by_type(type, [&](auto t) {
    using T = decltype(t);
    // (of q's rows only whether they start on 8 bytes counts)
    const bool q8 = (bits(q) | static_cast<uintptr_t>(ldq)) % 8 == 0;
    const uintptr_t at = q8 ? bits(y) | static_cast<uintptr_t>(ldy * sizeof(T)) : sizeof(T);
    return by_alignment(at, sizeof(T), [&](auto cols) {
      constexpr int N = decltype(cols)::value;
      return by_threads(ceil_div(a.cols, N), [&](auto per) {
        constexpr int PER = decltype(per)::value;
        return launch_pdl(dequantize_kernel<T, N, PER>, row_grid(a, PER), kRowThreads, 0, s, 1,
                          static_cast<const uint8_t*>(q), ldq, scales, lds, static_cast<T*>(y), ldy, a);
      });
    });
  });
}

}  // namespace asap

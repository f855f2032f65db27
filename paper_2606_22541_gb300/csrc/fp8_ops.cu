// e4m3 operators on plain tensors: the quantisers of activation rows and the
// matrix product with a scale per block of 128.
#include "common.cuh"
#include "e4m3.cuh"
#include "internal.h"

#include <algorithm>

namespace asap {

namespace {

constexpr unsigned kFull = 0xffffffffu;

// ------------------------------------------------------------ quantisers
// A team of 8 lanes takes a group of 128 columns, 16 to a lane; a warp's four teams
// take groups that follow one another.  W: columns per load (8, 4 or 1, by the
// alignment of the rows).  The arithmetic per column would bound a scalar kernel
// (45 us for 8045 rows of 7168), so quotients go in pairs (f32x2) and bf16
// magnitudes two to a register.  Loads are hidden by eight CTAs an SM rather than
// by several groups of a team on their way, whose registers cost more (1, 2 and 4
// groups: 29.5, 33 and 35 us; SwiGLU of 4014 rows of 4096: 16, 18 and 23).
constexpr int kQuantThreads = 256;
constexpr int kTeam = 8;

template <int W>
__device__ __forceinline__ void load8(const uint16_t* p, int left, uint32_t* v) {
  if constexpr (W == 8) {
    if (left >= 8) {
      asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                   : "l"(p));
      return;
    }
  } else if constexpr (W == 4) {
    if (left >= 8) {
      asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(v[0]), "=r"(v[1]) : "l"(p));
      asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(v[2]), "=r"(v[3]) : "l"(p + 4));
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint16_t lo = 0, hi = 0;
    if (2 * i < left) asm volatile("ld.global.b16 %0, [%1];" : "=h"(lo) : "l"(p + 2 * i));
    if (2 * i + 1 < left) asm volatile("ld.global.b16 %0, [%1];" : "=h"(hi) : "l"(p + 2 * i + 1));
    v[i] = lo | (static_cast<uint32_t>(hi) << 16);
  }
}

__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ float2 unpair(uint64_t p) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(p));
  return r;
}
// The larger magnitude of each half (a NaN loses).
__device__ __forceinline__ uint32_t max_abs2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 m = __hmax2(__habs2(*reinterpret_cast<const __nv_bfloat162*>(&a)),
                                   __habs2(*reinterpret_cast<const __nv_bfloat162*>(&b)));
  return *reinterpret_cast<const uint32_t*>(&m);
}

__device__ __forceinline__ float swiglu(float g, float u) { return __fdividef(g, 1.0f + __expf(-g)) * u; }

template <bool SWIGLU, int W>
__global__ void __launch_bounds__(kQuantThreads, 8) fp8_quantize_kernel(const uint16_t* x, const uint16_t* u, int rows,
                                                                    int cols, long long ld, uint8_t* q, long long ldq,
                                                                    float* s, long long lds, bool wide_q) {
  pdl_wait();
  pdl_launch();
  const int lane = threadIdx.x & (kTeam - 1);
  const int groups = (cols + 127) / 128;  // of a row
  const int teams = gridDim.x * (kQuantThreads / kTeam);
  const int first = blockIdx.x * (kQuantThreads / kTeam) + threadIdx.x / kTeam;
  // the team's groups are first, first + teams, ... of rows * groups
  const int dr = teams / groups, dg = teams % groups;
  int row = first / groups, grp = first % groups;
  // (a warp's teams leave together: their shuffles name the whole warp)
  while (__any_sync(kFull, row < rows)) {
    uint32_t g[8], up[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] = up[j] = 0u;
    const int c = grp * 128 + lane * 16;
    const bool in = row < rows && c < cols;
    if (in) {
      const long long at = row * ld + c;
      load8<W>(x + at, cols - c, g);
      load8<W>(x + at + 8, cols - c - 8, g + 4);
      if constexpr (SWIGLU) {
        load8<W>(u + at, cols - c, up);
        load8<W>(u + at + 8, cols - c - 8, up + 4);
      }
    }
    float f[16];
    float am;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      f[2 * j] = bf16_lo(g[j]);
      f[2 * j + 1] = bf16_hi(g[j]);
    }
    if constexpr (SWIGLU) {
      am = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        f[2 * j] = swiglu(f[2 * j], bf16_lo(up[j]));
        f[2 * j + 1] = swiglu(f[2 * j + 1], bf16_hi(up[j]));
        am = fmaxf(am, fmaxf(fabsf(f[2 * j]), fabsf(f[2 * j + 1])));
      }
#pragma unroll
      for (int o = kTeam / 2; o > 0; o >>= 1) am = fmaxf(am, __shfl_xor_sync(kFull, am, o));
    } else {
      uint32_t m = max_abs2(max_abs2(max_abs2(g[0], g[1]), max_abs2(g[2], g[3])),
                            max_abs2(max_abs2(g[4], g[5]), max_abs2(g[6], g[7])));
#pragma unroll
      for (int o = kTeam / 2; o > 0; o >>= 1) m = max_abs2(m, __shfl_xor_sync(kFull, m, o));
      am = fmaxf(fmaxf(bf16_lo(m), bf16_hi(m)), 0.f);  // (0 where there are only NaNs)
    }
    const GroupScale gs(am);
    if (in) {
      const uint64_t inv = pair(gs.inv, gs.inv), neg = pair(-gs.scaled, -gs.scaled);
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint64_t v0 = pair(f[4 * j], f[4 * j + 1]), v1 = pair(f[4 * j + 2], f[4 * j + 3]);
        if (gs.up != 1.0f) {
          const uint64_t by = pair(gs.up, gs.up);
          v0 = mul2(v0, by);
          v1 = mul2(v1, by);
        }
        uint64_t q0 = mul2(v0, inv), q1 = mul2(v1, inv);  // GroupScale's quotient, two at a time
        q0 = fma2(fma2(q0, neg, v0), inv, q0);
        q1 = fma2(fma2(q1, neg, v1), inv, q1);
        const float2 a = unpair(q0), b = unpair(q1);
        w[j] = e4m3x4(a.x, a.y, b.x, b.y);
      }
      uint8_t* out = q + row * ldq + c;
      if (wide_q && cols - c >= 16) {
        *reinterpret_cast<uint4*>(out) = make_uint4(w[0], w[1], w[2], w[3]);
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (j < cols - c) out[j] = static_cast<uint8_t>(w[j >> 2] >> (8 * (j & 3)));
      }
      if (lane == 0) s[row * lds + grp] = gs.s;
    }
    row += dr;
    grp += dg;
    if (grp >= groups) grp -= groups, ++row;
  }
}

// ------------------------------------------------------------ product, weights as the M operand
// A tile is 128 rows of B (M; one row of scale blocks) and NT rows of A (N); a
// cluster of S CTAs shares a tile, each with a slice of K.  Every 128-wide K block
// is multiplied into one of the TMEM partials, which the epilogue warps add, times
// the block's scales, into registers; the slices' sums meet in distributed shared
// memory, each CTA adding those of about 128 / S rows in rank order.  They travel as bulk
// copies, counted by the receiver's mbarrier.  (Plain stores between cluster
// barriers and 16-byte st.async move about 0.5 TB/s over the whole GPU: 64 rows x
// 4096 x 14336 on eight slices, 8 MB of sums, took 22 and 17 us.)  Two CTAs an
// SM, so that one's start and end pass beside the other's stream; persistent
// CTAs, one an SM with a ring twice as deep and the sums of a tile exchanged while
// the next one streams, took 8.9 us there and 30 instead of 24 for 45 rows x 28672
// x 4096: their four epilogue warps are a CTA's only ones.
//   warp 0: TMA producer; warp 1: TMEM and MMA; warps 2-5: epilogue, one TMEM
//   lane quarter (32 rows of B) each.
constexpr int kRows = 128;
constexpr int kBBytes = kRows * kFp8BK;
constexpr int kEpiThreads = 128;
constexpr int kThreads = 64 + kEpiThreads;
constexpr int kMaxSplit = 8;

template <int NT>
struct Skinny {
  static constexpr int kStage = kBBytes + NT * kFp8BK;
  static constexpr int kStages = NT == 16 ? 5 : NT == 32 ? 4 : 3;  // about 100 KB: two CTAs an SM
  static constexpr int kPartials = 4;
  static constexpr uint32_t kTmem = NT * kPartials;
  static constexpr int kPitch = NT + 4;  // floats of a row of the slices' sums
  static constexpr int kSums = (kRows + kMaxSplit - 1) * kPitch;  // slices x the rows of a rank, rounded up
  static constexpr int kBars = 2 * kStages + 2 * kPartials + 2;
  static constexpr size_t kSmem = kStages * kStage + 4 * kSums + 2 * NT * 4 + 8 * kBars + 16;
  static_assert(2 * (kSmem + 1024) <= 228 * 1024, "two CTAs an SM");
  static_assert(4 * kRows * kPitch <= kStages * kStage, "the ring holds the sums to be sent");
};

struct SkinnyArgs {
  Fp8MatmulArgs p;
  int split, m_tiles;
};

__device__ __forceinline__ uint32_t map_rank(uint32_t addr, uint32_t rank) {
  uint32_t d;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(d) : "r"(addr), "r"(rank));
  return d;
}
// Barrier of the cluster's threads; the first orders no memory (barriers are
// initialised with a fence of their own).
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory"); }
__device__ __forceinline__ void cluster_arrive_release() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait;" ::: "memory"); }
// Arrive on a barrier of the cluster's CTA that addr names (map_rank).  Neither
// this nor the waits take cluster scope, which stalls a thread for thousands of
// cycles behind the loads in flight: what they order is counted in bytes or has
// been seen to be done.
__device__ __forceinline__ void mbar_arrive_remote(uint32_t addr) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}
// tma_load_2d into both CTAs of a pair, at the same offsets, completing on both barriers.
__device__ __forceinline__ void tma_load_2d_both(uint32_t dst, const CUtensorMap* m, uint32_t bar, int x, int y,
                                                 uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.multicast::cluster.L2::cache_hint"
      " [%0], [%1, {%3, %4}], [%2], %5, %6;" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(x), "r"(y), "h"(static_cast<uint16_t>(3)), "l"(policy)
      : "memory");
}
// tc_commit on the barrier at this offset in both CTAs of a pair.
__device__ __forceinline__ void tc_commit_both(uint32_t bar) {
  asm volatile(
      "tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
      "h"(static_cast<uint16_t>(3))
      : "memory");
}
// Shared memory of this CTA into one of the cluster, whose barrier counts the bytes.
__device__ __forceinline__ void send(uint32_t to, uint32_t from, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to),
               "r"(from), "r"(bytes), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void mma_e4m3(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(acc)
      : "memory");
}

template <int NT>
__global__ void __launch_bounds__(kThreads, 2)
    fp8_skinny_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                      const SkinnyArgs args) {
  using C = Skinny<NT>;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t base = smem_u32(smem_raw);
  const Fp8MatmulArgs& p = args.p;
  const bool aligned = (base & 1023u) == 0;  // the 128-byte swizzle needs it; the same in the cluster
  const int S = args.split;
  const int rank = blockIdx.x % S;
  const int tile = blockIdx.x / S;
  const int row0 = tile / args.m_tiles * kRows;  // of B
  const int tok0 = tile % args.m_tiles * NT;     // of A
  const int blocks = (p.k + kFp8BK - 1) / kFp8BK;
  const int kb0 = static_cast<int>(static_cast<long long>(blocks) * rank / S);
  const int kb1 = static_cast<int>(static_cast<long long>(blocks) * (rank + 1) / S);
  float* sums = reinterpret_cast<float*>(smem_raw + C::kStages * C::kStage);  // [slice][row][column]
  float* scales = sums + C::kSums;                                            // [2][NT]
  uint64_t* bars = reinterpret_cast<uint64_t*>(scales + 2 * NT);
  const uint32_t bar0 = smem_u32(bars);
  auto full = [&](int i) { return bar0 + 8u * i; };
  auto empty = [&](int i) { return bar0 + 8u * (C::kStages + i); };
  auto pfull = [&](int i) { return bar0 + 8u * (2 * C::kStages + i); };
  auto pempty = [&](int i) { return bar0 + 8u * (2 * C::kStages + C::kPartials + i); };
  const uint32_t drain = bar0 + 8u * (C::kBars - 2), received = drain + 8u;
  auto first_row = [&](int to) { return kRows * to / S; };  // of the rows whose sums CTA ``to`` adds
  const int rows = first_row(rank + 1) - first_row(rank);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + C::kBars);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < C::kStages; ++i) {
      mbar_init(full(i), 1);
      mbar_init(empty(i), 1);
    }
    for (int i = 0; i < C::kPartials; ++i) {
      mbar_init(pfull(i), 1);
      mbar_init(pempty(i), 4);
    }
    mbar_init(drain, 1);
    mbar_init(received, 1);
    *abort_flag = aligned ? 0 : 1;
    fence_barrier_init();
    if (S > 1) mbar_arrive_expect_tx(received, static_cast<uint32_t>(4 * S * rows * C::kPitch));
    tma_prefetch_desc(&tmA);
    tma_prefetch_desc(&tmB);
  } else if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), C::kTmem);
    tmem_relinquish();
  }
  __syncwarp();
  if (S > 1) cluster_arrive();  // this CTA's barriers stand
  pdl_wait();
  if (!aligned && threadIdx.x == 0) record_status(p.status, ST_SMEM_ALIGN);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  auto give_up = [&]() {
    *abort_flag = 1;
    record_status(p.status, ST_WAIT_TIMEOUT);
  };
  if (warp == 0) {
    if (lane == 0 && aligned) {
      Ring<C::kStages> r;
      const uint64_t pol_b = l2_policy(args.m_tiles == 1 ? 1 : 0), pol_a = l2_policy(2);
      int issued = 0;
      bool ok = true;
      for (int kb = kb0; kb < kb1; ++kb) {
        ok = mbar_wait(empty(r.s), r.phase ^ 1u, abort_flag);
        if (!ok) break;
        const uint32_t st = base + r.s * C::kStage;
        mbar_arrive_expect_tx(full(r.s), C::kStage);
        tma_load_2d(st, &tmB, full(r.s), kb * kFp8BK, row0, pol_b);
        tma_load_2d(st + kBBytes, &tmA, full(r.s), kb * kFp8BK, tok0, pol_a);
        issued = min(issued + 1, C::kStages);
        r.advance();
      }
      pdl_launch();  // nothing left to load
      if (!ok) {
        give_up();
        // the copies in flight land before the CTA's memory goes away
        int dummy = 0;
        for (int i = issued; i > 0; --i) {
          const int b = r.s - i;
          mbar_wait(full(b < 0 ? b + C::kStages : b), b < 0 ? r.phase ^ 1u : r.phase, &dummy);
        }
      }
    }
  } else if (warp == 1) {
    const bool issuer = elect_one();
    constexpr uint32_t id =
        (1u << 4) | (static_cast<uint32_t>(NT >> 3) << 17) | (static_cast<uint32_t>(kRows >> 4) << 24);
    Ring<C::kStages> r;
    Ring<C::kPartials> t;
    bool ok = aligned, issued = false;
    for (int kb = kb0; ok && kb < kb1; ++kb) {
      ok = __all_sync(kFull, mbar_wait(full(r.s), r.phase, abort_flag) &&
                                 mbar_wait(pempty(t.s), t.phase ^ 1u, abort_flag));
      if (!ok) break;
      tc_fence_after();
      if (issuer) {
        const uint64_t bd = smem_desc_sw128(base + r.s * C::kStage);
        const uint64_t ad = smem_desc_sw128(base + r.s * C::kStage + kBBytes);
#pragma unroll
        for (int kk = 0; kk < kFp8BK / 32; ++kk)
          mma_e4m3(tmem_base + t.s * NT, bd + 2 * kk, ad + 2 * kk, id, kk > 0 ? 1u : 0u);
        tc_commit(pfull(t.s));
        tc_commit(empty(r.s));
      }
      __syncwarp();
      issued = true;
      r.advance();
      t.advance();
    }
    if (!ok) {
      if (lane == 0 && aligned) give_up();
      if (issued) {
        int dummy = 0;
        if (elect_one()) tc_commit(drain);
        __syncwarp();
        mbar_wait(drain, 0, &dummy);
      }
    }
  } else {
    // (a warp whose wait has failed goes on through the barriers that the four share)
    const int q = warp & 3;
    const int tid = threadIdx.x - 64;
    const int r = q * 32 + lane;  // row of the tile
    const uint32_t lanes = tmem_base + (static_cast<uint32_t>(q * 32) << 16);
    auto epi_sync = [&]() {
      __syncwarp();
      asm volatile("bar.sync 1, 128;" ::: "memory");
    };
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.c);
    Ring<C::kPartials> t;
    bool ok = aligned;
    // thread i: the scale of column i, times the block's of B, kLead blocks ahead
    constexpr int kLead = 4;
    const bool column = tid < NT && tok0 + tid < p.m;
    const float* sa = p.sa + static_cast<long long>(tok0 + tid) * p.lds_a;
    const float* sb = p.sb + static_cast<long long>(row0 / kRows) * p.lds_b;
    float na[kLead], nb[kLead];
    auto ahead = [&](int i, int kb) {
      na[i] = column && kb < kb1 ? ld_dep(sa + kb) : 0.f;
      nb[i] = column && kb < kb1 ? ld_dep(sb + kb) : 0.f;
    };
    float acc[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) acc[i] = 0.f;
#pragma unroll
    for (int i = 0; i < kLead; ++i) ahead(i, kb0 + i);
    for (int k4 = kb0; k4 < kb1; k4 += kLead) {
#pragma unroll
      for (int i = 0; i < kLead; ++i) {
        const int kb = k4 + i;
        if (kb >= kb1) break;
        float* sc = scales + (i & 1) * NT;
        if (tid < NT) sc[tid] = na[i] * nb[i];
        ahead(i, kb + kLead);
        epi_sync();
        ok = ok && __all_sync(kFull, mbar_wait(pfull(t.s), t.phase, abort_flag));
        if (ok) {
          tc_fence_after();
          constexpr int kCols = NT < 32 ? NT : 32;  // columns on their way at a time
#pragma unroll
          for (int c0 = 0; c0 < NT; c0 += kCols) {
            uint32_t v[kCols / 16][16];
#pragma unroll
            for (int c = 0; c < kCols / 16; ++c) tmem_ld16(lanes + t.s * NT + c0 + 16 * c, v[c]);
            tmem_ld_wait();
            if (c0 + kCols == NT) {  // the partial is in registers
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(pempty(t.s));
            }
#pragma unroll
            for (int c = 0; c < kCols; c += 4) {
              const float4 f = *reinterpret_cast<const float4*>(sc + c0 + c);
              const uint32_t* x = &v[c / 16][c % 16];
              acc[c0 + c] = fmaf(f.x, __uint_as_float(x[0]), acc[c0 + c]);
              acc[c0 + c + 1] = fmaf(f.y, __uint_as_float(x[1]), acc[c0 + c + 1]);
              acc[c0 + c + 2] = fmaf(f.z, __uint_as_float(x[2]), acc[c0 + c + 2]);
              acc[c0 + c + 3] = fmaf(f.w, __uint_as_float(x[3]), acc[c0 + c + 3]);
            }
          }
        }
        t.advance();
      }
    }
    if (S == 1) {
      const int n = row0 + r;
#pragma unroll
      for (int c = 0; c < NT; ++c)
        if (ok && n < p.n && tok0 + c < p.m)
          out[static_cast<long long>(tok0 + c) * p.ldc + n] = __float2bfloat16_rn(acc[c]);
    } else {
      // the ring is done with (its last MMA has been seen to be): it holds the sums until they are sent
      float4* row = reinterpret_cast<float4*>(smem_raw + r * C::kPitch * 4);
#pragma unroll
      for (int c = 0; c < NT / 4; ++c) row[c] = make_float4(acc[4 * c], acc[4 * c + 1], acc[4 * c + 2], acc[4 * c + 3]);
      fence_proxy_async_smem();
      epi_sync();
      cluster_wait();
      if (ok && tid < S) {
        const int at = first_row(tid);
        const uint32_t bytes = static_cast<uint32_t>((first_row(tid + 1) - at) * C::kPitch * 4);
        send(map_rank(smem_u32(sums) + rank * bytes, tid), base + at * C::kPitch * 4, bytes, map_rank(received, tid));
      }
      __syncwarp();
      ok = ok && __all_sync(kFull, mbar_wait(received, 0, abort_flag));
      // four columns of a row at a time, rows along the lanes
      const int cols = min(NT, p.m - tok0);
      int c = tid / rows * 4, rr = tid % rows;
      while (ok && c < cols) {
        const float* at = sums + rr * C::kPitch + c;
        float4 v = *reinterpret_cast<const float4*>(at);
        for (int s = 1; s < S; ++s) {
          at += rows * C::kPitch;
          const float4 w = *reinterpret_cast<const float4*>(at);
          v.x += w.x, v.y += w.y, v.z += w.z, v.w += w.w;
        }
        const int n = row0 + first_row(rank) + rr;
        const float f[4] = {v.x, v.y, v.z, v.w};
        __nv_bfloat16* o = out + static_cast<long long>(tok0 + c) * p.ldc + n;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (n < p.n && c + i < cols) o[i * p.ldc] = __float2bfloat16_rn(f[i]);
        rr += kEpiThreads % rows;
        c += kEpiThreads / rows * 4;
        if (rr >= rows) rr -= rows, c += 4;
      }
    }
    if (!ok && lane == 0 && aligned) give_up();
  }
  if (S > 1) {  // no CTA leaves while another may still send to it
    if (warp < 2) cluster_wait();
    __syncwarp();
    cluster_arrive_release();
    cluster_wait();
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, C::kTmem);
  }
}

// ------------------------------------------------------------ product, rows of A as the M operand
// A tile is 128 rows of A (M) and 256 of B (N).  Every 128-wide K block has one of
// two TMEM partials of 256 columns, which eight epilogue warps add, times row and
// block scale, into registers (warp w: TMEM lanes 32 (w % 4) .., one half of the
// columns, i.e. one row of scale blocks), two 16-column chunks in turn, so that one
// is on its way while the other is added.  Three forms: a CTA takes a tile after
// the other; CTA pairs do, on two tiles with the same rows of B, of which each loads
// one half for both (a tile's operands through L2 would be 16 TB/s at 2.7 PFLOP/s);
// or a cluster of S CTAs shares a tile as above.
//   warp 0: TMA producer; warp 1: TMEM and MMA; warps 4-11: epilogue, which takes
//   registers from the first four warps (56 + 2 x 224 a thread).
constexpr int kWideN = 256;
constexpr int kWideStages = 4;
constexpr int kWideStage = (kRows + kWideN) * kFp8BK;
constexpr int kWidePartials = 2;
constexpr int kWideThreads = 32 * 12;
constexpr int kCtrlRegs = 56, kEpiRegs = 224;
static_assert(kCtrlRegs + 2 * kEpiRegs <= 3 * 168, "the register split stays within the launch's registers");
constexpr int kWideBars = 2 * kWideStages + 2 * kWidePartials + 6;
constexpr int kWideSplit = 4;  // K slices at most
constexpr int kStageWarp = 32 * 4 * 16;   // output staging of an epilogue warp
enum { WIDE_SINGLE = 0, WIDE_PAIR = 1, WIDE_SPLIT = 2 };
// The slices' sums of a column half: those to be sent, then those that come, each at
// most (S - 1) / S of 128 x 128 floats, in the ring's place.
constexpr int kHalfSums = (kWideSplit - 1) * (kRows / kWideSplit) * 128 * 4;
constexpr size_t kWideSmem = kWideStages * kWideStage + 8 * kStageWarp + 8 * kWideBars + 16;
static_assert(kWideSmem <= 227 * 1024, "shared memory budget");
static_assert(4 * kHalfSums <= kWideStages * kWideStage, "the sums fit the ring");

struct WideArgs {
  Fp8MatmulArgs p;
  int cluster;  // K slices of a tile, or 2 for pairs
  int m_tiles;  // tiles, or pairs of tiles, along the rows of A
  int tiles;    // (pairs of) tiles in all
  int c_align;  // rows of c start on multiples of this many bytes (16, 4 or 2)
};

__device__ __forceinline__ void add16(float* acc, const uint32_t (&v)[16], float s) {
#pragma unroll
  for (int j = 0; j < 16; ++j) acc[j] = fmaf(s, __uint_as_float(v[j]), acc[j]);
}

template <int FORM>
__global__ void __launch_bounds__(kWideThreads, 1)
    fp8_wide_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                    const WideArgs args) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t base = smem_u32(smem_raw);
  const Fp8MatmulArgs& p = args.p;
  const bool aligned = (base & 1023u) == 0;  // the 128-byte swizzle needs it; the same in the cluster
  constexpr bool SPLIT = FORM == WIDE_SPLIT, PAIR = FORM == WIDE_PAIR;
  const int cluster = FORM == WIDE_SINGLE ? 1 : args.cluster;
  const int in_cluster = blockIdx.x % cluster, first = blockIdx.x / cluster;
  const int step = gridDim.x / cluster;  // (pairs of) tiles between a CTA's
  const int S = SPLIT ? cluster : 1, rank = SPLIT ? in_cluster : 0;
  const int blocks = (p.k + kFp8BK - 1) / kFp8BK;
  const int kb0 = static_cast<int>(static_cast<long long>(blocks) * rank / S);
  const int kb1 = static_cast<int>(static_cast<long long>(blocks) * (rank + 1) / S);
  uint4* stage_all = reinterpret_cast<uint4*>(smem_raw + kWideStages * kWideStage);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem_raw + kWideStages * kWideStage + 8 * kStageWarp);
  const uint32_t bar0 = smem_u32(bars);
  auto full = [&](int i) { return bar0 + 8u * i; };
  auto empty = [&](int i) { return bar0 + 8u * (kWideStages + i); };
  auto pfull = [&](int i) { return bar0 + 8u * (2 * kWideStages + i); };
  auto pempty = [&](int i) { return bar0 + 8u * (2 * kWideStages + kWidePartials + i); };
  // all CTAs' rings are done with; per column half: the rows to be sent are written, the slices have come
  const uint32_t drain = bar0 + 8u * (kWideBars - 6), rings = drain + 8u, written = drain + 16u, received = drain + 32u;
  const int rows = kRows / S;  // whose sums this CTA adds
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + kWideBars);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kWideStages; ++i) {
      mbar_init(full(i), 1);
      mbar_init(empty(i), PAIR ? 2 : 1);  // (pairs: both CTAs have read the stage)
    }
    for (int i = 0; i < kWidePartials; ++i) {
      mbar_init(pfull(i), 1);
      mbar_init(pempty(i), 8);
    }
    mbar_init(drain, 1);
    mbar_init(rings, S);
    for (uint32_t i = 0; i < 2; ++i) {
      mbar_init(written + 8u * i, 4);
      mbar_init(received + 8u * i, 1);
    }
    *abort_flag = aligned ? 0 : 1;
    fence_barrier_init();
    if (SPLIT)
      for (int i = 0; i < 2; ++i) mbar_arrive_expect_tx(received + 8u * i, static_cast<uint32_t>((S - 1) * rows * 512));
    tma_prefetch_desc(&tmA);
    tma_prefetch_desc(&tmB);
  } else if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), 512);
    tmem_relinquish();
  }
  __syncwarp();
  if (FORM != WIDE_SINGLE) cluster_arrive();  // this CTA's barriers stand
  pdl_wait();
  if (!aligned && threadIdx.x == 0) record_status(p.status, ST_SMEM_ALIGN);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  if (PAIR) cluster_wait();
  auto tok_of = [&](int tile) { return (tile % args.m_tiles * (PAIR ? 2 : 1) + (PAIR ? in_cluster : 0)) * kRows; };
  bool waited = false;  // for the cluster's barriers to stand
  auto give_up = [&]() {
    *abort_flag = 1;
    record_status(p.status, ST_WAIT_TIMEOUT);
  };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kCtrlRegs));
    if (warp == 0) {
      const bool issuer = elect_one();
      Ring<kWideStages> r;
      const uint64_t pol = l2_policy(2);
      int issued = 0;
      bool ok = aligned;
      for (int tile = first; ok && tile < args.tiles; tile += step) {
        const int tok0 = tok_of(tile), row0 = tile / args.m_tiles * kWideN;
        for (int kb = kb0; kb < kb1; ++kb) {
          ok = __all_sync(kFull, mbar_wait(empty(r.s), r.phase ^ 1u, abort_flag));
          if (!ok) break;
          if (issuer) {
            const uint32_t st = base + r.s * kWideStage;
            mbar_arrive_expect_tx(full(r.s), kWideStage);
            tma_load_2d(st, &tmA, full(r.s), kb * kFp8BK, tok0, pol);
            if (PAIR)  // this CTA's half of the rows of B, for both
              tma_load_2d_both(st + kRows * kFp8BK + in_cluster * kBBytes, &tmB, full(r.s), kb * kFp8BK,
                               row0 + in_cluster * kRows, pol);
            else
              tma_load_2d(st + kRows * kFp8BK, &tmB, full(r.s), kb * kFp8BK, row0, pol);
          }
          issued = min(issued + 1, kWideStages);
          r.advance();
        }
      }
      if (issuer) pdl_launch();  // nothing left to load
      if (PAIR)  // both CTAs' commits on this ring have come before the CTA may leave
        for (int i = 0; ok && i < kWideStages; ++i) {
          ok = __all_sync(kFull, mbar_wait(empty(r.s), r.phase ^ 1u, abort_flag));
          r.advance();
        }
      if (!ok && aligned) {
        if (issuer) give_up();
        // the copies in flight land before the CTA's memory goes away
        int dummy = 0;
        for (int i = issued; i > 0; --i) {
          const int b = r.s - i;
          mbar_wait(full(b < 0 ? b + kWideStages : b), b < 0 ? r.phase ^ 1u : r.phase, &dummy);
        }
        if (PAIR) {  // (and those into the other CTA, which only it can wait for: a TMA load takes microseconds)
          const uint64_t t0 = globaltimer_ns();
          while (globaltimer_ns() - t0 < 2000000ull) {
          }
        }
      }
    } else if (warp == 1) {
      const bool issuer = elect_one();
      constexpr uint32_t id =
          (1u << 4) | (static_cast<uint32_t>(kWideN >> 3) << 17) | (static_cast<uint32_t>(kRows >> 4) << 24);
      Ring<kWideStages> r;
      Ring<kWidePartials> t;
      bool ok = aligned, issued = false;
      for (int tile = first; ok && tile < args.tiles; tile += step) {
        for (int kb = kb0; kb < kb1; ++kb) {
          ok = mbar_wait_all(lane < 16 ? full(r.s) : pempty(t.s), lane < 16 ? r.phase : t.phase ^ 1u, abort_flag);
          if (!ok) break;
          tc_fence_after();
          if (issuer) {
            const uint64_t ad = smem_desc_sw128(base + r.s * kWideStage);
            const uint64_t bd = smem_desc_sw128(base + r.s * kWideStage + kRows * kFp8BK);
#pragma unroll
            for (int kk = 0; kk < kFp8BK / 32; ++kk)
              mma_e4m3(tmem_base + t.s * kWideN, ad + 2 * kk, bd + 2 * kk, id, kk > 0 ? 1u : 0u);
            tc_commit(pfull(t.s));
            if (PAIR) tc_commit_both(empty(r.s));
            else tc_commit(empty(r.s));
          }
          __syncwarp();
          issued = true;
          r.advance();
          t.advance();
        }
      }
      if (!ok && aligned) {
        if (lane == 0) give_up();
        if (issued) {
          int dummy = 0;
          if (elect_one()) tc_commit(drain);
          __syncwarp();
          mbar_wait(drain, 0, &dummy);
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kEpiRegs));
    const int q = warp & 3, half = (warp - 4) >> 2;
    const uint32_t col = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + half * 128;
    uint4* stage = stage_all + (warp - 4) * (kStageWarp / 16);
    Ring<kWidePartials> t;
    bool ok = aligned;
    for (int tile = first; tile < args.tiles; tile += step) {
      const int tok0 = tok_of(tile), row0 = tile / args.m_tiles * kWideN + half * 128;
      float acc[128];
#pragma unroll
      for (int j = 0; j < 128; ++j) acc[j] = 0.f;
      // (rows and columns that do not exist take the last one's scales; their products are zero)
      const float* sa = p.sa + static_cast<long long>(min(tok0 + q * 32 + lane, p.m - 1)) * p.lds_a;
      const float* sb = p.sb + static_cast<long long>(min(row0, p.n - 1) / 128) * p.lds_b;
      float a0 = ld_dep(sa + kb0), b0 = ld_dep(sb + kb0), a1 = 0.f, b1 = 0.f;
      if (kb0 + 1 < kb1) a1 = ld_dep(sa + kb0 + 1), b1 = ld_dep(sb + kb0 + 1);
      uint32_t c0[16], c1[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) c1[j] = 0u;
      float s_prev = 0.f;
      for (int kb = kb0; kb < kb1; ++kb) {
        const float s = a0 * b0;
        a0 = a1;
        b0 = b1;
        if (kb + 2 < kb1) a1 = ld_dep(sa + kb + 2), b1 = ld_dep(sb + kb + 2);
        ok = ok && __all_sync(kFull, mbar_wait(pfull(t.s), t.phase, abort_flag));
        if (!ok) break;
        tc_fence_after();
        const uint32_t ta = col + t.s * kWideN;
        tmem_ld16(ta, c0);
        add16(acc + 112, c1, s_prev);
        tmem_ld_wait();
        tmem_ld16(ta + 16, c1);
        add16(acc + 0, c0, s);
        tmem_ld_wait();
        tmem_ld16(ta + 32, c0);
        add16(acc + 16, c1, s);
        tmem_ld_wait();
        tmem_ld16(ta + 48, c1);
        add16(acc + 32, c0, s);
        tmem_ld_wait();
        tmem_ld16(ta + 64, c0);
        add16(acc + 48, c1, s);
        tmem_ld_wait();
        tmem_ld16(ta + 80, c1);
        add16(acc + 64, c0, s);
        tmem_ld_wait();
        tmem_ld16(ta + 96, c0);
        add16(acc + 80, c1, s);
        tmem_ld_wait();
        tmem_ld16(ta + 112, c1);
        add16(acc + 96, c0, s);
        tmem_ld_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(pempty(t.s));
        s_prev = s;
        t.advance();
      }
      if (!ok) break;
      add16(acc + 112, c1, s_prev);
      bool store = true;
      if constexpr (SPLIT) {
        // Every CTA sends the rows that others add (a warp's rows have one owner) and adds what comes for its own, in
        // rank order behind its own sums.  A row's 16-byte chunk c lies at c ^ (row % 8): no bank conflicts.
        const int owner = (q * 32) / rows, rr = q * 32 + lane - owner * rows;
        store = owner == rank;
        uint8_t* out_sums = smem_raw + half * 2 * kHalfSums;  // this CTA's ring is done with: its last MMA has been seen to be
        const uint8_t* in_sums = out_sums + kHalfSums;
        if (!store) {
          uint8_t* row = out_sums + ((owner - (owner > rank ? 1 : 0)) * rows + rr) * 512;
#pragma unroll
          for (int c = 0; c < 32; ++c)
            *reinterpret_cast<float4*>(row + ((c ^ (rr & 7)) << 4)) =
                make_float4(acc[4 * c], acc[4 * c + 1], acc[4 * c + 2], acc[4 * c + 3]);
          fence_proxy_async_smem();
        }
        cluster_wait();
        waited = true;
        if (warp == 4 && lane < S) mbar_arrive_remote(map_rank(rings, static_cast<uint32_t>(lane)));
        __syncwarp();
        if (lane == 0) mbar_arrive(written + 8u * half);
        if (q == 0) ok = __all_sync(kFull, mbar_wait(rings, 0, abort_flag) && mbar_wait(written + 8u * half, 0, abort_flag));
        if (!ok) break;
        if (q == 0 && lane < S - 1) {
          const int to = lane + (lane >= rank ? 1 : 0);
          const uint32_t bytes = static_cast<uint32_t>(rows * 512);
          send(map_rank(smem_u32(in_sums) + (rank - (rank > to ? 1 : 0)) * bytes, static_cast<uint32_t>(to)),
               smem_u32(out_sums) + lane * bytes, bytes, map_rank(received + 8u * half, static_cast<uint32_t>(to)));
        }
        __syncwarp();
        if (store) {
          ok = __all_sync(kFull, mbar_wait(received + 8u * half, 0, abort_flag));
          if (!ok) break;
          for (int s = 0; s < S - 1; ++s) {
            const uint8_t* row = in_sums + (s * rows + rr) * 512;
#pragma unroll
            for (int c = 0; c < 32; ++c) {
              const float4 v = *reinterpret_cast<const float4*>(row + ((c ^ (rr & 7)) << 4));
              acc[4 * c] += v.x, acc[4 * c + 1] += v.y, acc[4 * c + 2] += v.z, acc[4 * c + 3] += v.w;
            }
          }
        }
      }
      if (store) {
        // four rounds of 32 columns: a row's 64 bytes cross the warp's staging (chunk j of row r at slot
        // j ^ ((r / 2) % 4): no bank conflicts) and leave as eight rows x 64 bytes per store instruction
#pragma unroll
        for (int rd = 0; rd < 4; ++rd) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float* v = acc + 32 * rd + 8 * j;
            stage[lane * 4 + (j ^ ((lane >> 1) & 3))] = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                                                   pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
          }
          __syncwarp();
          const int t0 = tok0 + q * 32, n0 = row0 + 32 * rd;
          __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.c) + static_cast<long long>(t0) * p.ldc + n0;
          if (args.c_align == 16 && n0 + 32 <= p.n) {
            const int cu = lane & 3;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int r = (lane >> 2) + 8 * i;
              if (t0 + r < p.m)
                *reinterpret_cast<uint4*>(out + r * p.ldc + 8 * cu) = stage[r * 4 + (cu ^ ((r >> 1) & 3))];
            }
          } else if (args.c_align >= 4 && (p.n & 1) == 0) {
            // two columns a lane, two rows an instruction
            const int c = 2 * (lane & 15);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int r = (lane >> 4) + 2 * i;
              const uint32_t v =
                  reinterpret_cast<const uint32_t*>(&stage[r * 4 + ((c >> 3) ^ ((r >> 1) & 3))])[(c & 7) >> 1];
              if (t0 + r < p.m && n0 + c < p.n) *reinterpret_cast<uint32_t*>(out + r * p.ldc + c) = v;
            }
          } else {
#pragma unroll 8
            for (int r = 0; r < 32; ++r) {
              const uint16_t v =
                  reinterpret_cast<const uint16_t*>(&stage[r * 4 + ((lane >> 3) ^ ((r >> 1) & 3))])[lane & 7];
              if (t0 + r < p.m && n0 + lane < p.n) *reinterpret_cast<uint16_t*>(out + r * p.ldc + lane) = v;
            }
          }
          __syncwarp();
        }
      }
    }
    if (!ok && aligned && lane == 0) give_up();
  }
  if (FORM != WIDE_SINGLE) {  // no CTA leaves while another may still write to it
    if (SPLIT && !waited) cluster_wait();
    __syncwarp();
    cluster_arrive_release();
    cluster_wait();
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, 512);
  }
}

template <int NT>
cudaError_t skinny(const CUtensorMap& tmA, const CUtensorMap& tmB, const Fp8MatmulArgs& args, int num_sms,
                   cudaStream_t s) {
  const int blocks = ceil_div(args.k, kFp8BK);
  SkinnyArgs a{args, 1, ceil_div(args.m, NT)};
  const long long tiles = static_cast<long long>(ceil_div(args.n, kRows)) * a.m_tiles;
  // K slices of two blocks and more as long as all CTAs are resident at once (a second wave costs more than shorter
  // slices save: 45 rows x 28672 x 4096 on 1, 2 and 4 slices 24, 38 and 46 us; 64 x 4100 x 14300 on 4, 6 and 8, all
  // one wave, 18.0, 16.9 and 15.4; 64 x 12288 x 6144 on 1 and 3 23.6 and 18.7)
  a.split = static_cast<int>(std::max<long long>(1, std::min<long long>({kMaxSplit, 2 * num_sms / tiles, blocks / 2})));
  return launch_pdl(fp8_skinny_kernel<NT>, dim3(static_cast<unsigned>(tiles * a.split)), dim3(kThreads),
                    Skinny<NT>::kSmem, s, a.split, tmA, tmB, a);
}

cudaError_t wide(const void* a, long long lda, const void* b, long long ldb, const Fp8MatmulArgs& args, int num_sms,
                 cudaStream_t s, std::string* err) {
  const int blocks = ceil_div(args.k, kFp8BK);
  const int m_tiles = ceil_div(args.m, kRows);
  const long long tiles = static_cast<long long>(ceil_div(args.n, kWideN)) * m_tiles;
  // (slices that meet cost 2.5 us on two CTAs and 5 on four: 400 x 2048 x 2048, 16 blocks, on 1, 2 and 4 slices 10.2,
  // 10.0 and 12.2 us; 256 x 4096 x 4096, 32 blocks, 17.3, 14.4 and 15.5; 400 x 2048 x 7168, 56, 24.4, 19.0 and 17.8)
  int split = 1;
  while (split < kWideSplit && tiles * split * 2 <= num_sms && blocks >= 24 * split) split *= 2;
  // Pairs where operand traffic counts: long contractions in more than one wave of tiles (single / pairs, us: 8045 x
  // 4096 x 7168 191 / 174, 16000 x 2048 x 7168 218 / 197, 1024 x 28672 x 4096 99 / 94; but 700 x 4096 x 7168, one
  // wave, 28 / 34, and 4096 x 7168 x 2048 53 / 55 to 61: a pair's CTAs wait for one another at every tile's end).
  const bool pairs = split == 1 && m_tiles >= 2 && tiles > num_sms && blocks >= 32;
  CUtensorMap tmA, tmB;
  if (!encode_tmap_u8(&tmA, a, args.m, args.k, kRows, err, lda) ||
      !encode_tmap_u8(&tmB, b, args.n, args.k, pairs ? kWideN / 2 : kWideN, err, ldb))
    return cudaErrorInvalidValue;
  const uintptr_t at = reinterpret_cast<uintptr_t>(args.c) | static_cast<uintptr_t>(2 * args.ldc);
  WideArgs w{args, pairs ? 2 : split, pairs ? ceil_div(m_tiles, 2) : m_tiles, 0,
             (at & 15u) == 0 ? 16 : (at & 3u) == 0 ? 4 : 2};
  w.tiles = ceil_div(args.n, kWideN) * w.m_tiles;
  const dim3 block(kWideThreads);
  if (split > 1)
    return launch_pdl(fp8_wide_kernel<WIDE_SPLIT>, dim3(w.tiles * split), block, kWideSmem, s, split, tmA, tmB, w);
  if (pairs)
    return launch_pdl(fp8_wide_kernel<WIDE_PAIR>, dim3(2 * std::min(w.tiles, num_sms / 2)), block, kWideSmem, s, 2, tmA,
                      tmB, w);
  return launch_pdl(fp8_wide_kernel<WIDE_SINGLE>, dim3(std::min(w.tiles, num_sms)), block, kWideSmem, s, 1, tmA, tmB, w);
}

}  // namespace

cudaError_t fp8_matmul_set_attributes() {
  cudaError_t e = cudaSuccess;
  auto set = [&](auto* f, size_t bytes) {
    if (e == cudaSuccess)
      e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
  };
  set(fp8_skinny_kernel<16>, Skinny<16>::kSmem);
  set(fp8_skinny_kernel<32>, Skinny<32>::kSmem);
  set(fp8_skinny_kernel<64>, Skinny<64>::kSmem);
  set(fp8_wide_kernel<WIDE_SINGLE>, kWideSmem);
  set(fp8_wide_kernel<WIDE_PAIR>, kWideSmem);
  set(fp8_wide_kernel<WIDE_SPLIT>, kWideSmem);
  return e;
}

cudaError_t fp8_matmul_launch(const void* a, long long lda, const void* b, long long ldb, const Fp8MatmulArgs& args,
                              int num_sms, cudaStream_t s, std::string* err) {
  // More than 64 rows go to the wide tiles, unless the product is so small that its narrow tiles, cut into slices,
  // still are one wave and long enough to be worth cutting (wide / narrow: 65 x 512 x 2048 10.9 / 7.1 us, 128 x 2048 x
  // 7168 17.9 / 14.2, 200 x 2048 x 7168 18.9 / 17.3, 1000 x 512 x 4096 18.0 / 15.5; but twice as many tiles, 256 x
  // 4096 x 4096, 16.7 / 19.2, and half the blocks, 65 x 4096 x 1024, 8.0 / 10.7)
  const long long narrow = static_cast<long long>(ceil_div(args.m, 64)) * ceil_div(args.n, kRows);
  if (args.m > 64 && (narrow > num_sms / 2 || args.k <= 15 * kFp8BK)) return wide(a, lda, b, ldb, args, num_sms, s, err);
  CUtensorMap tmA, tmB;
  const int nt = args.m <= 16 ? 16 : args.m <= 32 ? 32 : 64;
  if (!encode_tmap_u8(&tmA, a, args.m, args.k, nt, err, lda) ||
      !encode_tmap_u8(&tmB, b, args.n, args.k, kRows, err, ldb))
    return cudaErrorInvalidValue;
  switch (nt) {
    case 16: return skinny<16>(tmA, tmB, args, num_sms, s);
    case 32: return skinny<32>(tmA, tmB, args, num_sms, s);
    default: return skinny<64>(tmA, tmB, args, num_sms, s);
  }
}

cudaError_t launch_fp8_quantize(const void* x, const void* u, int rows, int cols, long long ld, void* q,
                                long long ldq, float* s, long long lds, cudaStream_t st) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(u) | static_cast<uintptr_t>(2 * ld);
  const bool wide_q = ((reinterpret_cast<uintptr_t>(q) | static_cast<uintptr_t>(ldq)) & 15u) == 0;
  const long long groups = static_cast<long long>(rows) * ceil_div(cols, 128);
  const unsigned grid = static_cast<unsigned>(std::min<long long>((groups + 31) / 32, 152 * 32));
  const uint16_t *xp = static_cast<const uint16_t*>(x), *up = static_cast<const uint16_t*>(u);
  uint8_t* qp = static_cast<uint8_t*>(q);
#define ASAP_QUANT(SW, W)                                                                                            \
  return launch_pdl(fp8_quantize_kernel<SW, W>, dim3(grid), dim3(kQuantThreads), 0, st, 1, xp, up, rows, cols, ld, qp, ldq, \
                    s, lds, wide_q)
  if (u) {
    if ((at & 15u) == 0) ASAP_QUANT(true, 8);
    if ((at & 7u) == 0) ASAP_QUANT(true, 4);
    ASAP_QUANT(true, 1);
  }
  if ((at & 15u) == 0) ASAP_QUANT(false, 8);
  if ((at & 7u) == 0) ASAP_QUANT(false, 4);
  ASAP_QUANT(false, 1);
#undef ASAP_QUANT
}

}  // namespace asap

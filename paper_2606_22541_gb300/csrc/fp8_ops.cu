// e4m3 operators on plain tensors: the quantisers of activation rows and the
// matrix product with a scale per block of 128.
#include "common.cuh"
#include "e4m3.cuh"
#include "internal.h"
#include "pair.cuh"

#include <algorithm>

namespace asap {

namespace {

constexpr unsigned kFull = 0xffffffffu;

// ------------------------------------------------------------ quantisers
// A team of 8 lanes takes a group of 128 columns, 16 to a lane; a warp's four teams
// take groups that follow one another.  W: columns per load (8, 4 or 1, by the
// alignment of the rows).  The arithmetic per column would bound a scalar kernel
// (45 us for 8045 rows of 7168), so quotients go in pairs (f32x2) and bf16
// magnitudes two to a register.  Loads are hidden by eight CTAs an SM (six for
// SwiGLU's registers) rather than by several groups of a team on their way, whose
// registers cost more (1, 2 and 4 groups: 29.5, 33 and 35 us).
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
// a b + c rounded down, for the remainder of a quotient: that of an exact zero is -0, which leaves a quotient of -0 as it
// is (+0 would not); other remainders are exact, or far below what they correct.
__device__ __forceinline__ uint64_t remainder2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rm.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
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

// silu(g) * u of two columns: expf, and the quotient from the approximate reciprocal with one correction by its
// remainder (Markstein), which leaves it right but for the last bit's ties.  Where e^-g overflows, or nearly, it is
// divided.  Of 98.6 million values 83 came out other than the exact value's e4m3, as with a division, and 74 to 79 with
// fp32 arithmetic elsewhere.  With __expf and __fdividef it was 106, and 15.4 us instead of 20 (4014 x 4096; a division
// everywhere 22): not worth a third more values on the wrong side.
__device__ __noinline__ float swiglu_far(float g, float u) { return g / (1.0f + expf(-g)) * u; }
__device__ __forceinline__ float2 swiglu2(float2 g, float2 u) {
  const float dx = 1.0f + expf(-g.x), dy = 1.0f + expf(-g.y);
  float rx, ry;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(rx) : "f"(dx));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(ry) : "f"(dy));
  const uint64_t x = pair(g.x, g.y), nd = pair(-dx, -dy), r = pair(rx, ry), q = mul2(x, r);
  return unpair(mul2(fma2(remainder2(q, nd, x), r, q), pair(u.x, u.y)));
}

template <bool SWIGLU, int W>
__global__ void __launch_bounds__(kQuantThreads, SWIGLU ? 6 : 8)
    fp8_quantize_kernel(const uint16_t* x, const uint16_t* u, int rows, int cols, long long ld, uint8_t* q,
                        long long ldq, float* s, long long lds, bool wide_q) {
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
      const uint32_t m = max_abs2(max_abs2(max_abs2(g[0], g[1]), max_abs2(g[2], g[3])),
                                  max_abs2(max_abs2(g[4], g[5]), max_abs2(g[6], g[7])));
      const bool far = fmaxf(bf16_lo(m), bf16_hi(m)) >= 80.f;
      am = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float2 gj = make_float2(f[2 * j], f[2 * j + 1]), uj = make_float2(bf16_lo(up[j]), bf16_hi(up[j]));
        const float2 v = far ? make_float2(swiglu_far(gj.x, uj.x), swiglu_far(gj.y, uj.y)) : swiglu2(gj, uj);
        f[2 * j] = v.x;
        f[2 * j + 1] = v.y;
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
        q0 = fma2(remainder2(q0, neg, v0), inv, q0);
        q1 = fma2(remainder2(q1, neg, v1), inv, q1);
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
// Two CTAs of this file's kernels hold at most the 512 TMEM columns of an SM, and no other kernel that uses TMEM leaves
// shared memory for one of them: an allocation never waits for a CTA whose cluster waits for this one.
constexpr int kRows = 128;
constexpr int kBBytes = kRows * kFp8BK;
constexpr int kEpiThreads = 128;
constexpr int kThreads = 64 + kEpiThreads;
constexpr int kMaxSplit = 8;

template <int NT>
struct Skinny {
  static constexpr int kStage = kBBytes + NT * kFp8BK;
  static constexpr int kStages = NT == 16 ? 5 : NT == 32 ? 4 : 3;  // about 100 KB: two CTAs an SM
  static constexpr int kAlone = NT == 16 ? 8 : 7;  // of a CTA that has its SM to itself (0.1 to 0.5 us less)
  static constexpr int kPartials = 4;
  static constexpr uint32_t kTmem = NT * kPartials;
  static constexpr int kPitch = NT + 4;  // floats of a row of the slices' sums
  static constexpr int kSums = (kRows + kMaxSplit - 1) * kPitch;  // slices x the rows of a rank, rounded up
  // hundredths of a microsecond: a K block, the meeting of two slices, a second CTA on the SMs
  static constexpr int kBlock = NT == 16 ? 23 : NT == 32 ? 29 : 31;
  static constexpr int kMeet = NT == 16 ? 95 : NT == 32 ? 130 : 186;
  static constexpr int kTwo = NT == 16 ? 100 : NT == 32 ? 150 : 250;
  static constexpr int kBars = 2 * kAlone + 2 * kPartials + 2;
  static constexpr size_t kRest = 4 * kSums + 2 * NT * 4 + 8 * kBars + 16;
  static_assert(2 * (kStages * kStage + kRest + 1024) <= 228 * 1024, "two CTAs an SM");
  static_assert(kAlone * kStage + kRest <= 227 * 1024, "shared memory budget");
  static_assert(4 * kRows * kPitch <= kStages * kStage, "the ring holds the sums to be sent");
};

struct SkinnyArgs {
  Fp8MatmulArgs p;
  int split, m_tiles;
  int stages;  // of the ring
};

// Ring of a number of stages that the launch chooses.
struct RingOf {
  int stages, s = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ explicit RingOf(int n) : stages(n) {}
  __device__ __forceinline__ void advance() {
    if (++s == stages) {
      s = 0;
      phase ^= 1u;
    }
  }
};

// Barrier of the cluster's threads; the first orders no memory (barriers are
// initialised with a fence of their own).
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory"); }
__device__ __forceinline__ void cluster_arrive_release() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait;" ::: "memory"); }
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
  float* sums = reinterpret_cast<float*>(smem_raw + args.stages * C::kStage);  // [slice][row][column]
  float* scales = sums + C::kSums;                                            // [2][NT]
  uint64_t* bars = reinterpret_cast<uint64_t*>(scales + 2 * NT);
  const uint32_t bar0 = smem_u32(bars);
  auto full = [&](int i) { return bar0 + 8u * i; };
  auto empty = [&](int i) { return bar0 + 8u * (C::kAlone + i); };
  auto pfull = [&](int i) { return bar0 + 8u * (2 * C::kAlone + i); };
  auto pempty = [&](int i) { return bar0 + 8u * (2 * C::kAlone + C::kPartials + i); };
  const uint32_t drain = bar0 + 8u * (C::kBars - 2), received = drain + 8u;
  auto first_row = [&](int to) { return kRows * to / S; };  // of the rows whose sums CTA ``to`` adds
  const int rows = first_row(rank + 1) - first_row(rank);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + C::kBars);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < args.stages; ++i) {
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
      RingOf r(args.stages);
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
        issued = min(issued + 1, args.stages);
        r.advance();
      }
      pdl_launch();  // nothing left to load
      if (!ok) {
        give_up();
        // the copies in flight land before the CTA's memory goes away
        int dummy = 0;
        for (int i = issued; i > 0; --i) {
          const int b = r.s - i;
          mbar_wait(full(b < 0 ? b + args.stages : b), b < 0 ? r.phase ^ 1u : r.phase, &dummy);
        }
      }
    }
  } else if (warp == 1) {
    const bool issuer = elect_one();
    constexpr uint32_t id =
        (1u << 4) | (static_cast<uint32_t>(NT >> 3) << 17) | (static_cast<uint32_t>(kRows >> 4) << 24);
    RingOf r(args.stages);
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
        send(pair_map(smem_u32(sums) + rank * bytes, tid), base + at * C::kPitch * 4, bytes, pair_map(received, tid));
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
// A tile is 128 rows of A (M) and TN = 256 or 128 of B (N).  Every 128-wide K block has one of two TMEM partials of TN
// columns, which the epilogue warps add, times row and block scale, into registers (warp w: TMEM lanes 32 (w % 4) .., a
// half of 128 columns, i.e. one row of scale blocks): two 16-column chunks in turn, so that one is on its way while the
// other is added, in pairs (f32x2: 2 % of 8045 x 4096 x 7168, 4 % of 8045 x 28672 x 1024).  One CTA of 256 columns has
// an SM, up to two of 128 do.  A CTA takes a tile after the other, or a cluster of S CTAs shares one as above.
//   warp 0: TMA producer; warp 1: TMEM and MMA; from warp 4 on: epilogue, which takes
//   registers from the first four warps.
// What bounds it: the adding, and for long runs power.  8045 x 4096 x 7168 takes 198 to 204 us in a stream of calls (2.36
// PFLOP/s, in a steady state of power) and 172 after a pause (2.75 PFLOP/s at about 1.85 GHz); 154 with an epilogue that only passes the partials on (3.07
// PFLOP/s), 160 with one that reads them all and adds nothing.  On top of its K loop a tile takes 1.5 us to round and
// store, while the next tile's first two blocks are multiplied: with short contractions that shows (8045 x 28672 x 1024
// 232 us, 2.04 PFLOP/s).  Tried and no faster: chunks of 32 columns, four partials of 128 columns, pairs of CTAs that
// load each other's half of the rows of B by multicast, and pairs that multiply 256 rows by 256 together (cta_group::2,
// six stages: 198 us in the steady state too, 186 against 180 in single calls, 252 against 242 for 8045 x 28672 x 1024):
// what operands cost through L2 and shared memory is hidden behind the adding.
constexpr int kWideSplit = 4;  // K slices at most
template <int TN>
struct Wide {
  static constexpr int kStages = TN == 256 ? 4 : 3;
  // of a CTA that has its SM to itself (6 instead of 3: 256 x 7168 x 2048 10.0 to 8.8 us, 65 x 2048 x 14336 on one
  // slice 43 to 35: a load takes about a microsecond)
  static constexpr int kAlone = TN == 256 ? 4 : 6;
  static constexpr int kStage = (kRows + TN) * kFp8BK;
  static constexpr int kPartials = 2;
  static constexpr int kEpiWarps = TN / 32;
  static constexpr int kThreads = 128 + 32 * kEpiWarps;
  static constexpr int kCtas = 256 / TN;  // an SM
  static constexpr int kCtrlRegs = TN == 256 ? 56 : 40, kEpiRegs = TN == 256 ? 224 : 216;
  static constexpr int kLaunchRegs = 65536 / (kCtas * kThreads) / 8 * 8;
  static_assert(4 * kCtrlRegs + kEpiWarps * kEpiRegs <= kThreads / 32 * kLaunchRegs,
                "the register split stays within the launch's registers");
  static constexpr int kBars = 2 * kAlone + 2 * kPartials + 4;
  static constexpr int kStageWarp = 2 * 32 * 64;  // an epilogue warp's output staging: two rounds of 32 columns
  static constexpr size_t kRest = kEpiWarps * kStageWarp + 8 * kBars + 16;
  static_assert(kCtas * (kStages * kStage + kRest + 1024) <= 228 * 1024 && kAlone * kStage + kRest <= 227 * 1024,
                "shared memory budget");
  // slices: a tile's sums, then those that come for a CTA's rows, in the place of the ring and the staging
  static constexpr int kSums = kRows * TN * 4;
  static_assert(kSums + (kWideSplit - 1) * (kRows / kWideSplit) * TN * 4 <= kStages * kStage + kEpiWarps * kStageWarp &&
                kSums + 2 * ((kRows + 2) / 3) * TN * 4 <= kStages * kStage + kEpiWarps * kStageWarp, "the sums fit");
};
struct WideArgs {
  Fp8MatmulArgs p;
  int split;    // K slices of a tile: the cluster
  int m_tiles;  // tiles along the rows of A
  int tiles;    // in all
  int stages;   // of the ring
  int c_align;  // rows of c start on multiples of this many bytes (16, 8, 4 or 2)
};

__device__ __forceinline__ void add16(float* acc, const uint32_t (&v)[16], float s) {
  const uint64_t ss = pair(s, s);
#pragma unroll
  for (int j = 0; j < 16; j += 2) {
    const uint64_t r = fma2(pair(__uint_as_float(v[j]), __uint_as_float(v[j + 1])), ss, pair(acc[j], acc[j + 1]));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(acc[j]), "=f"(acc[j + 1]) : "l"(r));
  }
}

template <bool SPLIT, int TN>
__global__ void __launch_bounds__(Wide<TN>::kThreads, Wide<TN>::kCtas)
    fp8_wide_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                    const __grid_constant__ CUtensorMap tmC, const WideArgs args) {
  using C = Wide<TN>;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t base = smem_u32(smem_raw);
  const Fp8MatmulArgs& p = args.p;
  const bool aligned = (base & 1023u) == 0;  // the 128-byte swizzle needs it; the same in the cluster
  const int S = SPLIT ? args.split : 1, rank = SPLIT ? blockIdx.x % S : 0;
  const int first = blockIdx.x / S, step = gridDim.x / S;  // a CTA's tiles
  const int blocks = (p.k + kFp8BK - 1) / kFp8BK;
  const int kb0 = static_cast<int>(static_cast<long long>(blocks) * rank / S);
  const int kb1 = static_cast<int>(static_cast<long long>(blocks) * (rank + 1) / S);
  uint8_t* stage_all = smem_raw + args.stages * C::kStage;
  uint64_t* bars = reinterpret_cast<uint64_t*>(stage_all + C::kEpiWarps * C::kStageWarp);
  const uint32_t bar0 = smem_u32(bars);
  auto full = [&](int i) { return bar0 + 8u * i; };
  auto empty = [&](int i) { return bar0 + 8u * (C::kAlone + i); };
  auto pfull = [&](int i) { return bar0 + 8u * (2 * C::kAlone + i); };
  auto pempty = [&](int i) { return bar0 + 8u * (2 * C::kAlone + C::kPartials + i); };
  // all CTAs' rings are done with, this one's sums are written, the slices have come
  const uint32_t drain = bar0 + 8u * (C::kBars - 4), rings = drain + 8u, written = drain + 16u, received = drain + 24u;
  auto first_row = [&](int to) { return kRows * to / S; };  // of the rows whose sums CTA ``to`` adds
  const int own0 = first_row(rank), own1 = first_row(rank + 1);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + C::kBars);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < args.stages; ++i) {
      mbar_init(full(i), 1);
      mbar_init(empty(i), 1);
    }
    for (int i = 0; i < C::kPartials; ++i) {
      mbar_init(pfull(i), 1);
      mbar_init(pempty(i), C::kEpiWarps);
    }
    mbar_init(drain, 1);
    mbar_init(rings, S);
    mbar_init(written, C::kEpiWarps);
    mbar_init(received, 1);
    *abort_flag = aligned ? 0 : 1;
    fence_barrier_init();
    if (SPLIT) mbar_arrive_expect_tx(received, static_cast<uint32_t>((S - 1) * (own1 - own0) * TN * 4));
    tma_prefetch_desc(&tmA);
    tma_prefetch_desc(&tmB);
    if (!SPLIT && args.c_align == 16) tma_prefetch_desc(&tmC);
  } else if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), 2 * TN);
    tmem_relinquish();
  }
  __syncwarp();
  if (SPLIT) cluster_arrive();  // this CTA's barriers stand
  pdl_wait();
  if (!aligned && threadIdx.x == 0) record_status(p.status, ST_SMEM_ALIGN);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  bool waited = false;  // for the cluster's barriers to stand
  auto give_up = [&]() {
    *abort_flag = 1;
    record_status(p.status, ST_WAIT_TIMEOUT);
  };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kCtrlRegs));
    if (warp == 0) {
      const bool issuer = elect_one();
      RingOf r(args.stages);
      const uint64_t pol = l2_policy(2);
      int issued = 0;
      bool ok = aligned;
      for (int tile = first; ok && tile < args.tiles; tile += step) {
        const int tok0 = tile % args.m_tiles * kRows, row0 = tile / args.m_tiles * TN;
        for (int kb = kb0; kb < kb1; ++kb) {
          ok = __all_sync(kFull, mbar_wait(empty(r.s), r.phase ^ 1u, abort_flag));
          if (!ok) break;
          if (issuer) {
            const uint32_t st = base + r.s * C::kStage;
            mbar_arrive_expect_tx(full(r.s), C::kStage);
            tma_load_2d(st, &tmA, full(r.s), kb * kFp8BK, tok0, pol);
            tma_load_2d(st + kRows * kFp8BK, &tmB, full(r.s), kb * kFp8BK, row0, pol);
          }
          issued = min(issued + 1, args.stages);
          r.advance();
        }
      }
      if (issuer) pdl_launch();  // nothing left to load
      if (!ok && aligned) {
        if (issuer) give_up();
        // the copies in flight land before the CTA's memory goes away
        int dummy = 0;
        for (int i = issued; i > 0; --i) {
          const int b = r.s - i;
          mbar_wait(full(b < 0 ? b + args.stages : b), b < 0 ? r.phase ^ 1u : r.phase, &dummy);
        }
      }
    } else if (warp == 1) {
      const bool issuer = elect_one();
      constexpr uint32_t id =
          (1u << 4) | (static_cast<uint32_t>(TN >> 3) << 17) | (static_cast<uint32_t>(kRows >> 4) << 24);
      RingOf r(args.stages);
      Ring<C::kPartials> t;
      bool ok = aligned, issued = false;
      for (int tile = first; ok && tile < args.tiles; tile += step) {
        for (int kb = kb0; kb < kb1; ++kb) {
          ok = mbar_wait_all(lane < 16 ? full(r.s) : pempty(t.s), lane < 16 ? r.phase : t.phase ^ 1u, abort_flag);
          if (!ok) break;
          tc_fence_after();
          if (issuer) {
            const uint64_t ad = smem_desc_sw128(base + r.s * C::kStage);
            const uint64_t bd = smem_desc_sw128(base + r.s * C::kStage + kRows * kFp8BK);
#pragma unroll
            for (int kk = 0; kk < kFp8BK / 32; ++kk)
              mma_e4m3(tmem_base + t.s * TN, ad + 2 * kk, bd + 2 * kk, id, kk > 0 ? 1u : 0u);
            tc_commit(pfull(t.s));
            tc_commit(empty(r.s));
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
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kEpiRegs));
    const int q = warp & 3, half = (warp - 4) >> 2;
    const uint32_t col = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + half * 128;
    uint8_t* stage_warp = stage_all + (warp - 4) * C::kStageWarp;
    Ring<C::kPartials> t;
    bool ok = aligned;
    for (int tile = first; tile < args.tiles; tile += step) {
      const int tok0 = tile % args.m_tiles * kRows, row0 = tile / args.m_tiles * TN + half * 128;
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
        const uint32_t ta = col + t.s * TN;
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
      if constexpr (SPLIT) {
        // Every CTA sends the rows that others add, and its warps add what has come for its own, in rank order, 128
        // columns of a row at a time.  128 columns of a row are 512 bytes, 16-byte chunk c at c ^ (row % 8).  This CTA's
        // ring is done with: its last MMA has been seen to be.
        const int row = q * 32 + lane, mine = own1 - own0;
        constexpr int kHalf = kRows * 512;  // bytes of 128 columns
        uint8_t* to = smem_raw + half * kHalf + row * 512;
#pragma unroll
        for (int c = 0; c < 32; ++c)
          *reinterpret_cast<float4*>(to + ((c ^ (row & 7)) << 4)) =
              make_float4(acc[4 * c], acc[4 * c + 1], acc[4 * c + 2], acc[4 * c + 3]);
        fence_proxy_async_smem();
        cluster_wait();
        waited = true;
        if (warp == 4 && lane < S) mbar_arrive_pair(pair_map(rings, static_cast<uint32_t>(lane)));
        __syncwarp();
        if (lane == 0) mbar_arrive(written);
        ok = __all_sync(kFull, mbar_wait(written, 0, abort_flag) && (warp != 4 || mbar_wait(rings, 0, abort_flag)));
        if (!ok) break;
        if (warp == 4 && lane < (S - 1) * (TN / 128)) {
          const int h = lane / (S - 1), i = lane - h * (S - 1), dst = i + (i >= rank ? 1 : 0);
          const int r0 = first_row(dst), theirs = first_row(dst + 1) - r0;
          const uint32_t place = base + C::kSums + (h * (S - 1) + rank - (rank > dst ? 1 : 0)) * theirs * 512;
          send(pair_map(place, static_cast<uint32_t>(dst)), base + h * kHalf + r0 * 512, static_cast<uint32_t>(theirs * 512),
               pair_map(received, static_cast<uint32_t>(dst)));
        }
        __syncwarp();
        ok = __all_sync(kFull, mbar_wait(received, 0, abort_flag));
        if (!ok) break;
        // eight rows on their way at a time (where the warps that have the rows in registers added and stored them, the
        // others waited: up to 1.2 us longer)
        constexpr int kAhead = 8;
#pragma unroll 1
        for (int h = 0; h < TN / 128; ++h) {
          const int n0 = tile / args.m_tiles * TN + h * 128 + 4 * lane;
          const uint8_t* own = smem_raw + h * kHalf + own0 * 512;
          const uint8_t* come = smem_raw + C::kSums + h * (S - 1) * mine * 512;
#pragma unroll 1
          for (int r0 = warp - 4; r0 < mine; r0 += kAhead * C::kEpiWarps) {
            float4 v[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
            for (int sl = 0; sl < S; ++sl) {
              const uint8_t* from = sl == rank ? own : come + (sl - (sl > rank ? 1 : 0)) * mine * 512;
#pragma unroll
              for (int u = 0; u < kAhead; ++u) {
                const int r = min(r0 + u * C::kEpiWarps, mine - 1);
                const float4 w = *reinterpret_cast<const float4*>(from + r * 512 + ((lane ^ ((own0 + r) & 7)) << 4));
                v[u].x += w.x, v[u].y += w.y, v[u].z += w.z, v[u].w += w.w;
              }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
              const int r = r0 + u * C::kEpiWarps, t = tok0 + own0 + r;
              if (r >= mine || t >= p.m) break;
              __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.c) + static_cast<long long>(t) * p.ldc + n0;
              if (args.c_align >= 8 && n0 + 4 <= p.n) {
                *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16x2(v[u].x, v[u].y), pack_bf16x2(v[u].z, v[u].w));
              } else {
                const float f[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (n0 + e < p.n) out[e] = __float2bfloat16_rn(f[e]);
              }
            }
          }
        }
        break;  // (the only tile)
      } else {
        // Four rounds of 32 columns, in two buffers: a row's 64 bytes cross the warp's staging, chunk j of row r at slot
        // j ^ ((r / 2) % 4): no bank conflicts, and the 64-byte swizzle of a TMA box.
#pragma unroll
        for (int rd = 0; rd < 4; ++rd) {
          uint4* stage = reinterpret_cast<uint4*>(stage_warp + (rd & 1) * (C::kStageWarp / 2));
          const int t0 = tok0 + q * 32, n0 = row0 + 32 * rd;
          // (a box is cut at the tensor's edge in 16-byte pieces)
          const bool bulk = args.c_align == 16 && (n0 + 32 <= p.n || (p.n & 7) == 0);
          // the box of two rounds ago has been read
          if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
          __syncwarp();
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float* v = acc + 32 * rd + 8 * j;
            stage[lane * 4 + (j ^ ((lane >> 1) & 3))] = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                                                   pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
          }
          // (a group a round, an empty one too: the one that may stay pending above is the round before)
          if (bulk) {
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0 && t0 < p.m && n0 < p.n) tma_store_2d(&tmC, smem_u32(stage), n0, t0);
            if (lane == 0) bulk_commit_group();
            continue;
          }
          if (lane == 0) bulk_commit_group();
          __syncwarp();
          __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.c) + static_cast<long long>(t0) * p.ldc + n0;
          if (args.c_align >= 4 && (p.n & 1) == 0) {  // two columns a lane, two rows an instruction
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
    if (lane == 0) bulk_wait_group0();
    __syncwarp();
    if (!ok && aligned && lane == 0) give_up();
  }
  if (SPLIT) {  // no CTA leaves while another may still write to it
    if (!waited) cluster_wait();
    __syncwarp();
    cluster_arrive_release();
    cluster_wait();
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, 2 * TN);
  }
}

template <int NT>
cudaError_t skinny(const CUtensorMap& tmA, const CUtensorMap& tmB, const Fp8MatmulArgs& args, const Fp8MatmulDevice& dev,
                   cudaStream_t s) {
  using C = Skinny<NT>;
  const int blocks = ceil_div(args.k, kFp8BK);
  SkinnyArgs a{args, 1, ceil_div(args.m, NT)};
  const long long tiles = static_cast<long long>(ceil_div(args.n, kRows)) * a.m_tiles;
  // The number of slices by what they take: a slice's blocks, the meeting (the more slices, the fewer sums a CTA adds),
  // and 1 to 2.5 us for the second CTAs of the SMs, which start a microsecond later and share the rest; no second wave
  // (64 x 2048 x 2048 on 1, 2, 4, 6 and, more clusters than fit at once, 8 slices 8.9, 8.3, 6.6, 5.9 and 6.8 us; 64 x
  // 4100 x 14300 on 4 and, two CTAs an SM, 6 and 8 18.0, 16.9 and 15.4; 45 rows x 28672 x 4096, two CTAs an SM, on 1, 2
  // and, more waves, 4 24, 38 and 46).
  constexpr int kShare[kMaxSplit] = {0, 100, 82, 73, 62, 51, 47, 42};  // hundredths of kMeet
  long long best = -1;
  for (int S = 1; S <= std::min(kMaxSplit, blocks); ++S) {
    if (S > 1 && (tiles * S > 2 * dev.num_sms || dev.clusters[S] == 0)) continue;
    const long long cost = static_cast<long long>(ceil_div(blocks, S)) * C::kBlock + C::kMeet * kShare[S - 1] / 100 +
                           (tiles > dev.clusters[S] ? C::kTwo : 0);
    if (best < 0 || cost < best) best = cost, a.split = S;
  }
  a.stages = tiles <= dev.clusters[a.split] ? C::kAlone : C::kStages;
  return launch_pdl(fp8_skinny_kernel<NT>, dim3(static_cast<unsigned>(tiles * a.split)), dim3(kThreads),
                    a.stages * C::kStage + C::kRest, s, a.split, tmA, tmB, a);
}

template <bool SPLIT, int TN>
cudaError_t wide(const void* a, long long lda, const void* b, long long ldb, const Fp8MatmulArgs& args, int split,
                 const Fp8MatmulDevice& dev, cudaStream_t s, std::string* err) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(args.c) | static_cast<uintptr_t>(2 * args.ldc);
  const int c_align = (at & 15u) == 0 ? 16 : (at & 7u) == 0 ? 8 : (at & 3u) == 0 ? 4 : 2;
  WideArgs w{args, split, ceil_div(args.m, kRows), 0, 0, c_align};
  w.tiles = ceil_div(args.n, TN) * w.m_tiles;
  w.stages = w.tiles <= dev.clusters[split] ? Wide<TN>::kAlone : Wide<TN>::kStages;
  CUtensorMap tmA, tmB, tmC;
  if (!encode_tmap_u8(&tmA, a, args.m, args.k, kRows, err, lda) ||
      !encode_tmap_u8(&tmB, b, args.n, args.k, TN, err, ldb))
    return cudaErrorInvalidValue;
  if (SPLIT || c_align != 16) tmC = tmA;  // (not used)
  else if (!encode_tmap_out(&tmC, args.c, args.m, args.n, args.ldc, err)) return cudaErrorInvalidValue;
  const int grid = SPLIT ? w.tiles * split : std::min(w.tiles, Wide<TN>::kCtas * dev.num_sms);
  return launch_pdl(fp8_wide_kernel<SPLIT, TN>, dim3(grid), dim3(Wide<TN>::kThreads),
                    w.stages * Wide<TN>::kStage + Wide<TN>::kRest, s, split, tmA, tmB, tmC, w);
}

// Width and slices of the wide tiles, by what they take in hundredths of a microsecond: a K block of a CTA, times the
// blocks of its slice and the waves of CTAs, and the meeting of the slices.  A block takes 0.38 us in 256 columns, 0.3
// in 128 and 0.47 in 128 with two CTAs on an SM (1000 x 4096 x 7168 25 and 30 us, 256 x 7168 x 2048 10.8 and 8.8);
// slices are cut where every CTA has an SM to itself, at once (362 x 4100 x 14300 in 256 columns on 1 and 2 slices 48
// and 31 us, in 128 on 2 and 3 slices, two CTAs an SM, 41 and 46; 400 x 2048 x 7168 in 128 on 2 and, two CTAs an SM, 3
// 14.8 and 18.9).
cudaError_t wide(const void* a, long long lda, const void* b, long long ldb, const Fp8MatmulArgs& args,
                 const Fp8MatmulDevice& dev, cudaStream_t s, std::string* err) {
  const int num_sms = dev.num_sms;
  constexpr int kMeet[2][kWideSplit] = {{0, 390, 500, 580}, {0, 230, 300, 360}};
  const long long blocks = ceil_div(args.k, kFp8BK), m_tiles = ceil_div(args.m, kRows);
  bool narrow = false;
  int split = 1;
  long long best = -1;
  for (int half = 0; half < 2; ++half) {
    const long long tiles = m_tiles * ceil_div(args.n, half ? 128 : 256);
    for (int S = 1; S <= kWideSplit && S <= blocks && (S == 1 || tiles <= dev.clusters[S]); ++S) {
      const bool two = half && tiles > num_sms;
      const long long wave = two ? 2 * num_sms : num_sms, block = !half ? 38 : two ? 47 : 30;
      const long long cost = (tiles * S + wave - 1) / wave * ((blocks + S - 1) / S) * block + kMeet[half][S - 1];
      if (best < 0 || cost < best) best = cost, narrow = half != 0, split = S;
    }
  }
  if (narrow)
    return split > 1 ? wide<true, 128>(a, lda, b, ldb, args, split, dev, s, err)
                     : wide<false, 128>(a, lda, b, ldb, args, 1, dev, s, err);
  return split > 1 ? wide<true, 256>(a, lda, b, ldb, args, split, dev, s, err)
                   : wide<false, 256>(a, lda, b, ldb, args, 1, dev, s, err);
}

}  // namespace

cudaError_t fp8_matmul_device(Fp8MatmulDevice* dev) {
  cudaError_t e = cudaSuccess;
  auto set = [&](auto* f, size_t bytes) {
    if (e == cudaSuccess)
      e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
  };
  set(fp8_skinny_kernel<16>, Skinny<16>::kAlone * Skinny<16>::kStage + Skinny<16>::kRest);
  set(fp8_skinny_kernel<32>, Skinny<32>::kAlone * Skinny<32>::kStage + Skinny<32>::kRest);
  set(fp8_skinny_kernel<64>, Skinny<64>::kAlone * Skinny<64>::kStage + Skinny<64>::kRest);
  // (a register split that the launch's registers do not cover would wait for ever)
  auto split = [&](auto* f, int regs) {
    cudaFuncAttributes at{};
    if (e == cudaSuccess) e = cudaFuncGetAttributes(&at, f);
    if (e == cudaSuccess && at.numRegs < regs) e = cudaErrorInvalidConfiguration;
  };
  split(fp8_wide_kernel<false, 128>, Wide<128>::kLaunchRegs);
  split(fp8_wide_kernel<true, 128>, Wide<128>::kLaunchRegs);
  split(fp8_wide_kernel<false, 256>, Wide<256>::kLaunchRegs);
  split(fp8_wide_kernel<true, 256>, Wide<256>::kLaunchRegs);
  set(fp8_wide_kernel<false, 128>, Wide<128>::kAlone * Wide<128>::kStage + Wide<128>::kRest);
  set(fp8_wide_kernel<true, 128>, Wide<128>::kAlone * Wide<128>::kStage + Wide<128>::kRest);
  set(fp8_wide_kernel<false, 256>, Wide<256>::kAlone * Wide<256>::kStage + Wide<256>::kRest);
  set(fp8_wide_kernel<true, 256>, Wide<256>::kAlone * Wide<256>::kStage + Wide<256>::kRest);
  // clusters that are resident at once with one CTA an SM
  dev->clusters[1] = dev->num_sms;
  for (int S = 2; S <= kMaxSplit && e == cudaSuccess; ++S) {
    cudaLaunchConfig_t c{};
    c.gridDim = dim3(S * dev->num_sms);
    c.blockDim = dim3(Wide<256>::kThreads);
    c.dynamicSmemBytes = Wide<256>::kStages * Wide<256>::kStage + Wide<256>::kRest;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = S;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    c.attrs = at;
    c.numAttrs = 1;
    e = cudaOccupancyMaxActiveClusters(&dev->clusters[S], fp8_wide_kernel<true, 256>, &c);
  }
  return e;
}

cudaError_t fp8_matmul_launch(const void* a, long long lda, const void* b, long long ldb, const Fp8MatmulArgs& args,
                              const Fp8MatmulDevice& dev, cudaStream_t s, std::string* err) {
  // More than 64 rows go to the wide tiles, unless there are so few narrow tiles that they can be cut into eight slices
  // (64 rows of A at a time; wide / narrow, us: 65 x 512 x 2048 8.0 / 5.4, 128 x 2048 x 7168 12.9 / 10.4, 65 x 2048 x
  // 14336 17.5 / 13.2; but with twice as many tiles 200 x 2048 x 7168 13.3 / 14.0, and 65 x 1024 x 1024, eight blocks,
  // no faster)
  const long long narrow = static_cast<long long>(ceil_div(args.m, 64)) * ceil_div(args.n, kRows);
  if (args.m > 64 && (narrow * kMaxSplit > 2 * dev.num_sms || args.k <= 15 * kFp8BK))
    return wide(a, lda, b, ldb, args, dev, s, err);
  CUtensorMap tmA, tmB;
  const int nt = args.m <= 16 ? 16 : args.m <= 32 ? 32 : 64;
  if (!encode_tmap_u8(&tmA, a, args.m, args.k, nt, err, lda) ||
      !encode_tmap_u8(&tmB, b, args.n, args.k, kRows, err, ldb))
    return cudaErrorInvalidValue;
  switch (nt) {
    case 16: return skinny<16>(tmA, tmB, args, dev, s);
    case 32: return skinny<32>(tmA, tmB, args, dev, s);
    default: return skinny<64>(tmA, tmB, args, dev, s);
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

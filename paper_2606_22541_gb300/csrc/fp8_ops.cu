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
// A lane holds 8 consecutive columns, 16 lanes a group of 128; a warp works on
// 256 columns of a row at a time, kAhead of them on their way.  W: columns per
// load (8, 4 or 1, by the alignment of the rows).
constexpr int kAhead = 4;
constexpr int kQuantThreads = 256;

template <int W>
__device__ __forceinline__ void load8(const uint16_t* p, int left, uint32_t (&v)[4]) {
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

__device__ __forceinline__ float swiglu(float g, float u) { return g / (1.0f + __expf(-g)) * u; }

template <bool SWIGLU, int W>
__global__ void __launch_bounds__(kQuantThreads) fp8_quantize_kernel(const uint16_t* x, const uint16_t* u, int rows,
                                                                    int cols, long long ld, uint8_t* q, long long ldq,
                                                                    float* s, long long lds, bool wide_q) {
  pdl_wait();
  pdl_launch();
  const int lane = threadIdx.x & 31;
  // (a tensor of 2^31 parts would not fit the GPU)
  const uint32_t parts = (static_cast<uint32_t>(cols) + 255) / 256;  // of a row
  const uint32_t total = static_cast<uint32_t>(rows) * parts;
  const uint32_t warps = gridDim.x * (kQuantThreads / 32);
  for (uint32_t i0 = blockIdx.x * (kQuantThreads / 32) + (threadIdx.x >> 5); i0 < total; i0 += warps * kAhead) {
    uint32_t g[kAhead][4], up[kAhead][4];
#pragma unroll
    for (int r = 0; r < kAhead; ++r) {
      const uint32_t i = i0 + r * warps;
      g[r][0] = g[r][1] = g[r][2] = g[r][3] = 0u;
      up[r][0] = up[r][1] = up[r][2] = up[r][3] = 0u;
      if (i < total) {
        const long long row = i / parts;
        const int c = static_cast<int>(i % parts) * 256 + lane * 8;
        if (c < cols) {
          load8<W>(x + row * ld + c, cols - c, g[r]);
          if constexpr (SWIGLU) load8<W>(u + row * ld + c, cols - c, up[r]);
        }
      }
    }
#pragma unroll
    for (int r = 0; r < kAhead; ++r) {
      const uint32_t i = i0 + r * warps;
      if (i >= total) break;
      const long long row = i / parts;
      const int c = static_cast<int>(i % parts) * 256 + lane * 8;
      float f[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        f[2 * j] = bf16_lo(g[r][j]);
        f[2 * j + 1] = bf16_hi(g[r][j]);
        if constexpr (SWIGLU) {
          f[2 * j] = swiglu(f[2 * j], bf16_lo(up[r][j]));
          f[2 * j + 1] = swiglu(f[2 * j + 1], bf16_hi(up[r][j]));
        }
      }
      float am = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) am = fmaxf(am, fabsf(f[j]));
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) am = fmaxf(am, __shfl_xor_sync(kFull, am, o));
      const GroupScale gs(am);
      if (c >= cols) continue;
      const uint32_t w[2] = {e4m3x4(gs, f[0], f[1], f[2], f[3]), e4m3x4(gs, f[4], f[5], f[6], f[7])};
      uint8_t* out = q + row * ldq + c;
      if (wide_q && cols - c >= 8) {
        *reinterpret_cast<uint2*>(out) = make_uint2(w[0], w[1]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < cols - c) out[j] = static_cast<uint8_t>(w[j >> 2] >> (8 * (j & 3)));
      }
      if ((lane & 15) == 0) s[row * lds + (c >> 7)] = gs.s;
    }
  }
}

// ------------------------------------------------------------ product, weights as the M operand
// A tile is 128 rows of B (M; one row of scale blocks) and NT rows of A (N); a
// cluster of S CTAs shares a tile, each with a slice of K.  Every 128-wide K block
// is multiplied into one of the TMEM partials, which the epilogue warps add, times
// the block's scales, into registers; the slices' sums meet in distributed shared
// memory, each CTA adding those of NT / S columns in rank order.
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
  static constexpr int kStages = NT <= 32 ? 5 : NT == 64 ? 4 : 3;  // about 100 KB: two CTAs an SM
  static constexpr int kPartials = NT <= 32 ? 4 : 256 / NT;
  static constexpr uint32_t kTmem = NT * kPartials;
  static constexpr bool kAlias = NT >= 64;  // the slices' sums take the ring's place
  static constexpr int kSums = kRows * NT * 4;
  static constexpr int kBars = 2 * kStages + 2 * kPartials + 1;
  static constexpr size_t kSmem = kStages * kStage + (kAlias ? 0 : kSums) + 2 * NT * 4 + 8 * kBars + 16;
  static_assert(!kAlias || kSums <= kStages * kStage, "the sums fit the ring");
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
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
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
  float* sums = reinterpret_cast<float*>(smem_raw + (C::kAlias ? 0 : C::kStages * C::kStage));  // [src][column][row]
  float* scales = reinterpret_cast<float*>(smem_raw + C::kStages * C::kStage + (C::kAlias ? 0 : C::kSums));  // [2][NT]
  uint64_t* bars = reinterpret_cast<uint64_t*>(scales + 2 * NT);
  const uint32_t bar0 = smem_u32(bars);
  auto full = [&](int i) { return bar0 + 8u * i; };
  auto empty = [&](int i) { return bar0 + 8u * (C::kStages + i); };
  auto pfull = [&](int i) { return bar0 + 8u * (2 * C::kStages + i); };
  auto pempty = [&](int i) { return bar0 + 8u * (2 * C::kStages + C::kPartials + i); };
  const uint32_t drain = bar0 + 8u * (C::kBars - 1);
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
    *abort_flag = aligned ? 0 : 1;
    fence_barrier_init();
    tma_prefetch_desc(&tmA);
    tma_prefetch_desc(&tmB);
    if (!aligned) record_status(p.status, ST_SMEM_ALIGN);
  } else if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), C::kTmem);
    tmem_relinquish();
  }
  pdl_wait();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  auto give_up = [&]() {
    *abort_flag = 1;
    record_status(p.status, ST_WAIT_TIMEOUT);
  };
  float acc[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) acc[i] = 0.f;

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
    const int q = warp & 3;
    const int tid = threadIdx.x - 64;
    const uint32_t lanes = tmem_base + (static_cast<uint32_t>(q * 32) << 16);
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
    bool ok = aligned;
#pragma unroll
    for (int i = 0; i < kLead; ++i) ahead(i, kb0 + i);
    Ring<C::kPartials> t;
    for (int k4 = kb0; k4 < kb1; k4 += kLead) {
#pragma unroll
      for (int i = 0; i < kLead; ++i) {
        const int kb = k4 + i;
        if (kb >= kb1) break;
        float* sc = scales + (i & 1) * NT;
        if (tid < NT) sc[tid] = na[i] * nb[i];
        ahead(i, kb + kLead);
        asm volatile("bar.sync 1, 128;" ::: "memory");  // every warp comes here for every block, whatever its waits said
        ok = ok && __all_sync(kFull, mbar_wait(pfull(t.s), t.phase, abort_flag));
        if (ok) {
          tc_fence_after();
#pragma unroll
          for (int c0 = 0; c0 < NT; c0 += 16) {
            uint32_t v[16];
            tmem_ld16(lanes + t.s * NT + c0, v);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float4 f = *reinterpret_cast<const float4*>(sc + c0 + 4 * j);
              acc[c0 + 4 * j] = fmaf(f.x, __uint_as_float(v[4 * j]), acc[c0 + 4 * j]);
              acc[c0 + 4 * j + 1] = fmaf(f.y, __uint_as_float(v[4 * j + 1]), acc[c0 + 4 * j + 1]);
              acc[c0 + 4 * j + 2] = fmaf(f.z, __uint_as_float(v[4 * j + 2]), acc[c0 + 4 * j + 2]);
              acc[c0 + 4 * j + 3] = fmaf(f.w, __uint_as_float(v[4 * j + 3]), acc[c0 + 4 * j + 3]);
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(pempty(t.s));
        }
        t.advance();
      }
    }
    if (!ok && lane == 0 && aligned) give_up();
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, C::kTmem);
  }

  // ---- out
  __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.c);
  if (S == 1) {
    if (warp >= 2) {
      const int n = row0 + (warp & 3) * 32 + lane;
#pragma unroll
      for (int c = 0; c < NT; ++c)
        if (n < p.n && tok0 + c < p.m) out[static_cast<long long>(tok0 + c) * p.ldc + n] = __float2bfloat16_rn(acc[c]);
    }
    return;
  }
  const int cols = NT / S;  // that this CTA adds
  cluster_sync();           // the ring's place may be written (and every CTA of the cluster has started)
  if (warp >= 2) {
    const int r = (warp & 3) * 32 + lane;
#pragma unroll
    for (int c = 0; c < NT; ++c) {
      const int to = c / cols;
      const uint32_t at = map_rank(smem_u32(sums + (rank * cols + (c - to * cols)) * kRows + r), static_cast<uint32_t>(to));
      if (tok0 + c < p.m) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(acc[c]) : "memory");
    }
  }
  cluster_sync();
  for (int i = threadIdx.x; i < cols * kRows; i += kThreads) {
    const int c = i / kRows, t = tok0 + rank * cols + c, n = row0 + i % kRows;
    if (t >= p.m || n >= p.n) continue;
    float v = sums[i];
    for (int s = 1; s < S; ++s) v += sums[s * cols * kRows + i];
    out[static_cast<long long>(t) * p.ldc + n] = __float2bfloat16_rn(v);
  }
}

template <int NT>
cudaError_t skinny(const CUtensorMap& tmA, const CUtensorMap& tmB, const Fp8MatmulArgs& args, int num_sms,
                   cudaStream_t s) {
  const int blocks = ceil_div(args.k, kFp8BK);
  SkinnyArgs a{args, 1, ceil_div(args.m, NT)};
  const long long tiles = static_cast<long long>(ceil_div(args.n, kRows)) * a.m_tiles;
  // K slices until the tiles fill the GPU twice over, with at least four blocks each
  while (a.split < kMaxSplit && tiles * a.split < 2 * num_sms && blocks / (2 * a.split) >= 4) a.split *= 2;
  return launch_pdl(fp8_skinny_kernel<NT>, dim3(static_cast<unsigned>(tiles * a.split)), dim3(kThreads),
                    Skinny<NT>::kSmem, s, a.split, tmA, tmB, a);
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
  set(fp8_skinny_kernel<128>, Skinny<128>::kSmem);
  return e;
}

cudaError_t fp8_matmul_launch(const void* a, long long lda, const void* b, long long ldb, const Fp8MatmulArgs& args,
                              int num_sms, cudaStream_t s, std::string* err) {
  CUtensorMap tmA, tmB;
  const int nt = args.m <= 16 ? 16 : args.m <= 32 ? 32 : args.m <= 64 ? 64 : 128;
  if (!encode_tmap_u8(&tmA, a, args.m, args.k, nt, err, lda)) {
    *err = "a: " + *err;
    return cudaErrorInvalidValue;
  }
  if (!encode_tmap_u8(&tmB, b, args.n, args.k, kRows, err, ldb)) {
    *err = "b: " + *err;
    return cudaErrorInvalidValue;
  }
  switch (nt) {
    case 16: return skinny<16>(tmA, tmB, args, num_sms, s);
    case 32: return skinny<32>(tmA, tmB, args, num_sms, s);
    case 64: return skinny<64>(tmA, tmB, args, num_sms, s);
    default: return skinny<128>(tmA, tmB, args, num_sms, s);
  }
}

cudaError_t launch_fp8_quantize(const void* x, const void* u, int rows, int cols, long long ld, void* q,
                                long long ldq, float* s, long long lds, cudaStream_t st) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(u) | static_cast<uintptr_t>(2 * ld);
  const bool wide_q = ((reinterpret_cast<uintptr_t>(q) | static_cast<uintptr_t>(ldq)) & 7u) == 0;
  const long long parts = static_cast<long long>(rows) * ceil_div(cols, 256);
  const unsigned grid = static_cast<unsigned>(std::min<long long>((parts + 7) / 8, 152 * 8));
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

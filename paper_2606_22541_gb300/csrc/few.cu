// The whole MoE layer for a few tokens (1 .. kFewTokens): two kernels.
//
//   out[t] = sum_j w[t,j] Wd_e (silu(Wg_e x_t) * (Wu_e x_t)) + shared expert,  e = idx[t,j]
//
// With one to a few rows per expert every weight is used once, so the layer is a
// stream of the active experts' matrices (three of H x I each) and nothing else
// matters but that this stream never stops.
//
// few_logits_kernel: router logits with mma.sync, 16 experts and a slice of K per
// CTA, as planes of partial sums; the hidden states as an image of the operand
// tiles (128-byte rows, 128-byte swizzle; e4m3 with scales for FP8), which the
// second kernel copies to shared memory as they are; and zeroed counters.
//
// few_ffn_kernel (one CTA per SM): a list of work items, gate/up tiles of all
// experts, then down tiles, then the outputs, claimed one by one from a counter.  An item is a
// 256-row weight tile (a box per k-step, 32 KB, as the handle packs them) over
// a slice of K.  The weights are the M operand of the MMA and all tokens the N
// operand, so a tile costs the same whatever its rows; the tensor core is idle
// most of the time.  The shared expert, which every token meets, comes first:
// while its weights stream, every CTA learns the routing (it gates a few tokens
// for itself, one thread per expert) and lists the active experts, each with the set of its tokens as a
// 64-bit mask, so that a row's place in its expert is a popcount.
//  - gate/up: the partial sums of a K slice go to the workspace in fp32; the
//    last slice of a tile to arrive adds them in slice order, applies SwiGLU
//    and writes h as an operand image: e4m3 with scales, or, for BF16, as the
//    sum of two bf16 (the value and what its rounding left), since N has room:
//    h keeps 16 bits at no cost.
//  - down: a tile waits until its expert's h is complete; its partial sums are
//    fp32.
//  - combine: 256 channels of one token, or from 8 tokens on of eight, once the
//    output tile's partial sums are complete: the experts' in slot order, then
//    the shared expert's.
// Sums are taken in a fixed order, so a call gives the same bits each time.
// An item waits only for items claimed before it, by CTAs that are running,
// so the launch needs no co-residency to make progress.
//
// What bounds it: the weight stream, after 10 us of start (4 to 7 of them the
// logits, up to 6 the gating from 4 tokens on) that the shared expert's weights
// fill where there is one, and 2 to 4 us of last sums at the end.  One token:
// Mixtral's shape (two experts of 176 M parameters) 108.6 us, 6.5 TB/s;
// DeepSeek-V3's 113 us, 7.0 TB/s (the stream alone passes the rate of a plain
// copy), in e4m3 64.8 us, 6.2 TB/s; 61 tokens of the latter, 209 experts, 1300 to
// 1327 us, 7.0 to 7.1 TB/s.
#include "common.cuh"
#include "e4m3.cuh"
#include "few.h"
#include "internal.h"

#include <math_constants.h>

#include <algorithm>
#include <cstddef>

namespace asap {

namespace {

constexpr unsigned kFull = 0xffffffffu;

// ------------------------------------------------------------ operand images
// A k-step's rows: R rows of 128 bytes, 16-byte chunk c of row r at chunk
// c ^ (r % 8) (the 128-byte swizzle of a tile that starts on a 1024-byte
// boundary), then, for FP8, R fp32 scales, up to a multiple of 16 bytes.
template <bool FP8>
__host__ __device__ constexpr int step_bytes(int rows) {
  return rows * 128 + (FP8 ? (rows + 3) / 4 * 16 : 0);
}
__device__ __forceinline__ int swizzled(int row, int byte) {
  return row * 128 + ((((byte >> 4) ^ (row & 7)) << 4) | (byte & 15));
}

// u / d for 0 <= u < 2^21 from r = 1 / d rounded to fp32 (u + 1/2 is at least 1/(2 d) from a multiple of d, in
// units of d, and the product's error is below 2^-23 u / d).
__device__ __forceinline__ int quick_div(int u, float r) { return static_cast<int>((u + 0.5f) * r); }

// Float as an unsigned that orders the same way (-0 as +0).
__device__ __forceinline__ uint32_t ordered(float f) {
  const uint32_t u = __float_as_uint(f + 0.0f);
  return (u >> 31) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t o) { return __uint_as_float((o >> 31) ? o & 0x7fffffffu : ~o); }

// ------------------------------------------------------------ logits
// Hidden states as operand image.
template <bool FP8>
__device__ __forceinline__ void write_image(const FewArgs& a, int thread, int threads) {
  constexpr int kAhead = 4;
  const int V = a.H / 8;  // 16-byte vectors of a row
  const int total = a.n * V;
  const uint4* x = static_cast<const uint4*>(a.x);
  // FP8: 16 threads a group of 128 channels (total and the stride are multiples of 32: a warp stays together)
  for (int i0 = thread; i0 < total; i0 += kAhead * threads) {
    uint4 d[kAhead];
#pragma unroll
    for (int r = 0; r < kAhead; ++r) {
      const int i = i0 + r * threads;
      d[r] = i < total ? ld_dep(x + i) : make_uint4(0, 0, 0, 0);  // (rows follow one another)
    }
#pragma unroll
    for (int r = 0; r < kAhead; ++r) {
      const int i = i0 + r * threads;
      if (i >= total) break;
      const int t = i / V, v = i - t * V;
      if constexpr (!FP8) {
        *reinterpret_cast<uint4*>(a.ximg + static_cast<long long>(v >> 3) * step_bytes<false>(a.n) +
                                  swizzled(t, (v & 7) * 16)) = d[r];
      } else {
        const float f[8] = {bf16_lo(d[r].x), bf16_hi(d[r].x), bf16_lo(d[r].y), bf16_hi(d[r].y),
                            bf16_lo(d[r].z), bf16_hi(d[r].z), bf16_lo(d[r].w), bf16_hi(d[r].w)};
        float am = 0.f;
#pragma unroll
        for (int u = 0; u < 8; ++u) am = fmaxf(am, fabsf(f[u]));
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) am = fmaxf(am, __shfl_xor_sync(kFull, am, o));
        const GroupScale gs(am);
        const uint2 q = make_uint2(e4m3x4(gs, f[0], f[1], f[2], f[3]), e4m3x4(gs, f[4], f[5], f[6], f[7]));
        uint8_t* step = a.ximg + static_cast<long long>(v >> 4) * step_bytes<true>(a.n);
        *reinterpret_cast<uint2*>(step + swizzled(t, (v & 15) * 8)) = q;
        if ((v & 15) == 0) *reinterpret_cast<float*>(step + a.n * 128 + t * 4) = gs.s;
      }
    }
  }
}

constexpr int kLogitWarps = 8;
constexpr int kLogitThreads = 32 * kLogitWarps;
constexpr int kUnits = 4;    // K units (32 channels) of a warp on their way at a time
constexpr int kLogitSlices = 8;
// CTA (tile, slice): logits of 16 experts (M) over a slice of K for all tokens (8 per MMA, N).  Its warps take
// every eighth K unit; thread (g, q) feeds 16 bytes of a row to two MMAs, whose K order both operands share.
// CTAs past the router's help with the rest.
// NJ: groups of 8 tokens at most.
template <bool FP8, int NJ>
__global__ void __launch_bounds__(kLogitThreads) few_logits_kernel(const __grid_constant__ FewArgs a) {
  pdl_launch();  // the second kernel may come up meanwhile
  __shared__ float part[kLogitWarps][8 * NJ][16];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int E = a.gate.n_experts, n = a.n;
  const int slice = blockIdx.x % kLogitSlices, tile = blockIdx.x / kLogitSlices;
  const int g = lane >> 2, q = lane & 3;
  const int V = a.H / 8, units = a.H / 32;
  const int u0 = units * slice / kLogitSlices, u1 = units * (slice + 1) / kLogitSlices;
  const int e0 = tile * 16 + g, e1 = e0 + 8;
  const uint4 zero = make_uint4(0, 0, 0, 0);
  uint4 w0[kUnits], w1[kUnits];
  auto load_weights = [&](int layer, int ub) {
    const uint4* __restrict__ wr = static_cast<const uint4*>(a.lref.table[layer].router_w);
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int u = ub + kLogitWarps * i, v = 4 * u + q;
      w0[i] = u < u1 && e0 < E ? __ldg(wr + static_cast<long long>(e0) * V + v) : zero;
      w1[i] = u < u1 && e1 < E ? __ldg(wr + static_cast<long long>(e1) * V + v) : zero;
    }
  };
  // The first weights are on their way before what the kernels in front write may be read; a layer id that
  // turns out to have been written since has them loaded again.
  const int early = load_layer(a.lref.layer, a.lref.n_layers, a.status, false);
  load_weights(early, u0 + warp);
  // (and the hidden states in L2, in front of the expert weights that the second kernel fetches meanwhile:
  // behind these the logits of 61 tokens took 19 us)
  for (long long i = (blockIdx.x * kLogitThreads + threadIdx.x) * 128ll; i < 2ll * n * a.H; i += gridDim.x * kLogitThreads * 128ll)
    asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const uint8_t*>(a.x) + i));
  pdl_wait();
  if (tile * 16 < E) {
    const int layer = a.fixed_layer ? early
                                    : load_layer(a.lref.layer, a.lref.n_layers, a.status, blockIdx.x == 0 && threadIdx.x == 0);
    const uint4* x = static_cast<const uint4*>(a.x);
    float c[NJ][4];
#pragma unroll
    for (int j = 0; j < NJ; ++j) c[j][0] = c[j][1] = c[j][2] = c[j][3] = 0.f;
    for (int ub = u0 + warp; ub < u1; ub += kLogitWarps * kUnits) {
      if (layer != early || ub != u0 + warp) load_weights(layer, ub);
      constexpr int kGroups = NJ < 4 ? NJ : 4;  // token groups on their way at a time
#pragma unroll
      for (int j0 = 0; j0 < NJ; j0 += kGroups) {
        uint4 xv[kGroups][kUnits];
#pragma unroll
        for (int j = 0; j < kGroups; ++j)
#pragma unroll
          for (int i = 0; i < kUnits; ++i) {
            const int t = 8 * (j0 + j) + g, u = ub + kLogitWarps * i;
            xv[j][i] = u < u1 && t < n ? ld_dep(x + static_cast<long long>(t) * V + 4 * u + q) : zero;
          }
#pragma unroll
        for (int j = 0; j < kGroups; ++j)
#pragma unroll
          for (int i = 0; i < kUnits; ++i) {
            mma_bf16_16816(c[j0 + j], w0[i].x, w1[i].x, w0[i].y, w1[i].y, xv[j][i].x, xv[j][i].y);
            mma_bf16_16816(c[j0 + j], w0[i].z, w1[i].z, w0[i].w, w1[i].w, xv[j][i].z, xv[j][i].w);
          }
      }
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = 8 * j + 2 * q + (i & 1);
        if (t < n) part[warp][t][g + 8 * (i >> 1)] = c[j][i];
      }
    __syncthreads();
    for (int i = threadIdx.x; i < n * 16; i += kLogitThreads) {
      const int t = i / 16, e = tile * 16 + i % 16;
      float sum = part[0][t][i % 16];
#pragma unroll
      for (int w = 1; w < kLogitWarps; ++w) sum += part[w][t][i % 16];
      if (e < E) a.logits[(slice * n + t) * E + e] = sum;
    }
  }
  const int thread = blockIdx.x * kLogitThreads + threadIdx.x, threads = gridDim.x * kLogitThreads;
  for (int i = thread; i < a.n_counters; i += threads) a.counters[i] = 0;
  write_image<FP8>(a, thread, threads);
}

// ------------------------------------------------------------ expert FFN
constexpr int kWBytes = 256 * 128;  // weight box
constexpr int kEpiWarps = 8;
constexpr int kEpiThreads = 32 * kEpiWarps;
constexpr int kThreads = 32 * (4 + kEpiWarps);
constexpr int kQ = 6;               // items in flight in a CTA
constexpr int kQReaders = 3 + kEpiWarps;
constexpr uint32_t kTmemCols = 512;
constexpr int kMaxPartials = 8;     // FP8: TMEM partials of 2 x NT columns
constexpr int kAccs = 2;            // BF16: accumulators of 2 x 128 columns

struct FewItem {
  bool down, combine, shared;
  int j;           // index among the active experts
  int tile;        // 256-row weight tile of the expert's matrix
  int slice, kb0, kb1;
  int tokens;      // of the expert
  int rows;        // operand rows of a k-step
  int n;           // N of the MMA
  int start;       // the expert's first row among the routed rows
  int ticket;      // counter of the gate/up or output tile
  int arrivals;    // that complete it
  int token;       // combine
  unsigned long long mask;
};

struct FewGate {  // of one token
  uint32_t key[kMaxExperts];
  float two[2][32];        // a group's two best selection scores
  unsigned long long cand[kEpiWarps * kMaxTopK];
  float val[kEpiWarps * kMaxTopK];
  uint32_t top[kEpiWarps];
  float sum[kEpiWarps];
  int slot_e[kMaxTopK];
  float slot_v[kMaxTopK];
  int claim;
};

struct FewSmem {  // behind the rings
  alignas(16) uint64_t bar[2 * kFewMaxStages + 2 * kFewMaxStages + 2 * kMaxPartials + 3 * kQ + 2];
  int q[kQ];
  uint32_t tmem;
  int abort;
  int active;
  int items;
  int warp_total[kEpiWarps];
  int expert[kMaxExperts], start[kMaxExperts], quads[kMaxExperts];
  unsigned long long mask[kMaxExperts];
  int pos[kFewTokens * kMaxTopK];
  float w[kFewTokens * kMaxTopK];
  float bias[kMaxExperts];  // of the router's selection
  FewGate gate;
  int first_row[kMaxExperts];               // of expert e
  unsigned long long mask_of[kMaxExperts];
  alignas(16) float sum[kEpiWarps][256];    // combine; accessed as float4
};
static_assert(sizeof(FewSmem) <= kFewSmemState, "shared memory budget");
static_assert(offsetof(FewSmem, sum) % 16 == 0, "float4 accesses");

template <bool FP8>
__device__ __forceinline__ FewItem decode(const FewArgs& a, const FewSmem& s, int item) {
  FewItem T{};
  const int tI = a.I / 128, tS = a.Is / 128, tH = a.H / 256;
  // (items below first_routed do not need the routing, which may not be there yet)
  const bool early = item < a.first_routed;
  const int active = early ? 0 : s.active;
  const int gu = (tS + active * tI) * a.s1;  // gate/up items
  const int arrivals = active * a.s2 + (a.Is ? a.s2s : 0);
  const int dn = tH * arrivals;              // down items
  T.down = !early && item >= gu;
  int kit, sl;
  if (!T.down) {
    const int t = quick_div(item, a.r_s1);
    T.slice = item - t * a.s1;
    T.shared = t < tS;
    T.j = T.shared ? 0 : quick_div(t - tS, a.r_tI);
    T.tile = T.shared ? t : (t - tS) - T.j * tI;
    T.arrivals = a.s1;
    T.ticket = 1 + t;
    kit = a.H / (FP8 ? 128 : 64);
    sl = a.s1;
  } else {
    int u = item - gu;
    T.arrivals = arrivals;
    if (u >= dn) {
      u -= dn;
      T.combine = true;
      const int group = quick_div(u, a.r_tH);
      T.token = group * a.out_tokens;
      T.tile = u - group * tH;
      T.ticket = a.down_tickets + T.tile;
      return T;
    }
    const int sh = a.Is ? tH * a.s2s : 0;
    T.shared = u < sh;
    if (!T.shared) u -= sh;
    sl = T.shared ? a.s2s : a.s2;
    T.j = T.shared ? 0 : quick_div(u, a.r_down);
    u -= T.j * tH * sl;
    T.tile = quick_div(u, T.shared ? a.r_s2s : a.r_s2);
    T.slice = u - T.tile * sl;
    T.ticket = a.down_tickets + T.tile;
    kit = (T.shared ? a.Is : a.I) / (FP8 ? 128 : 64);
  }
  const float r_sl = T.down ? (T.shared ? a.r_s2s : a.r_s2) : a.r_s1;
  T.kb0 = quick_div(kit * T.slice, r_sl);
  T.kb1 = quick_div(kit * (T.slice + 1), r_sl);
  T.mask = T.shared ? (a.n == 64 ? ~0ull : (1ull << a.n) - 1) : s.mask[T.j];
  T.tokens = T.shared ? a.n : __popcll(T.mask);
  T.start = T.shared ? 0 : s.start[T.j];
  T.rows = T.down ? T.tokens : a.n;
  T.n = round_up_dev(T.down && !FP8 ? 2 * round_up_dev(T.rows, 8) : T.rows, 16);
  return T;
}

// The h image of an expert: its first byte (the shared expert's rows first, then the active experts'; FP8:
// quads[j] groups of four scales before expert j's).  A k-step of BF16 holds the values' rows, then the rows of
// what their rounding left.
template <bool FP8>
__device__ __forceinline__ uint8_t* h_image(const FewArgs& a, const FewSmem& s, const FewItem& T) {
  if (T.shared) return a.himg;
  const long long kit = a.I / (FP8 ? 128 : 64), kits = a.Is / (FP8 ? 128 : 64);
  return a.himg + kits * step_bytes<FP8>(FP8 ? a.n : 2 * a.n) +
         kit * (FP8 ? s.start[T.j] * 128 + s.quads[T.j] * 16 : s.start[T.j] * 256);
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}
constexpr int kPrefetchBoxes = 1344;  // of 32 KB: 44 MB, what HBM delivers until the routed experts are known

__device__ __forceinline__ void prefetch_box(const CUtensorMap* m, int y) {
  asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(reinterpret_cast<uint64_t>(m)),
               "r"(0), "r"(y)
               : "memory");
}

__device__ __forceinline__ void fence_proxy_async_all() { asm volatile("fence.proxy.async;" ::: "memory"); }
__device__ __forceinline__ int ld_acquire(const int* p) {
  int v;
  asm volatile("ld.acquire.gpu.global.b32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
// One arrival on a counter, after everything this thread has seen done (by its CTA's barriers: by the CTA).
__device__ __forceinline__ void arrive_release(int* p) {
  asm volatile("red.release.gpu.global.add.s32 [%0], 1;" ::"l"(p) : "memory");
}
__device__ __forceinline__ int arrive_acq_rel(int* p) {
  int v;
  asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
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
__device__ __forceinline__ void epi_sync() {
  __syncwarp();
  asm volatile("bar.sync 1, 256;" ::: "memory");
}
// Whether ok holds in every thread of the epilogue warps (a barrier too).
__device__ __forceinline__ bool epi_all(bool ok) {
  uint32_t r;
  __syncwarp();
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "bar.red.and.pred q, 2, 256, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"(ok ? 1u : 0u)
      : "memory");
  return r != 0;
}

// Gating of token t by the epilogue warps, one thread per expert, from the planes
// of its logits: expert (-1: none left) and weight of slot j to e[j], w[j].  The
// rules and tie-breaks of gate_kernel (route.cu).  No rounds: an expert's place is
// the number of experts in front of it, counted in its group, for groups against
// one another, in its warp, and among the warps' best.
__device__ __forceinline__ void gate_token(const FewArgs& a, FewSmem& s, int t, int warp, int lane, int tid, int* e_out,
                                           float* w_out) {
  const GateParams& p = a.gate;
  const int E = p.n_experts, k = p.top_k;
  const bool grouped = p.gating == 2, in = tid < E;
  float logit = 0.f;
  if (in) {
    float l[kLogitSlices];
#pragma unroll
    for (int r = 0; r < kLogitSlices; ++r) l[r] = __ldcg(a.logits + (r * a.n + t) * E + tid);
    logit = l[0];
#pragma unroll
    for (int r = 1; r < kLogitSlices; ++r) logit += l[r];
  }
  FewGate& g = s.gate;
  const float val = grouped ? gate_sigmoid(logit) : logit;
  const float sel = grouped ? val + s.bias[tid] : val;
  uint32_t key = in ? ordered(sel) : 0u;  // 0: may not be chosen
  if (grouped) {
    const int gsz = E / p.n_groups;
    const int grp = in ? quick_div(tid, 1.0f / static_cast<float>(gsz)) : 0, first = grp * gsz;
    g.key[tid] = key;
    epi_sync();
    int rank = 0;  // members of the group in front of this one
#pragma unroll 8
    for (int m = first; m < first + gsz; ++m) {
      const uint32_t o = g.key[m];
      rank += (o > key || (o == key && m < tid)) ? 1 : 0;
    }
    if (in && rank < 2) g.two[rank][grp] = sel;
    epi_sync();
    const float score = g.two[0][grp] + g.two[1][grp];
    int before = 0;  // groups in front of this one
#pragma unroll 4
    for (int m = 0; m < p.n_groups; ++m) {
      const float o = g.two[0][m] + g.two[1][m];
      before += (o > score || (o == score && m < grp)) ? 1 : 0;
    }
    if (before >= p.topk_groups) key = 0u;
  }
  if (p.gating == 0) {  // the softmax sum over all experts, from the largest logit
    const uint32_t mx = __reduce_max_sync(kFull, key);
    if (lane == 0) g.top[warp] = mx;
    epi_sync();
    uint32_t top = g.top[0];
#pragma unroll
    for (int w = 1; w < kEpiWarps; ++w) top = max(top, g.top[w]);
    float z = in ? expf(logit - unordered(top)) : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(kFull, z, o);
    if (lane == 0) g.sum[warp] = z;
  }
  int rank = 0;  // experts of this warp in front of this one
#pragma unroll
  for (int m = 0; m < 32; ++m) {
    const uint32_t o = __shfl_sync(kFull, key, m);
    rank += (o > key || (o == key && m < lane)) ? 1 : 0;
  }
  // the warps' first k are candidates: larger keys first, of equal ones the lower expert
  if (rank < kMaxTopK) {
    g.cand[warp * kMaxTopK + rank] =
        key == 0u ? 0ull : (static_cast<unsigned long long>(key) << 32) | static_cast<uint32_t>(kMaxExperts - 1 - tid);
    g.val[warp * kMaxTopK + rank] = val;
  }
  if (tid < kMaxTopK) g.slot_e[tid] = -1;
  epi_sync();
  if (tid < kEpiWarps * kMaxTopK) {
    const unsigned long long mine = g.cand[tid];
    int place = 0;
#pragma unroll 16
    for (int m = 0; m < kEpiWarps * kMaxTopK; ++m) place += g.cand[m] > mine ? 1 : 0;
    if (mine != 0ull && place < k) {
      g.slot_e[place] = kMaxExperts - 1 - static_cast<int>(mine & 0xffffffffu);
      g.slot_v[place] = g.val[tid];
    }
  }
  epi_sync();
  if (warp == 0) {
    const int e = lane < k ? g.slot_e[lane] : -1;
    const float num = e >= 0 ? (grouped ? g.slot_v[lane] : expf(g.slot_v[lane] - g.slot_v[0])) : 0.f;
    float den = 0.f;  // in slot order
    if (p.gating == 0) {
#pragma unroll
      for (int w = 0; w < kEpiWarps; ++w) den += g.sum[w];
    } else {
#pragma unroll
      for (int j = 0; j < kMaxTopK; ++j) den += __shfl_sync(kFull, num, j);
    }
    if (lane < k) {
      e_out[lane] = e;
      w_out[lane] = num / den * (grouped ? p.route_scale : 1.0f);
      if (e < 0) record_status(a.status, ST_BAD_EXPERT_INDEX);
    }
  }
}

// The routing of the call in every CTA, by its epilogue warps: active experts in
// increasing order, their tokens and first rows, the row and weight
// of every slot, and the number of work items.  Up to kOwnGate tokens every CTA
// gates for itself (a token takes about 1.5 us); more are gated once, claimed one
// by one, and read by every CTA when all are done (about 4 us for the round trips).
constexpr int kOwnGate = 3;
__device__ __forceinline__ bool list_experts(const FewArgs& a, FewSmem& s, int warp, int lane, int tid,
                                             volatile int* abort_flag) {
  const int k = a.gate.top_k, n = a.n;
  s.mask[tid] = 0ull;
  if (n <= kOwnGate) {
    for (int t = 0; t < n; ++t) gate_token(a, s, t, warp, lane, tid, s.pos + t * k, s.w + t * k);  // (pos: the expert, for now)
    epi_sync();
  } else {
    int* claims = a.counters + a.gate_claims;
    while (true) {
      if (tid == 0) s.gate.claim = atomicAdd(claims, 1);
      epi_sync();
      const int t = *reinterpret_cast<volatile int*>(&s.gate.claim);
      if (t >= n) break;
      gate_token(a, s, t, warp, lane, tid, a.sel_e + t * k, a.sel_w + t * k);
      if (warp == 0) {
        __syncwarp();
        if (lane == 0) arrive_release(claims + 1);
      }
    }
    if (!epi_all(tid != 0 || bounded_wait([&]() { return ld_acquire(claims + 1) >= n; }, abort_flag))) return false;
    for (int p = tid; p < n * k; p += kEpiThreads) s.pos[p] = __ldcg(a.sel_e + p), s.w[p] = __ldcg(a.sel_w + p);
    epi_sync();
  }
  for (int p = tid; p < n * k; p += kEpiThreads)
    if (s.pos[p] >= 0) atomicOr(&s.mask[s.pos[p]], 1ull << (p / k));
  epi_sync();
  const unsigned long long mask = s.mask[tid];  // thread e: expert e
  const int m = __popcll(mask);
  const int v = m ? 1 | (m << 10) | (((m + 3) / 4) << 20) : 0;  // at most 256, 512 and 512 in all
  int incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int b = __shfl_up_sync(kFull, incl, o);
    if (lane >= o) incl += b;
  }
  if (lane == 31) s.warp_total[warp] = incl;
  epi_sync();
  int before = incl - v;
  for (int w = 0; w < warp; ++w) before += s.warp_total[w];
  s.first_row[tid] = (before >> 10) & 1023;
  s.mask_of[tid] = mask;
  epi_sync();  // every mask has been read: the list takes their place
  if (v) {
    const int j = before & 1023;
    s.expert[j] = tid;
    s.start[j] = (before >> 10) & 1023;
    s.quads[j] = before >> 20;
    s.mask[j] = mask;
  }
  if (tid == kMaxExperts - 1) {
    const int active = (before + v) & 1023;
    s.active = active;
    s.items = (a.Is / 128 + active * (a.I / 128)) * a.s1 +
              a.H / 256 * (active * a.s2 + (a.Is ? a.s2s : 0) + ceil_div_dev(n, a.out_tokens));
  }
  for (int p = tid; p < n * k; p += kEpiThreads) {
    const int ex = s.pos[p], t = p / k;
    s.pos[p] = ex >= 0 ? s.first_row[ex] + __popcll(s.mask_of[ex] & ((1ull << t) - 1)) : -1;
  }
  epi_sync();
  return true;
}

// The last slice of a gate/up tile: the slices' sums, SwiGLU and the tile's 128
// channels of h into the expert's image, by a warp; lane l has channels 4l ..
// 4l + 3 and kAhead tokens on their way.
template <bool FP8>
__device__ __forceinline__ void write_h(const FewArgs& a, const FewSmem& s, const FewItem& T, int lane) {
  constexpr int kAhead = 4;
  const int W = 2 * (T.shared ? a.Is : a.I);
  const long long plane = static_cast<long long>(T.shared ? a.n : a.n * a.gate.top_k) * W;
  // packed rows: gate and up alternate in eights (bf16) or by 128
  const int grow = FP8 ? 4 * lane : 16 * (lane >> 1) + 4 * (lane & 1);
  constexpr int up = FP8 ? 128 : 8;
  const float* src = (T.shared ? a.p1s : a.p1) + static_cast<long long>(T.start) * W + T.tile * 256 + grow;
  uint8_t* img = h_image<FP8>(a, s, T);
  const int m = T.tokens;
  for (int c0 = 0; c0 < m; c0 += kAhead) {
    float4 g[kAhead], u[kAhead];
#pragma unroll
    for (int r = 0; r < kAhead; ++r) g[r] = u[r] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < a.s1; ++i) {
      float4 gi[kAhead], ui[kAhead];
#pragma unroll
      for (int r = 0; r < kAhead; ++r) {
        const float* at = src + i * plane + static_cast<long long>(min(c0 + r, m - 1)) * W;
        gi[r] = __ldcg(reinterpret_cast<const float4*>(at));
        ui[r] = __ldcg(reinterpret_cast<const float4*>(at + up));
      }
#pragma unroll
      for (int r = 0; r < kAhead; ++r) {
        g[r].x += gi[r].x, g[r].y += gi[r].y, g[r].z += gi[r].z, g[r].w += gi[r].w;
        u[r].x += ui[r].x, u[r].y += ui[r].y, u[r].z += ui[r].z, u[r].w += ui[r].w;
      }
    }
#pragma unroll
    for (int r = 0; r < kAhead; ++r) {
      const int c = c0 + r;
      if (c >= m) break;
      const float h[4] = {g[r].x / (1.0f + expf(-g[r].x)) * u[r].x, g[r].y / (1.0f + expf(-g[r].y)) * u[r].y,
                          g[r].z / (1.0f + expf(-g[r].z)) * u[r].z, g[r].w / (1.0f + expf(-g[r].w)) * u[r].w};
      if constexpr (FP8) {
        float am = fmaxf(fmaxf(fabsf(h[0]), fabsf(h[1])), fmaxf(fabsf(h[2]), fabsf(h[3])));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) am = fmaxf(am, __shfl_xor_sync(kFull, am, o));
        const GroupScale gs(am);
        uint8_t* step = img + static_cast<long long>(T.tile) * step_bytes<true>(m);
        *reinterpret_cast<uint32_t*>(step + swizzled(c, 4 * lane)) = e4m3x4(gs, h[0], h[1], h[2], h[3]);
        if (lane == 0) *reinterpret_cast<float*>(step + m * 128 + c * 4) = gs.s;
      } else {
        uint8_t* step = img + static_cast<long long>(2 * T.tile + (lane >> 4)) * step_bytes<false>(2 * m);
        // (the value stays below what bf16 rounds to infinity: the difference is then the rest of a finite h and,
        // with the sign of h, infinite for an infinite one; a NaN is in the difference)
        constexpr float kMost = 0x1.fep127f;  // the largest bf16
        auto within = [](float v) { return fminf(fmaxf(v, -kMost), kMost); };
        const uint32_t a0 = pack_bf16x2(within(h[0]), within(h[1])), a1 = pack_bf16x2(within(h[2]), within(h[3]));
        const uint32_t b0 = pack_bf16x2(h[0] - bf16_lo(a0), h[1] - bf16_hi(a0));
        const uint32_t b1 = pack_bf16x2(h[2] - bf16_lo(a1), h[3] - bf16_hi(a1));
        *reinterpret_cast<uint2*>(step + swizzled(c, 8 * (lane & 15))) = make_uint2(a0, a1);
        *reinterpret_cast<uint2*>(step + m * 128 + swizzled(c, 8 * (lane & 15))) = make_uint2(b0, b1);
      }
    }
  }
}

// 256 channels of an item's tokens.  A token's terms are its slots' partial sums,
// slot by slot, then the shared expert's; lane l adds channels 4l .. and 128 + 4l
// .. of terms first, first + step, ...
__device__ __forceinline__ void add_terms(const FewArgs& a, const FewSmem& s, int t, int tile, int first, int step,
                                          int lane, float4& lo, float4& hi) {
  constexpr int kAhead = 4;
  const int k = a.gate.top_k, H = a.H;
  const long long plane = static_cast<long long>(a.n) * k * H, plane_s = static_cast<long long>(a.n) * H;
  const int routed = k * a.s2, terms = routed + (a.Is ? a.s2s : 0);
  const int ch = tile * 256 + 4 * lane;
  lo = hi = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i0 = first; i0 < terms; i0 += step * kAhead) {
    float w[kAhead];
    float4 l[kAhead], h[kAhead];
#pragma unroll
    for (int r = 0; r < kAhead; ++r) {
      const int i = i0 + r * step;
      w[r] = 0.f;
      l[r] = h[r] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i >= terms) continue;
      const float* src;
      if (i < routed) {
        const int j = quick_div(i, a.r_s2), pos = s.pos[t * k + j];
        if (pos < 0) continue;
        w[r] = s.w[t * k + j];
        src = a.y + (i - j * a.s2) * plane + static_cast<long long>(pos) * H + ch;
      } else {
        w[r] = 1.0f;
        src = a.ys + (i - routed) * plane_s + static_cast<long long>(t) * H + ch;
      }
      l[r] = __ldcg(reinterpret_cast<const float4*>(src));
      h[r] = __ldcg(reinterpret_cast<const float4*>(src + 128));
    }
#pragma unroll
    for (int r = 0; r < kAhead; ++r) {
      lo.x = fmaf(w[r], l[r].x, lo.x), lo.y = fmaf(w[r], l[r].y, lo.y);
      lo.z = fmaf(w[r], l[r].z, lo.z), lo.w = fmaf(w[r], l[r].w, lo.w);
      hi.x = fmaf(w[r], h[r].x, hi.x), hi.y = fmaf(w[r], h[r].y, hi.y);
      hi.z = fmaf(w[r], h[r].z, hi.z), hi.w = fmaf(w[r], h[r].w, hi.w);
    }
  }
}
// An item of one token: its terms over the warps, whose sums are then added in
// order; of several: a token per warp.
__device__ __forceinline__ void write_out(const FewArgs& a, FewSmem& s, const FewItem& T, int warp, int lane, int tid) {
  float4 lo, hi;
  __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) + static_cast<long long>(T.token) * a.H + T.tile * 256;
  if (a.out_tokens > 1) {
    if (T.token + warp >= a.n) return;
    add_terms(a, s, T.token + warp, T.tile, 0, 1, lane, lo, hi);
    uint2* o = reinterpret_cast<uint2*>(out + static_cast<long long>(warp) * a.H);
    o[lane] = make_uint2(pack_bf16x2(lo.x, lo.y), pack_bf16x2(lo.z, lo.w));
    o[32 + lane] = make_uint2(pack_bf16x2(hi.x, hi.y), pack_bf16x2(hi.z, hi.w));
    return;
  }
  add_terms(a, s, T.token, T.tile, warp, kEpiWarps, lane, lo, hi);
  *reinterpret_cast<float4*>(&s.sum[warp][4 * lane]) = lo;
  *reinterpret_cast<float4*>(&s.sum[warp][128 + 4 * lane]) = hi;
  epi_sync();
  float acc = s.sum[0][tid];
#pragma unroll
  for (int w = 1; w < kEpiWarps; ++w) acc += s.sum[w][tid];
  out[tid] = __float2bfloat16_rn(acc);
}

// NT: columns (tokens) the FP8 epilogue keeps in registers; unused for BF16.
// (Bounded to 512 threads' registers where that suffices: the next call's logits kernel then fits beside it.)
template <bool FP8, int NT>
__global__ void __launch_bounds__(FP8 && NT == 64 ? kThreads : 512, 1) few_ffn_kernel(const __grid_constant__ FewArgs a) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t base = smem_u32(smem_raw);
  if (base & 1023u) {  // uniform for the CTA: nothing is initialised yet
    pdl_wait();
    if (threadIdx.x == 0) record_status(a.status, ST_SMEM_ALIGN);
    return;
  }
  const int SW = a.stages_w, SX = a.stages_x;
  const uint32_t sW = base, sX = base + SW * kWBytes;
  FewSmem& s = *reinterpret_cast<FewSmem*>(smem_raw + SW * kWBytes + SX * a.x_slot);
  auto bar = [&](int i) { return smem_u32(&s.bar[i]); };
  constexpr int B_FW = 0, B_EW = kFewMaxStages, B_FX = 2 * kFewMaxStages, B_EX = 3 * kFewMaxStages,
                B_PF = 4 * kFewMaxStages, B_PE = B_PF + kMaxPartials, B_QF = B_PE + kMaxPartials, B_QE = B_QF + kQ,
                B_QD = B_QE + kQ, B_DR = B_QD + kQ, B_META = B_DR + 1;
  constexpr int kPartials = FP8 ? (NT == 16 ? 8 : 4) : kAccs;
  constexpr int kHalf = FP8 ? NT : 128;  // columns of a row half
  static_assert(2 * kHalf * kPartials <= kTmemCols, "tensor memory budget");
  volatile int* abort_flag = &s.abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (warp == 0) {
    if (lane == 0) {
      for (int i = 0; i < kFewMaxStages; ++i) {
        mbar_init(bar(B_FW + i), 1);
        mbar_init(bar(B_EW + i), 1);
        mbar_init(bar(B_FX + i), 1);
        mbar_init(bar(B_EX + i), FP8 ? 1 + kEpiWarps : 1);  // FP8: the epilogue reads its scales
      }
      for (int i = 0; i < kMaxPartials; ++i) {
        mbar_init(bar(B_PF + i), 1);
        mbar_init(bar(B_PE + i), kEpiWarps);
      }
      for (int i = 0; i < kQ; ++i) {
        mbar_init(bar(B_QF + i), 1);
        mbar_init(bar(B_QE + i), kQReaders);
        mbar_init(bar(B_QD + i), kEpiWarps);
      }
      mbar_init(bar(B_DR), 1);
      mbar_init(bar(B_META), kEpiThreads);
      s.abort = 0;
      fence_barrier_init();
    }
  } else if (warp == 1) {
    tmem_alloc(smem_u32(&s.tmem), kTmemCols);
    tmem_relinquish();
  }
  // the weight maps are acquired while the logits are computed (a layer id that is still being written would
  // only acquire another layer's)
  const int early = load_layer(a.lref.layer, a.lref.n_layers, a.status, false);
  auto acquire_maps = [&](int l) {
    for (int m = MAP_GATE_UP; m <= (a.Is ? MAP_SH_DOWN : MAP_DOWN); ++m) tensormap_acquire(&a.lref.table[l].map[m]);
  };
  auto load_bias = [&](int l) {
    const float* bias = a.lref.table[l].router_bias;
    if (bias && threadIdx.x < a.gate.n_experts) s.bias[threadIdx.x] = __ldg(bias + threadIdx.x);
    else if (threadIdx.x < kMaxExperts) s.bias[threadIdx.x] = 0.f;
  };
  if ((warp == 0 || warp == 2) && lane == 0) acquire_maps(early);
  load_bias(early);
  // The shared expert's weights are needed whatever the router says: fetched into L2 meanwhile.  (By the time
  // this kernel comes up the logits kernel has asked for the router's, which would have to wait behind these:
  // with these first its logits took 13 us instead of 5.)
  if (warp == 2 && lane == 0 && a.Is) {
    constexpr int kx = FP8 ? 128 : 64;
    const CUtensorMap* m = a.lref.table[early].map;
    const int gu = a.Is / 128 * (a.H / kx), all = gu + a.H / 256 * (a.Is / kx);
    for (int b = blockIdx.x; b < min(all, kPrefetchBoxes); b += gridDim.x)
      prefetch_box(m + (b < gu ? MAP_SH_GATE_UP : MAP_SH_DOWN), (b < gu ? b : b - gu) * 256);
  }
  pdl_wait();
  int claim = 0;
  if (threadIdx.x == 0) claim = atomicAdd(&a.counters[0], 1);
  const int layer = a.fixed_layer ? early : load_layer(a.lref.layer, a.lref.n_layers, a.status, false);
  if (layer != early) load_bias(layer);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = s.tmem;
  const LayerEntry& le = a.lref.table[layer];
  auto give_up = [&]() {
    *abort_flag = 1;
    record_status(a.status, ST_WAIT_TIMEOUT);
  };
  // the next item of a reader of the queue (-1: none left); false: gave up
  auto pop = [&](Ring<kQ>& r, int& item) {
    if (!__all_sync(kFull, mbar_wait(bar(B_QF + r.s), r.phase, abort_flag))) return false;
    item = *reinterpret_cast<volatile int*>(&s.q[r.s]);
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(B_QE + r.s));
    r.advance();
    return true;
  };

  bool routed = false;  // the routing has been waited for
  auto wait_routing = [&](int item) {
    if (!routed && item >= a.first_routed) routed = mbar_wait(bar(B_META), 0, abort_flag);
    return routed || item < a.first_routed;
  };

  if (warp == 0) {
    // -------------------------------------------------------- claims and weights
    if (lane == 0) {
      bool ok = true;
      int st = 0, issued = 0;
      uint32_t ph = 0;
      Ring<kQ> rq;
      const uint64_t pol = l2_policy(1);
      if (layer != early) acquire_maps(layer);
      int next = claim;
      while (ok) {
        ok = wait_routing(next);
        if (!ok) break;
        const int item = next < a.first_routed || next < s.items ? next : -1;
        ok = mbar_wait(bar(B_QE + rq.s), rq.phase ^ 1u, abort_flag);
        if (!ok) break;
        s.q[rq.s] = item;
        mbar_arrive(bar(B_QF + rq.s));
        rq.advance();
        if (item < 0) break;
        next = atomicAdd(&a.counters[0], 1);
        const FewItem T = decode<FP8>(a, s, item);
        if (T.combine) continue;
        const CUtensorMap* m = &le.map[T.down ? (T.shared ? MAP_SH_DOWN : MAP_DOWN)
                                              : (T.shared ? MAP_SH_GATE_UP : MAP_GATE_UP)];
        const int tiles = T.down ? a.H / 256 : a.I / 128;
        const int kit = (T.down ? (T.shared ? a.Is : a.I) : a.H) / (FP8 ? 128 : 64);
        const int box0 = ((T.shared ? 0 : s.expert[T.j] * tiles) + T.tile) * kit;
        for (int kb = T.kb0; kb < T.kb1; ++kb) {
          ok = mbar_wait(bar(B_EW + st), ph ^ 1u, abort_flag);
          if (!ok) break;
          mbar_arrive_expect_tx(bar(B_FW + st), kWBytes);
          tma_load_2d(sW + st * kWBytes, m, bar(B_FW + st), 0, (box0 + kb) * 256, pol);
          issued = min(issued + 1, SW);
          if (++st == SW) st = 0, ph ^= 1u;
        }
      }
      pdl_launch();  // no items left for this CTA
      if (!ok) {
        give_up();
        // the copies in flight land before the CTA's memory goes away
        int dummy = 0;
        for (int i = issued; i > 0; --i) {
          const int b = st - i;
          mbar_wait(bar(B_FW + (b < 0 ? b + SW : b)), b < 0 ? ph ^ 1u : ph, &dummy);
        }
      }
    }
  } else if (warp == 2) {
    // -------------------------------------------------------- operand rows
    Ring<kQ> rq;
    bool ok = true;
    int st = 0, issued = 0, item;
    uint32_t ph = 0;
    if (lane == 0) fence_proxy_async_all();
    while (ok) {
      ok = pop(rq, item);
      ok = ok && (item < 0 || __all_sync(kFull, wait_routing(item)));
      if (!ok || item < 0) break;
      if (lane == 0) {
        const FewItem T = decode<FP8>(a, s, item);
        // (BF16 h: the second rows go to the next multiple of 8, where their columns begin)
        const bool two = T.down && !FP8;
        const uint32_t bytes = step_bytes<FP8>(T.rows), step = two ? 2 * bytes : bytes;
        const uint32_t second = round_up_dev(T.rows, 8) * 128;
        const uint8_t* img = T.down ? h_image<FP8>(a, s, T) : a.ximg;
        if (T.down && !T.combine) {
          const int* ready = a.counters + a.h_ready + (T.shared ? 0 : 1 + T.j);
          const int want = (T.shared ? a.Is : a.I) / 128;
          ok = bounded_wait([&]() { return ld_acquire(ready) >= want; }, abort_flag);
          fence_proxy_async_all();
        }
        for (int kb = T.kb0; ok && kb < T.kb1; ++kb) {
          ok = mbar_wait(bar(B_EX + st), ph ^ 1u, abort_flag);
          if (!ok) break;
          mbar_arrive_expect_tx(bar(B_FX + st), step);
          const uint8_t* from = img + static_cast<long long>(kb) * step;
          bulk_load(sX + st * a.x_slot, from, bytes, bar(B_FX + st));
          if (two) bulk_load(sX + st * a.x_slot + second, from + bytes, bytes, bar(B_FX + st));
          issued = min(issued + 1, SX);
          if (++st == SX) st = 0, ph ^= 1u;
        }
      }
      ok = __all_sync(kFull, ok);
    }
    if (!ok && lane == 0) {
      give_up();
      int dummy = 0;
      for (int i = issued; i > 0; --i) {
        const int b = st - i;
        mbar_wait(bar(B_FX + (b < 0 ? b + SX : b)), b < 0 ? ph ^ 1u : ph, &dummy);
      }
    }
  } else if (warp == 1) {
    // -------------------------------------------------------- MMA
    const bool issuer = elect_one();
    Ring<kQ> rq;
    Ring<kPartials> p;
    int sw = 0, sx = 0, item;
    uint32_t pw = 0, px = 0;
    bool ok = true, issued = false;
    const uint64_t wdesc = smem_desc_sw128(sW), xdesc = smem_desc_sw128(sX);
    while (ok) {
      ok = pop(rq, item);
      ok = ok && (item < 0 || __all_sync(kFull, wait_routing(item)));
      if (!ok || item < 0) break;
      const FewItem T = decode<FP8>(a, s, item);
      const uint32_t id = FP8 ? (1u << 4) | (static_cast<uint32_t>(T.n >> 3) << 17) | (8u << 24) : idesc_bf16_f32(128, T.n);
      for (int kb = T.kb0; kb < T.kb1; ++kb) {
        ok = mbar_wait(bar(B_FX + sx), px, abort_flag) && mbar_wait(bar(B_FW + sw), pw, abort_flag);
        if (FP8 || kb == T.kb0) ok = ok && mbar_wait(bar(B_PE + p.s), p.phase ^ 1u, abort_flag);
        ok = __all_sync(kFull, ok);
        if (!ok) break;
        tc_fence_after();
        if (issuer) {
          const uint64_t wd = wdesc + static_cast<uint32_t>(sw * (kWBytes >> 4));
          const uint64_t xd = xdesc + static_cast<uint32_t>(sx * (a.x_slot >> 4));
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const uint32_t d = tmem_base + (2 * p.s + half) * kHalf;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
              const uint64_t w = wd + half * (16384 >> 4) + 2 * kk, x = xd + 2 * kk;
              if constexpr (FP8) mma_e4m3(d, w, x, id, kk > 0 ? 1u : 0u);
              else tc_mma_bf16(d, w, x, id, kb > T.kb0 || kk > 0 ? 1u : 0u);
            }
          }
          if (FP8 || kb == T.kb1 - 1) tc_commit(bar(B_PF + p.s));
          tc_commit(bar(B_EW + sw));
          tc_commit(bar(B_EX + sx));
        }
        __syncwarp();
        issued = true;
        if (FP8 || kb == T.kb1 - 1) p.advance();
        if (++sw == SW) sw = 0, pw ^= 1u;
        if (++sx == SX) sx = 0, px ^= 1u;
      }
    }
    if (!ok) {
      if (lane == 0) give_up();
      if (issued) {
        int dummy = 0;
        if (elect_one()) tc_commit(bar(B_DR));
        __syncwarp();
        mbar_wait(bar(B_DR), 0, &dummy);
      }
    }
  } else if (warp == 3) {
    // -------------------------------------------------------- finisher
    // An item whose partial sums are stored is counted; the arrival that completes a gate/up tile makes its h.
    // (A warp of its own: under the weight stream a release and the counter's answer take microseconds.)
    Ring<kQ> rq;
    bool ok = true;
    while (ok) {
      ok = __all_sync(kFull, mbar_wait(bar(B_QF + rq.s), rq.phase, abort_flag));
      if (!ok) break;
      const int item = *reinterpret_cast<volatile int*>(&s.q[rq.s]);
      if (item < 0) break;
      ok = __all_sync(kFull, wait_routing(item));
      if (!ok) break;
      const FewItem T = decode<FP8>(a, s, item);
      // (an output's place is left as it is: the epilogue does not arrive there, so its phase is made up for)
      if (T.combine) {
        if (lane < kEpiWarps) mbar_arrive(bar(B_QD + rq.s));
      } else {
        ok = __all_sync(kFull, mbar_wait(bar(B_QD + rq.s), rq.phase, abort_flag));
        if (!ok) break;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_QE + rq.s));
      rq.advance();
      if (T.combine) continue;
      if (T.down) {
        if (lane == 0) arrive_release(a.counters + T.ticket);
        continue;
      }
      int last = 0;
      if (lane == 0) last = arrive_acq_rel(a.counters + T.ticket) == T.arrivals - 1;
      if (!__shfl_sync(kFull, last, 0)) continue;
      __syncwarp();  // what lane 0 has acquired is every lane's to read
      write_h<FP8>(a, s, T, lane);
      fence_proxy_async_all();
      __syncwarp();
      if (lane == 0) arrive_release(a.counters + a.h_ready + (T.shared ? 0 : 1 + T.j));
    }
    if (!ok && lane == 0) give_up();
  } else {
    // -------------------------------------------------------- epilogue
    // warp w: TMEM lanes 32 (w % 4) .. of row half (w - 4) / 4
    const int q = warp & 3, half = (warp - 4) >> 2;
    const int tid = threadIdx.x - 128;
    const uint32_t lanes = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + half * kHalf;
    const int row = half * 128 + q * 32 + lane;  // of the weight tile
    bool ok = list_experts(a, s, warp - 4, lane, tid, abort_flag);
    if (ok) mbar_arrive(bar(B_META));
    Ring<kQ> rq;
    Ring<kPartials> p;
    int sx = 0, item = -1;
    uint32_t px = 0;
    FewItem T{};
    // FP8: the scales of this warp's 128 weight rows, k-step kb0 + l in lane l (32 steps at a time), on their
    // way before the item in front is finished
    const float* bs_lo = nullptr;
    float scales = 0.f;
    auto load_scales = [&](int kb) {
      if (kb + lane < T.kb1) scales = __ldg(bs_lo + kb + lane);
    };
    int at = 0;  // the item's place in the queue
    auto next_item = [&]() {
      at = rq.s;
      if (!pop(rq, item)) return false;
      if (item < 0) return true;
      T = decode<FP8>(a, s, item);
      if (FP8 && !T.combine) {
        const int scale_rows = T.down ? a.H / 128 : 2 * a.I / 128;
        const int kit = (T.down ? (T.shared ? a.Is : a.I) : a.H) / 128;
        bs_lo = le.scale[T.down ? (T.shared ? MAP_SH_DOWN : MAP_DOWN) : (T.shared ? MAP_SH_GATE_UP : MAP_GATE_UP)] +
                (static_cast<long long>(T.shared ? 0 : s.expert[T.j]) * scale_rows + 2 * T.tile + half) * kit;
        load_scales(T.kb0);
      }
      return true;
    };
    ok = ok && next_item();
    while (true) {
      const bool work = ok && item >= 0;
      // the item's sums of this thread's row go to plane ``slice`` of the workspace, row start + c for the
      // expert's c-th token
      const long long rows_all = T.shared ? a.n : a.n * a.gate.top_k;
      const long long ld = T.down ? a.H : 2 * (T.shared ? a.Is : a.I);
      float* dst = (T.down ? (T.shared ? a.ys : a.y) : (T.shared ? a.p1s : a.p1)) +
                   (T.slice * rows_all + T.start) * ld + T.tile * 256 + row;
      if (work && T.combine) {
        const int* done = a.counters + T.ticket;
        ok = tid != 0 || bounded_wait([&]() { return ld_acquire(done) == T.arrivals; }, abort_flag);
      } else if (FP8 && work) {
        float acc[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) acc[i] = 0.f;
        // (gate/up computes every token's column; 16 columns without a token of this expert are left out)
        uint32_t live = 0;
#pragma unroll
        for (int ch = 0; ch < NT / 16; ++ch)
          live |= (T.down ? 16 * ch < T.tokens : ((T.mask >> (16 * ch)) & 0xffffull) != 0) ? 1u << ch : 0u;
        for (int kb = T.kb0; kb < T.kb1; ++kb) {
          const int l = (kb - T.kb0) & 31;
          if (l == 0 && kb > T.kb0) load_scales(kb);
          const float ws = __shfl_sync(kFull, scales, l);
          ok = __all_sync(kFull, mbar_wait(bar(B_FX + sx), px, abort_flag) &&
                                     mbar_wait(bar(B_PF + p.s), p.phase, abort_flag));
          if (!ok) break;
          tc_fence_after();
          const float4* sc = reinterpret_cast<const float4*>(smem_raw + SW * kWBytes + sx * a.x_slot + T.rows * 128);
#pragma unroll
          for (int ch = 0; ch < NT / 16; ++ch) {
            if ((live >> ch) & 1u) {
              uint32_t v[16];
              tmem_ld16(lanes + p.s * 2 * kHalf + 16 * ch, v);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float4 f = sc[4 * ch + i];
                acc[16 * ch + 4 * i] = fmaf(ws * f.x, __uint_as_float(v[4 * i]), acc[16 * ch + 4 * i]);
                acc[16 * ch + 4 * i + 1] = fmaf(ws * f.y, __uint_as_float(v[4 * i + 1]), acc[16 * ch + 4 * i + 1]);
                acc[16 * ch + 4 * i + 2] = fmaf(ws * f.z, __uint_as_float(v[4 * i + 2]), acc[16 * ch + 4 * i + 2]);
                acc[16 * ch + 4 * i + 3] = fmaf(ws * f.w, __uint_as_float(v[4 * i + 3]), acc[16 * ch + 4 * i + 3]);
              }
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(bar(B_EX + sx));
            mbar_arrive(bar(B_PE + p.s));
          }
          p.advance();
          if (++sx == SX) sx = 0, px ^= 1u;
        }
        if (ok) {
          int c = 0;
#pragma unroll
          for (int i = 0; i < NT; ++i)
            if (T.down ? i < T.tokens : (T.mask >> i) & 1ull) dst[ld * c++] = acc[i];
        }
      } else if (work) {
        ok = __all_sync(kFull, mbar_wait(bar(B_PF + p.s), p.phase, abort_flag));
        if (ok) {
          tc_fence_after();
          const uint32_t t0 = lanes + p.s * 2 * kHalf;
          const int cols = round_up_dev(T.rows, 8);  // down: the columns of the roundings follow
          int c = 0;
          for (int c0 = 0; c0 < cols; c0 += 8) {
            const uint32_t some = T.down ? (c0 + 8 <= T.tokens ? 0xffu : (1u << (T.tokens - c0)) - 1u)
                                         : static_cast<uint32_t>(T.mask >> c0) & 0xffu;
            if (!some) continue;
            uint32_t v[8], r[8];
            tmem_ld8(t0 + c0, v);
            if (T.down) tmem_ld8(t0 + cols + c0, r);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if ((some >> i) & 1u)
                dst[ld * c++] = T.down ? __uint_as_float(v[i]) + __uint_as_float(r[i]) : __uint_as_float(v[i]);
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(B_PE + p.s));
          p.advance();
        }
      }
      if (work && ok && !T.combine) {  // the finisher takes it from here
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B_QD + at));
        ok = next_item();
        continue;
      }
      // An output, the end or a failure.  The outputs' barriers are shared: all warps go on or none does, and
      // each passes this one before it leaves.
      if (!epi_all(ok)) {
        ok = false;
        break;
      }
      if (item < 0) break;
      write_out(a, s, T, warp - 4, lane, tid);
      ok = next_item();
    }
    if (!ok && lane == 0) give_up();
  }

  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, kTmemCols);
  }
}

template <bool FP8, int NT>
cudaError_t launch_ffn(const FewArgs& a, int grid, cudaStream_t st) {
  return launch_pdl(few_ffn_kernel<FP8, NT>, dim3(grid), dim3(kThreads), a.smem, st, 1, a);
}

}  // namespace

cudaError_t few_set_attributes() {
  cudaError_t e = cudaSuccess;
  auto set = [&](auto* f, size_t bytes) {
    if (e == cudaSuccess)
      e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
  };
  // the logits kernels leave their SM in the configuration that the FFN's shared memory needs, which can then
  // come up beside them
  auto carve = [&](auto* f) {
    if (e == cudaSuccess)
      e = cudaFuncSetAttribute(f, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
  };
  carve(few_logits_kernel<false, 1>);
  carve(few_logits_kernel<true, 1>);
  carve(few_logits_kernel<false, kFewTokens / 8>);
  carve(few_logits_kernel<true, kFewTokens / 8>);
  set(few_ffn_kernel<false, 16>, kFewSmem);
  set(few_ffn_kernel<true, 16>, kFewSmem);
  set(few_ffn_kernel<true, 64>, kFewSmem);
  return e;
}

cudaError_t few_launch(const FewArgs& a, bool fp8, int grid, cudaStream_t st) {
  // (at least a CTA for every two tokens, whose rows the image takes, up to a third of the GPU)
  const int ctas = std::max(ceil_div(a.gate.n_experts, 16) * kLogitSlices, std::min(48, a.n / 2));
  const dim3 grid_l(ctas), block_l(kLogitThreads);
  cudaError_t e;
  if (a.n <= 8)
    e = fp8 ? launch_pdl(few_logits_kernel<true, 1>, grid_l, block_l, 0, st, 1, a)
            : launch_pdl(few_logits_kernel<false, 1>, grid_l, block_l, 0, st, 1, a);
  else
    e = fp8 ? launch_pdl(few_logits_kernel<true, kFewTokens / 8>, grid_l, block_l, 0, st, 1, a)
            : launch_pdl(few_logits_kernel<false, kFewTokens / 8>, grid_l, block_l, 0, st, 1, a);
  if (e != cudaSuccess) return e;
  if (!fp8) return launch_ffn<false, 16>(a, grid, st);
  return a.n <= 16 ? launch_ffn<true, 16>(a, grid, st) : launch_ffn<true, 64>(a, grid, st);
}

}  // namespace asap

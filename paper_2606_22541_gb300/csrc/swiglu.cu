// SwiGLU between the two products of an expert (or dense) layer in training:
// what the backward pass needs is kept in e4m3 with a scale per row and 128
// columns, the format of the FP8 layers.
//   forward:  h = g s(g) u, s(g) = 1 / (1 + e^-g); gate and up quantised as asap_moe_fp8_quantize does
//   backward: with G, U the kept values, S = s(G):
//             d_gate = d_h U (S + G S (1 - S)),  d_up = d_h G S,  h = G S U
#include "common.cuh"
#include "e4m3.cuh"
#include "elem.cuh"
#include "rows.h"

#include <algorithm>

namespace asap {

namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr int kThreads = 256;
// Both kernels stream: 8 bytes a column forward (bf16), 10 backward, which the copy
// rate would move in 79.6 and 99.4 us for 32768 x 2048; they take 84 and 101.
// The forward pass has the arithmetic to hide as well (two scales, two quotients, a
// sigmoid), so a lane has 16 columns, over which the maximum's exchange and the scales
// are spread, and four CTAs an SM (3: 93 us); with 8 columns a lane it took 103 to 113,
// and 95 with lanes of 16 neighbouring columns, whose accesses are half as wide as they
// look.  Backward there is little, so a lane has one 16-byte chunk and its next group's
// loads on their way (118 us with 16 columns and no loads ahead; 106 with the e4m3 values
// decoded before the next loads are out, which takes the registers).
// Grids of a few waves' CTAs, so that the SMs' ends are level: forward 4 to 50 CTAs for
// each SM make no difference, backward 10, 20, 40 and all: 112, 104, 100, 110 us (32768 x 2048;
// other sizes were not tried).
// Narrow rows are further from the copy rate: 31962 x 288 forward 20.5 us (10.9), backward 21.3 (13.7), 38502 x 256
// backward 19.1 (14.6).  Forward a team has one group or two there and loads none ahead.
// Odd widths, one column an access: 11259 x 5961 forward 128 us (79.7), 8558 x 4785
// backward 92 (60.7); with the accesses of neighbouring lanes 8 columns apart 291 and 102.
constexpr int kSaveCtas = 4, kSaveGrid = 16;  // CTAs an SM, CTAs of the grid for each SM
constexpr int kGradCtas = 5, kGradGrid = 40;
// Lanes of a group, by the columns of an access.
__host__ __device__ constexpr int save_team(int v) { return v >= 4 ? 8 : 16; }
__host__ __device__ constexpr int grad_team(int v) { return v == 8 ? 16 : 32; }

// 1 / (1 + e^-g) of two columns.  fp32 results take expf and a division (0 where e^-g passes fp32, below -88.7); 16-bit
// ones the fast exponential and reciprocal.  These are off by 2^-22 and 2^-23 (relative, by their documentation) and the
// exponent's own rounding adds |g| 2^-23: (5 + 1.2 |g|) 2^-23 in all, 110 of these units at most, since the result is 0
// where e^-g passes 2^126 (below -87.3).  A result's own rounding is 2^-8 in bf16 and 2^-11 in fp16, 32768 and 4096 units:
// the sigmoid's error stays below 0.4 % of bf16's and 3 % of fp16's.
template <typename T>
__device__ __forceinline__ uint64_t sigmoid2(uint64_t g) {
  if constexpr (sizeof(T) == 4) {
    const float2 v = unpair(g);
    return pair(1.0f / (1.0f + expf(-v.x)), 1.0f / (1.0f + expf(-v.y)));
  } else {
    constexpr float kLog2E = 1.4426950408889634f;
    float2 e = unpair(mul2(g, pair(-kLog2E, -kLog2E)));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.x));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.y));
    e.x += 1.0f;
    e.y += 1.0f;
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(e.x));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(e.y));
    return pair(e.x, e.y);
  }
}

// A lane's kCols columns of a group, as kChunks chunks of V columns, one access each (of V bytes in e4m3): chunk i of
// lane l starts at column i kTeam V + l V, so that a team's accesses are contiguous.  V: 16 bytes, or as many columns as
// the alignment of every row allows.
template <typename T, int V, int kTeam>
struct Lane {
  static constexpr int kCols = 128 / kTeam, kChunks = kCols / V;
  Cols<T, V> c[kChunks];
  __device__ static __forceinline__ int column(int lane, int i) { return (i * kTeam + lane) * V; }
  // p: the group's first column, left: columns from there
  __device__ __forceinline__ void load(const T* p, int left, int lane) {
#pragma unroll
    for (int i = 0; i < kChunks; ++i) c[i].load(p + column(lane, i), left - column(lane, i));
  }
  __device__ __forceinline__ void to(float (&f)[kCols]) const {
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      float v[V];
      c[i].to(v);
#pragma unroll
      for (int k = 0; k < V; ++k) f[i * V + k] = v[k];
    }
  }
  __device__ static __forceinline__ void store(T* p, int left, int lane, const float (&f)[kCols]) {
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      float v[V];
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = f[i * V + k];
      Cols<T, V> o;
      o.from(v);
      const int at = column(lane, i);
      if (left > at) o.store(p + at, left - at);
    }
  }
  // The same columns in e4m3.
  __device__ static __forceinline__ void store_q(uint8_t* p, int left, int lane, const uint32_t (&w)[kCols / 4]) {
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      const int at = column(lane, i);
      if (left - at >= V) {
        if constexpr (V == 8)
          *reinterpret_cast<uint2*>(p + at) = make_uint2(w[2 * i], w[2 * i + 1]);
        else if constexpr (V == 4)
          *reinterpret_cast<uint32_t*>(p + at) = w[i];
        else if constexpr (V == 2)
          *reinterpret_cast<uint16_t*>(p + at) = static_cast<uint16_t>(w[i / 2] >> (16 * (i & 1)));
        else
          p[at] = static_cast<uint8_t>(w[i / 4] >> (8 * (i & 3)));
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (at + j < left) p[at + j] = static_cast<uint8_t>(w[(i * V + j) >> 2] >> (8 * ((i * V + j) & 3)));
      }
    }
  }
  __device__ static __forceinline__ void load_q(const uint8_t* p, int left, int lane, uint32_t (&w)[kCols / 4]) {
#pragma unroll
    for (int i = 0; i < kCols / 4; ++i) w[i] = 0;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      const int at = column(lane, i);
      if (V > 1 && left - at >= V) {
        if constexpr (V == 8) {
          asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(w[2 * i]), "=r"(w[2 * i + 1]) : "l"(p + at));
        } else if constexpr (V == 4) {
          asm volatile("ld.global.b32 %0, [%1];" : "=r"(w[i]) : "l"(p + at));
        } else if constexpr (V == 2) {
          uint16_t v;
          asm volatile("ld.global.b16 %0, [%1];" : "=h"(v) : "l"(p + at));
          w[i / 2] |= static_cast<uint32_t>(v) << (16 * (i & 1));
        }
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (at + j < left)
            w[(i * V + j) >> 2] |= static_cast<uint32_t>(*const_cast<const volatile uint8_t*>(p + at + j))
                                   << (8 * ((i * V + j) & 3));
      }
    }
  }
};
template <int N>
__device__ __forceinline__ void decode(const uint32_t (&q)[N / 4], float s, float (&f)[N]) {
#pragma unroll
  for (int j = 0; j < N / 2; ++j) {
    const __half2 h = __half2(
        __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(q[j >> 1] >> (16 * (j & 1))), __NV_E4M3));
    const float2 v = __half22float2(h);
    f[2 * j] = s * v.x;
    f[2 * j + 1] = s * v.y;
  }
}

// Rows and groups of a team: the groups first, first + teams, ... of rows x groups.
struct Walk {
  int row, grp, dr, dg, groups;
  __device__ __forceinline__ Walk(int cols, int team) {
    const int per = kThreads / team;
    groups = (cols + 127) / 128;
    const int teams = gridDim.x * per;
    const int first = blockIdx.x * per + threadIdx.x / team;
    dr = teams / groups, dg = teams % groups;
    row = first / groups, grp = first % groups;
  }
  __device__ __forceinline__ void next() {
    row += dr;
    grp += dg;
    if (grp >= groups) grp -= groups, ++row;
  }
};
__device__ __forceinline__ int filled(const SwigluArgs& a) {
  return a.n_rows ? min(max(ld_dep(a.n_rows), 0), a.rows) : a.rows;
}
// Largest magnitudes of a group of gate's and of up's columns (a NaN loses).
// 16-bit values: gate's in the lower half of a register, up's in the upper, so that one exchange serves both.
template <typename T, int V, int kTeam>
__device__ __forceinline__ float2 amax(const Lane<T, V, kTeam>& gate, const Lane<T, V, kTeam>& up) {
  using L = Lane<T, V, kTeam>;
  if constexpr (sizeof(T) == 4) {
    float g[L::kCols], u[L::kCols];
    gate.to(g);
    up.to(u);
    float2 m = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < L::kCols; ++i) m.x = fmaxf(m.x, fabsf(g[i])), m.y = fmaxf(m.y, fabsf(u[i]));
#pragma unroll
    for (int o = kTeam / 2; o > 0; o >>= 1) {
      m.x = fmaxf(m.x, __shfl_xor_sync(kFull, m.x, o));
      m.y = fmaxf(m.y, __shfl_xor_sync(kFull, m.y, o));
    }
    return m;
  } else {
    using T2 = std::conditional_t<std::is_same_v<T, __half>, __half2, __nv_bfloat162>;
    auto larger = [](uint32_t a, uint32_t b) {
      const T2 m = __hmax2(*reinterpret_cast<const T2*>(&a), *reinterpret_cast<const T2*>(&b));
      return *reinterpret_cast<const uint32_t*>(&m);
    };
    constexpr uint32_t kAbs = 0x7FFF7FFFu;
    uint32_t mg = 0, mu = 0;
#pragma unroll
    for (int i = 0; i < L::kChunks; ++i)
#pragma unroll
      for (int k = 0; k < Cols<T, V>::kWords; ++k)
        mg = larger(mg, gate.c[i].w[k] & kAbs), mu = larger(mu, up.c[i].w[k] & kAbs);
    uint32_t m = larger(__byte_perm(mg, mu, 0x5410), __byte_perm(mg, mu, 0x7632));
#pragma unroll
    for (int o = kTeam / 2; o > 0; o >>= 1) m = larger(m, __shfl_xor_sync(kFull, m, o));
    return unpack2<T>(m);  // (zeros and NaNs alone: 0)
  }
}

template <typename T, int V>
__global__ void __launch_bounds__(kThreads, kSaveCtas)
    swiglu_save_kernel(const T* gate, const T* up, long long ld, T* __restrict__ h, long long ldh, const SwigluArgs a) {
  constexpr int kTeam = save_team(V);
  using L = Lane<T, V, kTeam>;
  pdl_wait();
  pdl_launch();
  const int lane = threadIdx.x & (kTeam - 1), rows = filled(a);
  // (a warp's teams leave together: their shuffles name the whole warp)
  for (Walk at(a.cols, kTeam); __any_sync(kFull, at.row < rows); at.next()) {
    const int c = at.grp * 128, left = at.row < rows ? a.cols - c : 0;
    L gl, ul;
    gl.load(gate + at.row * ld + c, left, lane);
    ul.load(up + at.row * ld + c, left, lane);
    const float2 m = amax<T, V, kTeam>(gl, ul);
    const GroupScale gs(m.x), us(m.y);
    if (left <= 0) continue;
    float g[L::kCols], u[L::kCols];
    gl.to(g);
    ul.to(u);
    uint32_t q[L::kCols / 4];
    const long long to = at.row * a.ldq + c;
    e4m3_pairs(gs, g, q);
    L::store_q(a.gate_q + to, left, lane, q);
    e4m3_pairs(us, u, q);
    L::store_q(a.up_q + to, left, lane, q);
    if (lane == 0) {
      a.gate_s[at.row * a.lds + at.grp] = gs.s;
      a.up_s[at.row * a.lds + at.grp] = us.s;
    }
#pragma unroll
    for (int i = 0; i < L::kCols; i += 2) {
      const uint64_t g2 = pair(g[i], g[i + 1]);
      const float2 v = unpair(mul2(mul2(g2, sigmoid2<T>(g2)), pair(u[i], u[i + 1])));
      g[i] = v.x;
      g[i + 1] = v.y;
    }
    L::store(h + at.row * ldh + c, left, lane, g);
  }
}

template <typename T, int V>
__global__ void __launch_bounds__(kThreads, kGradCtas)
    swiglu_backward_kernel(const T* d_h, long long ldd, T* __restrict__ d_gate, T* __restrict__ d_up, long long ldg,
                           T* __restrict__ h, long long ldh, const SwigluArgs a) {
  constexpr int kTeam = grad_team(V);
  using L = Lane<T, V, kTeam>;
  constexpr int N = L::kCols;
  pdl_wait();
  pdl_launch();
  const int lane = threadIdx.x & (kTeam - 1), rows = filled(a);
  L dn;  // the next group's
  uint32_t gn[N / 4], un[N / 4];
  float gsn, usn;
  Walk at(a.cols, kTeam);
  auto fetch = [&]() {
    const int c = at.grp * 128;
    const int left = at.row < rows ? a.cols - c : 0;
    if (left <= L::column(lane, 0)) return;
    dn.load(d_h + at.row * ldd + c, left, lane);
    const long long from = at.row * a.ldq + c, scale = at.row * a.lds + at.grp;
    L::load_q(a.gate_q + from, left, lane, gn);
    L::load_q(a.up_q + from, left, lane, un);
    gsn = ld_dep(a.gate_s + scale);
    usn = ld_dep(a.up_s + scale);
  };
  fetch();
  while (at.row < rows) {
    const L dc = dn;
    uint32_t gq[N / 4], uq[N / 4];
#pragma unroll
    for (int i = 0; i < N / 4; ++i) gq[i] = gn[i], uq[i] = un[i];
    const float gs = gsn, us = usn;
    const int row = at.row, c = at.grp * 128, left = a.cols - c;
    at.next();
    fetch();
    if (left <= L::column(lane, 0)) continue;
    float d[N], g[N], u[N], dg[N], du[N];
    dc.to(d);
    decode(gq, gs, g);
    decode(uq, us, u);
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const float2 s2 = unpair(sigmoid2<T>(pair(g[i], g[i + 1])));
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float s = j ? s2.y : s2.x, t = g[i + j] * s, slope = fmaf(t, 1.0f - s, s), p = d[i + j] * u[i + j];
        // The slope is at most 1.1, so (d u) slope loses bits only where the result is below 2^-126.  Where d u passes
        // fp32 the slope goes before u: it may be 0, and a closed gate's gradient meets no infinity.  (d slope always
        // first lost results whose d slope is below 2^-126; it took 0.2 us less of 101 for 32768 x 2048, 0.6 of 45 for
        // 1996 x 14336, 0.9 of 21 for 31962 x 288.)
        dg[i + j] = p * slope;
        if (isinf(p)) dg[i + j] = d[i + j] * slope * u[i + j];
        du[i + j] = d[i + j] * t;
        u[i + j] *= t;
      }
    }
    L::store(d_gate + row * ldg + c, left, lane, dg);
    L::store(d_up + row * ldg + c, left, lane, du);
    if (h) L::store(h + row * ldh + c, left, lane, u);
  }
}

uintptr_t bits(const void* p) { return reinterpret_cast<uintptr_t>(p); }

template <typename F>
cudaError_t by_type(int type, F f) {
  switch (type) {
    case kElemBf16: return f(__nv_bfloat16{});
    case kElemF16: return f(__half{});
    case kElemF32: return f(0.f);
    default: return cudaErrorInvalidValue;
  }
}
// Columns an access, for rows of T whose addresses and strides make up ``at`` and the kept rows.
template <typename T, typename F>
cudaError_t by_alignment(uintptr_t at, const SwigluArgs& a, F f) {
  const uintptr_t cols = at / sizeof(T) | bits(a.gate_q) | bits(a.up_q) | static_cast<uintptr_t>(a.ldq);
  if constexpr (sizeof(T) == 2) {
    if (cols % 8 == 0) return f(std::integral_constant<int, 8>{});
  }
  if (cols % 4 == 0) return f(std::integral_constant<int, 4>{});
  if (cols % 2 == 0) return f(std::integral_constant<int, 2>{});
  return f(std::integral_constant<int, 1>{});
}
unsigned grid_of(const SwigluArgs& a, int team, int most) {
  const long long groups = static_cast<long long>(a.rows) * ceil_div(a.cols, 128);
  const int teams = kThreads / team;
  return static_cast<unsigned>(std::min<long long>((groups + teams - 1) / teams, 152 * most));
}

}  // namespace

cudaError_t launch_swiglu_save(int type, const void* gate, const void* up, long long ld, void* h, long long ldh,
                               const SwigluArgs& a, cudaStream_t s) {
  return by_type(type, [&](auto t) {
    using T = decltype(t);
    const uintptr_t at = bits(gate) | bits(up) | bits(h) | static_cast<uintptr_t>((ld | ldh) * sizeof(T));
    return by_alignment<T>(at, a, [&](auto v) {
      constexpr int V = decltype(v)::value;
      return launch_pdl(swiglu_save_kernel<T, V>, grid_of(a, save_team(V), kSaveGrid), kThreads, 0, s, 1,
                        static_cast<const T*>(gate), static_cast<const T*>(up), ld, static_cast<T*>(h), ldh, a);
    });
  });
}

cudaError_t launch_swiglu_backward(int type, const void* d_h, long long ldd, void* d_gate, void* d_up, long long ldg,
                                   void* h, long long ldh, const SwigluArgs& a, cudaStream_t s) {
  return by_type(type, [&](auto t) {
    using T = decltype(t);
    uintptr_t at = bits(d_h) | bits(d_gate) | bits(d_up) | bits(h) | static_cast<uintptr_t>((ldd | ldg) * sizeof(T));
    if (h) at |= static_cast<uintptr_t>(ldh * sizeof(T));
    return by_alignment<T>(at, a, [&](auto v) {
      constexpr int V = decltype(v)::value;
      return launch_pdl(swiglu_backward_kernel<T, V>, grid_of(a, grad_team(V), kGradGrid), kThreads, 0, s, 1,
                        static_cast<const T*>(d_h), ldd, static_cast<T*>(d_gate), static_cast<T*>(d_up), ldg,
                        static_cast<T*>(h), ldh, a);
    });
  });
}

}  // namespace asap

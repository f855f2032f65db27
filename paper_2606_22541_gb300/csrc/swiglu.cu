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
constexpr int kTeam = 8;  // lanes of a group of 128 columns, 16 columns each
constexpr int kTeams = kThreads / kTeam;

// 1 / (1 + e^-g).  fp32 results take expf and a division; 16-bit ones, whose
// rounding is 2^14 times coarser, the fast exponential and reciprocal (within
// 2 + 1.16 |g| and 2 units of 2^-23 by CUDA's documentation; 0 where e^-g passes
// 2^126, as it is there to 38 digits).
template <typename T>
__device__ __forceinline__ float sigmoid(float g) {
  if constexpr (sizeof(T) == 4)
    return 1.0f / (1.0f + expf(-g));
  else
    return __fdividef(1.0f, 1.0f + __expf(-g));
}

// 16 columns of a lane, W per access.
template <typename T, int W>
__device__ __forceinline__ void load16(const T* p, int left, float (&f)[16]) {
#pragma unroll
  for (int i = 0; i < 16; i += W) {
    Cols<T, W> c;
    c.load(p + i, left - i);
    float v[W];
    c.to(v);
#pragma unroll
    for (int j = 0; j < W; ++j) f[i + j] = v[j];
  }
}
template <typename T, int W>
__device__ __forceinline__ void store16(T* p, int left, const float (&f)[16]) {
#pragma unroll
  for (int i = 0; i < 16; i += W) {
    float v[W];
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] = f[i + j];
    Cols<T, W> c;
    c.from(v);
    if (left > i) c.store(p + i, left - i);
  }
}
__device__ __forceinline__ void store_q(uint8_t* p, bool wide, int left, const uint32_t (&w)[4]) {
  if (wide && left >= 16) {
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    return;
  }
#pragma unroll
  for (int j = 0; j < 16; ++j)
    if (j < left) p[j] = static_cast<uint8_t>(w[j >> 2] >> (8 * (j & 3)));
}
__device__ __forceinline__ void load_q(const uint8_t* p, bool wide, int left, float s, float (&f)[16]) {
  uint32_t w[4] = {0, 0, 0, 0};
  if (wide && left >= 16) {
    const uint4 v = ld_dep(reinterpret_cast<const uint4*>(p));
    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
  } else {
#pragma unroll
    for (int j = 0; j < 16; ++j)
      if (j < left) w[j >> 2] |= static_cast<uint32_t>(*const_cast<const volatile uint8_t*>(p + j)) << (8 * (j & 3));
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const __half2 h = __half2(__nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w[j >> 1] >> (16 * (j & 1))),
                                                         __NV_E4M3));
    const float2 v = __half22float2(h);
    f[2 * j] = s * v.x;
    f[2 * j + 1] = s * v.y;
  }
}

// Rows and groups of a team: the groups first, first + teams, ... of rows x groups.
struct Walk {
  int row, grp, dr, dg, groups;
  __device__ __forceinline__ Walk(int cols) {
    groups = (cols + 127) / 128;
    const int teams = gridDim.x * kTeams;
    const int first = blockIdx.x * kTeams + threadIdx.x / kTeam;
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
__device__ __forceinline__ float amax16(const float (&f)[16]) {
  float m = 0.f;  // (a NaN loses)
#pragma unroll
  for (int i = 0; i < 16; ++i) m = fmaxf(m, fabsf(f[i]));
#pragma unroll
  for (int o = kTeam / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kFull, m, o));
  return m;
}

template <typename T, int W>
__global__ void __launch_bounds__(kThreads)
    swiglu_save_kernel(const T* gate, const T* up, long long ld, T* __restrict__ h, long long ldh, const SwigluArgs a,
                       bool wide_q) {
  pdl_wait();
  pdl_launch();
  const int lane = threadIdx.x & (kTeam - 1), rows = filled(a);
  // (a warp's teams leave together: their shuffles name the whole warp)
  for (Walk at(a.cols); __any_sync(kFull, at.row < rows); at.next()) {
    const int c = at.grp * 128 + lane * 16;
    const bool in = at.row < rows && c < a.cols;
    const int left = in ? a.cols - c : 0;
    float g[16], u[16];
    load16<T, W>(gate + at.row * ld + c, left, g);
    load16<T, W>(up + at.row * ld + c, left, u);
    const GroupScale gs(amax16(g)), us(amax16(u));
    if (!in) continue;
    uint32_t q[4];
    e4m3x16(gs, g, q);
    store_q(a.gate_q + at.row * a.ldq + c, wide_q, left, q);
    e4m3x16(us, u, q);
    store_q(a.up_q + at.row * a.ldq + c, wide_q, left, q);
    if (lane == 0) {
      a.gate_s[at.row * a.lds + at.grp] = gs.s;
      a.up_s[at.row * a.lds + at.grp] = us.s;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) g[i] = g[i] * sigmoid<T>(g[i]) * u[i];
    store16<T, W>(h + at.row * ldh + c, left, g);
  }
}

template <typename T, int W>
__global__ void __launch_bounds__(kThreads)
    swiglu_backward_kernel(const T* d_h, long long ldd, T* __restrict__ d_gate, T* __restrict__ d_up, long long ldg,
                           T* __restrict__ h, long long ldh, const SwigluArgs a, bool wide_q) {
  pdl_wait();
  pdl_launch();
  const int lane = threadIdx.x & (kTeam - 1), rows = filled(a);
  for (Walk at(a.cols); at.row < rows; at.next()) {
    const int c = at.grp * 128 + lane * 16;
    if (c >= a.cols) continue;
    const int left = a.cols - c;
    float d[16], g[16], u[16];
    load16<T, W>(d_h + at.row * ldd + c, left, d);
    load_q(a.gate_q + at.row * a.ldq + c, wide_q, left, ld_dep(a.gate_s + at.row * a.lds + at.grp), g);
    load_q(a.up_q + at.row * a.ldq + c, wide_q, left, ld_dep(a.up_s + at.row * a.lds + at.grp), u);
    float dg[16], du[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float s = sigmoid<T>(g[i]), t = g[i] * s;
      dg[i] = d[i] * u[i] * fmaf(t, 1.0f - s, s);
      du[i] = d[i] * t;
      u[i] *= t;
    }
    store16<T, W>(d_gate + at.row * ldg + c, left, dg);
    store16<T, W>(d_up + at.row * ldg + c, left, du);
    if (h) store16<T, W>(h + at.row * ldh + c, left, u);
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
// Columns per access, by the alignment (in bytes) of every row.
template <typename F>
cudaError_t by_alignment(uintptr_t at, int elem, F f) {
  if (at % 16 == 0) return f(std::integral_constant<int, 8>{});
  if (at % (4 * elem) == 0) return f(std::integral_constant<int, 4>{});
  return f(std::integral_constant<int, 1>{});
}
unsigned grid_of(const SwigluArgs& a) {
  const long long groups = static_cast<long long>(a.rows) * ceil_div(a.cols, 128);
  return static_cast<unsigned>(std::min<long long>((groups + kTeams - 1) / kTeams, 152 * 32));
}
bool wide(const SwigluArgs& a) { return ((bits(a.gate_q) | bits(a.up_q) | static_cast<uintptr_t>(a.ldq)) & 15u) == 0; }

}  // namespace

cudaError_t launch_swiglu_save(int type, const void* gate, const void* up, long long ld, void* h, long long ldh,
                               const SwigluArgs& a, cudaStream_t s) {
  return by_type(type, [&](auto t) {
    using T = decltype(t);
    const uintptr_t at = bits(gate) | bits(up) | bits(h) | static_cast<uintptr_t>((ld | ldh) * sizeof(T));
    return by_alignment(at, sizeof(T), [&](auto w) {
      return launch_pdl(swiglu_save_kernel<T, decltype(w)::value>, grid_of(a), kThreads, 0, s, 1,
                        static_cast<const T*>(gate), static_cast<const T*>(up), ld, static_cast<T*>(h), ldh, a, wide(a));
    });
  });
}

cudaError_t launch_swiglu_backward(int type, const void* d_h, long long ldd, void* d_gate, void* d_up, long long ldg,
                                   void* h, long long ldh, const SwigluArgs& a, cudaStream_t s) {
  return by_type(type, [&](auto t) {
    using T = decltype(t);
    uintptr_t at = bits(d_h) | bits(d_gate) | bits(d_up) | bits(h) | static_cast<uintptr_t>((ldd | ldg) * sizeof(T));
    if (h) at |= static_cast<uintptr_t>(ldh * sizeof(T));
    return by_alignment(at, sizeof(T), [&](auto w) {
      return launch_pdl(swiglu_backward_kernel<T, decltype(w)::value>, grid_of(a), kThreads, 0, s, 1,
                        static_cast<const T*>(d_h), ldd, static_cast<T*>(d_gate), static_cast<T*>(d_up), ldg,
                        static_cast<T*>(h), ldh, a, wide(a));
    });
  });
}

}  // namespace asap

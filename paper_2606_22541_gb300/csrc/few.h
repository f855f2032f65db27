// The layer for a few tokens (few.cu): arguments of its two kernels and the
// limits its host side and its kernels share.
#pragma once

#include "internal.h"

namespace asap {

constexpr int kFewTokens = 64;                // tokens of a call at most (one bit each in a 64-bit mask)
constexpr int kFewCluster = 16;               // CTAs of the route kernel
constexpr int kFewMaxStages = 8;              // ring stages of either operand at most
constexpr size_t kFewSmemState = 18944;       // barriers, queue and metadata behind the rings
constexpr size_t kFewSmem = 227 * 1024;       // dynamic shared memory of a few_ffn_kernel CTA at most
constexpr size_t kFewRouteSmem = (448 + 2 * 4 * 256) * kFewTokens;  // rows, partial and gathered logits at most

// Routing as the second kernel reads it.  Active experts are in increasing
// order; expert j's tokens are the bits of mask[j], its rows start[j] .. of the
// routed rows, in token order.
struct FewMeta {
  int active;
  int pad[3];
  int expert[256];
  int start[256];
  int row8[256];                 // groups of 8 operand rows before expert j's
  unsigned long long mask[256];
  int pos[kFewTokens * 8];       // (token t, slot j) at t * k + j -> routed row, -1: no expert
  float w[kFewTokens * 8];
};

struct FewArgs {
  LayerRef lref;
  GateParams gate;
  uint32_t* status;
  const void* x;
  void* out;
  int n, H, I, Is;               // Is 0: no shared expert
  int max_active;                // min(E, n * k)
  int s1, s2, s2s;               // K slices of a gate/up, a down and a shared down tile
  int stages_w, stages_x, x_slot;  // rings: stages, bytes of a stage of operand rows
  size_t smem;
  // workspace
  FewMeta* meta;
  int* counters;                 // [0] claims, [1 ..] arrivals per gate/up tile, per output tile, h tiles done per expert
  int n_counters, down_tickets, h_ready;
  uint8_t* ximg;                 // hidden states as operand image
  uint8_t* himg;                 // h as operand image: the shared expert's, then the active experts'
  float *p1, *p1s;               // gate/up partial sums [s1][n k][2 I], [s1][n][2 Is]
  float *y, *ys;                 // down partial sums [s2][n k][H], [s2s][n][H]
};

cudaError_t few_set_attributes();
cudaError_t few_launch(const FewArgs& a, bool fp8, int grid, cudaStream_t st);

__host__ __device__ constexpr int ceil_div_dev(int a, int b) { return (a + b - 1) / b; }
__host__ __device__ constexpr int round_up_dev(int a, int b) { return (a + b - 1) / b * b; }

}  // namespace asap

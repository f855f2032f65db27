// The layer for a few tokens (few.cu): arguments of its two kernels and the
// limits its host side and its kernels share.
#pragma once

#include "internal.h"

namespace asap {

constexpr int kFewTokens = 64;                // tokens of a call at most (one bit each in a 64-bit mask)
constexpr int kFewMaxStages = 8;              // ring stages of either operand at most
constexpr size_t kFewSmemState = 25600;       // barriers, queue and metadata behind the rings
constexpr size_t kFewSmem = 227 * 1024;       // dynamic shared memory of a few_ffn_kernel CTA at most
struct FewArgs {
  LayerRef lref;
  int fixed_layer;               // *lref.layer never changes
  GateParams gate;
  uint32_t* status;
  const void* x;
  void* out;
  int n, H, I, Is;               // Is 0: no shared expert
  int max_active;                // min(E, n * k)
  int s1, s2, s2s;               // K slices of a gate/up, a down and a shared down tile
  int out_tokens;                // tokens of an output item: 1, or one per epilogue warp
  int first_routed;              // work items in front of the first that needs the routing
  float r_s1, r_s2, r_s2s, r_tI, r_tH, r_down;  // reciprocals: of the slices, tiles and down items of an expert
  int stages_w, stages_x, x_slot;  // rings: stages, bytes of a stage of operand rows
  size_t smem;
  // workspace
  float* logits;                 // [8][n][E] partial sums
  int* counters;                 // [0] claims, [1 ..] arrivals per gate/up tile, per output tile, h tiles done per expert
  int n_counters, down_tickets, h_ready, gate_claims;  // (gate_claims: tokens claimed, tokens gated)
  int* sel_e;                    // [n][k] experts and weights of gated tokens
  float* sel_w;
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

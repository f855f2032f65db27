// Tokens sorted by expert and back on plain tensors (rows.cu), and SwiGLU with
// kept activations (swiglu.cu).
#pragma once

#include "internal.h"

namespace asap {

enum ElemType { kElemBf16 = 0, kElemF16 = 1, kElemF32 = 2, kElemE4m3 = 3 };

constexpr int kSortMaxExperts = 1024;

size_t sort_workspace(long long entries, int experts);
cudaError_t launch_sort(const int32_t* idx, long long entries, int k, int E, int32_t* offsets, int32_t* perm_dst,
                        int32_t* perm_src, void* ws, cudaStream_t s);

// Rows of n tokens, k places each (perm [n][k]; -1: none) among the rows of y.
struct RowsArgs {
  const int32_t* perm;
  int n, k;
  int rows;           // of y: places outside are skipped and recorded
  int cols;
  const float* w;     // [n][k] or NULL
  uint32_t* status;
};

cudaError_t launch_permute(int elem_bytes, const void* x, long long ldx, void* y, long long ldy, const RowsArgs& a,
                           cudaStream_t s);
cudaError_t launch_unpermute(int type, const void* y, long long ldy, void* out, long long ldo, const RowsArgs& a,
                             cudaStream_t s);
cudaError_t launch_unpermute_backward(int type, const void* d_out, long long ldo, const void* y, long long ldy, void* d_y,
                                      long long ldd, float* d_w, const RowsArgs& a, cudaStream_t s);
// a.perm NULL: row t to place t
cudaError_t launch_dequantize(int type, const void* q, long long ldq, const float* scales, long long lds, void* y,
                              long long ldy, const RowsArgs& a, cudaStream_t s);

struct SwigluArgs {
  int rows, cols;
  const int32_t* n_rows;  // NULL, or how many rows there are (device)
  uint8_t *gate_q, *up_q;
  long long ldq;
  float *gate_s, *up_s;
  long long lds;
};
cudaError_t launch_swiglu_save(int type, const void* gate, const void* up, long long ld, void* h, long long ldh,
                               const SwigluArgs& a, cudaStream_t s);
cudaError_t launch_swiglu_backward(int type, const void* d_h, long long ldd, void* d_gate, void* d_up, long long ldg,
                                   void* h, long long ldh, const SwigluArgs& a, cudaStream_t s);

}  // namespace asap

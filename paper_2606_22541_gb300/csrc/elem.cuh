// Element types of the operators on plain tensors (bf16, fp16, fp32): N
// neighbouring columns of a row to fp32 and back, in as few accesses as their
// alignment allows.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace asap {

template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  if constexpr (std::is_same_v<T, __half>) {
    const __half2 p = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&p);
  } else {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&p);
  }
}
template <typename T>
__device__ __forceinline__ float2 unpack2(uint32_t v) {
  if constexpr (std::is_same_v<T, __half>)
    return __half22float2(*reinterpret_cast<const __half2*>(&v));
  else
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
}

// N columns as they lie in memory (N a power of two up to 8; the address is a
// multiple of N elements, or of 16 bytes).
template <typename T, int N>
struct Cols {
  static constexpr int kBytes = N * static_cast<int>(sizeof(T));
  static constexpr int kWords = kBytes >= 4 ? kBytes / 4 : 1;
  uint32_t w[kWords];

  // Coherent loads that stay behind pdl_wait (volatile).
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (kBytes >= 16) {
#pragma unroll
      for (int i = 0; i < kWords; i += 4)
        asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3])
                     : "l"(reinterpret_cast<const char*>(p) + 4 * i));
    } else if constexpr (kBytes == 8) {
      asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
    } else if constexpr (kBytes == 4) {
      asm volatile("ld.global.b32 %0, [%1];" : "=r"(w[0]) : "l"(p));
    } else {
      uint16_t v;
      asm volatile("ld.global.b16 %0, [%1];" : "=h"(v) : "l"(p));
      w[0] = v;
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (kBytes >= 16) {
#pragma unroll
      for (int i = 0; i < kWords; i += 4)
        *reinterpret_cast<uint4*>(reinterpret_cast<char*>(p) + 4 * i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
    } else if constexpr (kBytes == 8) {
      *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    } else if constexpr (kBytes == 4) {
      *reinterpret_cast<uint32_t*>(p) = w[0];
    } else {
      *reinterpret_cast<uint16_t*>(p) = static_cast<uint16_t>(w[0]);
    }
  }
  // The first ``left`` columns alone; the others are zero.
  __device__ __forceinline__ void load(const T* p, int left) {
    if (left >= N) {
      load(p);
      return;
    }
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < left) {
        if constexpr (sizeof(T) == 4) {
          asm volatile("ld.global.b32 %0, [%1];" : "=r"(w[i]) : "l"(p + i));
        } else {
          uint16_t v;
          asm volatile("ld.global.b16 %0, [%1];" : "=h"(v) : "l"(p + i));
          w[i / 2] |= static_cast<uint32_t>(v) << (16 * (i & 1));
        }
      }
  }
  __device__ __forceinline__ void store(T* p, int left) const {
    if (left >= N) {
      store(p);
      return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < left) {
        if constexpr (sizeof(T) == 4)
          reinterpret_cast<uint32_t*>(p)[i] = w[i];
        else
          reinterpret_cast<uint16_t*>(p)[i] = static_cast<uint16_t>(w[i / 2] >> (16 * (i & 1)));
      }
  }
  __device__ __forceinline__ void to(float (&f)[N]) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < N; ++i) f[i] = __uint_as_float(w[i]);
    } else if constexpr (N == 1) {
      f[0] = unpack2<T>(w[0]).x;
    } else {
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        const float2 v = unpack2<T>(w[i]);
        f[2 * i] = v.x;
        f[2 * i + 1] = v.y;
      }
    }
  }
  __device__ __forceinline__ void from(const float (&f)[N]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = __float_as_uint(f[i]);
    } else if constexpr (N == 1) {
      w[0] = pack2<T>(f[0], 0.f);
    } else {
#pragma unroll
      for (int i = 0; i < N / 2; ++i) w[i] = pack2<T>(f[2 * i], f[2 * i + 1]);
    }
  }
};

}  // namespace asap

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

// Rows at any address are still read and written 16 bytes at a time: written
// where the row itself has them on 16 bytes, read by the aligned 16 bytes that hold
// them, shifted.  N: elements of 16 bytes.
template <typename T>
struct Any {
  static constexpr int kSize = static_cast<int>(sizeof(T)), N = 16 / kSize;
  using V = Cols<T, N>;

  // Elements by which a row starts behind a boundary.
  __device__ static __forceinline__ int past(const T* row) {
    return static_cast<int>(reinterpret_cast<uintptr_t>(row) & 15) / kSize;
  }
  // Bytes o .. o + 15 of lo and hi, 0 <= o <= 16.
  __device__ static __forceinline__ V shifted(const V& lo, const V& hi, int o) {
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = lo.w[i], b[4 + i] = hi.w[i];
    if (o & 16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) b[i] = b[i + 4];
    }
    if (o & 8) {
#pragma unroll
      for (int i = 0; i < 6; ++i) b[i] = b[i + 2];
    }
    if (o & 4) {
#pragma unroll
      for (int i = 0; i < 5; ++i) b[i] = b[i + 1];
    }
    V v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v.w[i] = kSize == 4 ? b[i] : __funnelshift_r(b[i], b[i + 1], 8 * (o & 3));
    return v;
  }
  // The N columns ``pre`` before those of hi, lo being the N before it.
  __device__ static __forceinline__ V before(const V& lo, const V& hi, int pre) {
    return pre == 0 ? hi : shifted(lo, hi, 16 - pre * kSize);
  }

  // Columns c .. c + N - 1 of a row (cols > 0, c > -N) in two steps, so that several rows' loads are on their way before the
  // first is looked at: the two aligned 16 bytes that hold them, then the columns.  Of the 16 bytes only those that hold
  // some of the row are read (they lie in one allocation with it; others are replaced by the nearest); what lies beside the
  // row comes along.
  struct Raw {
    V lo, hi;
  };
  __device__ static __forceinline__ Raw fetch(const T* row, int c, int cols) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(row);
    const int pre = static_cast<int>(at & 15) / kSize;
    const int last = (pre + cols - 1) / N, i = (pre + c) >= 0 ? (pre + c) / N : -1;
    const T* base = reinterpret_cast<const T*>(at & ~static_cast<uintptr_t>(15));
    Raw r;
    r.lo.load(base + static_cast<long long>(min(max(i, 0), last)) * N);
    r.hi.load(base + static_cast<long long>(min(i + 1, last)) * N);
    return r;
  }
  __device__ static __forceinline__ V columns(const Raw& r, const T* row, int c) {
    const int o = static_cast<int>(reinterpret_cast<uintptr_t>(row + c) & 15);
    return o == 0 ? r.lo : shifted(r.lo, r.hi, o);
  }
  // Columns c .. c + N - 1 back into a row, c on a boundary: those inside it.
  __device__ static __forceinline__ void store(T* row, int c, int cols, const V& v) {
    if (c >= 0 && c + N <= cols) {
      v.store(row + c);
      return;
    }
    char* to = reinterpret_cast<char*>(row + c);
    if (c >= 0) {  // the first n bytes, the larger pieces first
      const int n = (cols - c) * kSize;
      const uint32_t word = n & 8 ? v.w[2] : v.w[0], next = n & 8 ? v.w[3] : v.w[1], half = n & 4 ? next : word;
      if (n & 8) *reinterpret_cast<uint2*>(to) = make_uint2(v.w[0], v.w[1]);
      if (n & 4) *reinterpret_cast<uint32_t*>(to + (n & 8)) = word;
      if (kSize <= 2 && n & 2) *reinterpret_cast<uint16_t*>(to + (n & 12)) = static_cast<uint16_t>(half);
      if (kSize == 1 && n & 1) to[n & 14] = static_cast<char>(n & 2 ? half >> 16 : half);
    } else if (c + N <= cols) {  // the last n
      const int n = (c + N) * kSize;
      const uint32_t word = n & 8 ? v.w[1] : v.w[3], before_word = n & 8 ? v.w[0] : v.w[2];
      const uint32_t half = n & 4 ? before_word : word;
      if (n & 8) *reinterpret_cast<uint2*>(to + 8) = make_uint2(v.w[2], v.w[3]);
      if (n & 4) *reinterpret_cast<uint32_t*>(to + 12 - (n & 8)) = word;
      if (kSize <= 2 && n & 2) *reinterpret_cast<uint16_t*>(to + 14 - (n & 12)) = static_cast<uint16_t>(half >> 16);
      if (kSize == 1 && n & 1) to[15 - (n & 14)] = static_cast<char>(n & 2 ? half >> 8 : half >> 24);
    } else {  // a row of less than 16 bytes
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (c + i >= 0 && c + i < cols) {
          if constexpr (kSize == 4)
            reinterpret_cast<uint32_t*>(row)[c + i] = v.w[i];
          else if constexpr (kSize == 2)
            reinterpret_cast<uint16_t*>(row)[c + i] = static_cast<uint16_t>(v.w[i / 2] >> (16 * (i & 1)));
          else
            reinterpret_cast<uint8_t*>(row)[c + i] = static_cast<uint8_t>(v.w[i / 4] >> (8 * (i & 3)));
        }
    }
  }
};

}  // namespace asap

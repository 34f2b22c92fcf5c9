// Row-wise helpers of the tower's memory-bound kernels (gfx950): rows of whole
// 16-byte chunks, read and written by groups of 4 to 64 lanes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.hpp"

namespace infcl {

// Element types as template parameters (the codes of infcl_dtype).
constexpr int kBF16 = 0, kF32 = 1, kF16 = 2;

// 16 bytes of type T as floats: 8 values (16-bit) or 4 (fp32).
template <int T>
struct Chunk {
  static constexpr int N = T == kF32 ? 4 : 8;
  static __device__ __forceinline__ void load(const u32x4& c, float (&x)[N]) {
    if constexpr (T == kF32) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(c[i]);
    } else if constexpr (T == kBF16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(c[i] << 16);
        x[2 * i + 1] = __uint_as_float(c[i] & 0xFFFF0000u);
      }
    } else {
      const f16x8 h = __builtin_bit_cast(f16x8, c);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = (float)h[i];
    }
  }
  static __device__ __forceinline__ u32x4 store(const float (&x)[N]) {
    u32x4 c;
    if constexpr (T == kF32) {
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = __float_as_uint(x[i]);
    } else if constexpr (T == kBF16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = pk_bf16(x[2 * i], x[2 * i + 1]);
    } else {
      f16x8 h;
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] = (_Float16)x[i];
      c = __builtin_bit_cast(u32x4, h);
    }
    return c;
  }
};

// Lanes that share a row of c chunks: the power of two in [lo, 64] that covers
// the row, or 64.  log2 of it.
inline int row_lanes_log2(int64_t c, int lo) {
  int s = 0;
  while ((1 << s) < lo || ((1 << s) < c && s < 6)) ++s;
  return s;
}

}  // namespace infcl

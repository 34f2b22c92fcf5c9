// Blocks of 128 entries in 8-bit floats with a power of two.
#pragma once

#include "block.hpp"

namespace infcl {

constexpr int kFp8Block = 128;
constexpr uint32_t kFp8Nan = 0x7F7F7F7Fu;

inline int64_t fp8_blocks(int64_t k) { return (k + 127) / 128; }
// Bytes from row to row: whole blocks, and one more where that is a multiple of 16 KiB (rows
// that far apart meet in few memory channels: a product of 4096 x 1024 x 65536 takes 359 us
// with rows 64 KiB apart, 295 with a block more; 8192 and 4096 bytes make no difference).
inline int64_t fp8_pitch(int64_t k) {
  const int64_t p = fp8_blocks(k) * 128;
  return p > 0 && p % 16384 == 0 ? p + 128 : p;
}
// Exponents of a row: words of four, 127 past the last block.
inline int64_t fp8_ep(int64_t k) { return (fp8_blocks(k) + 3) / 4 * 4; }

__device__ __forceinline__ uint32_t top_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// The exponent byte of a block whose largest |x| has these bits: the least e >= -126 with
// max 2^-e <= 448 = 1.75 2^8, plus 127.  A fraction above .75 (0x600000) carries into
// the exponent.  255 where an entry is not finite.
__device__ __forceinline__ uint32_t fp8_exponent(uint32_t m) {
  if (m >= 0x7F800000u) return 255;
  const int b = (int)((m + 0x1FFFFFu) >> 23) - 8;
  return (uint32_t)(b < 1 ? 1 : b);
}
// 2^-e: exact, and so are the products with it that do not round to zero anyway.
__device__ __forceinline__ float fp8_inverse(uint32_t byte) { return __uint_as_float((254u - (byte == 255 ? 254u : byte)) << 23); }

// Four entries, times 2^-e, as 8-bit floats (v_cvt_pk_fp8_f32 rounds to nearest even;
// nothing is above 448).
__device__ __forceinline__ uint32_t fp8_pack4(float a, float b, float c, float d, float inv) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, w, true);
}

// The largest of m over 16 lanes (a DPP row), in each of them.
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t row16_max(uint32_t m) {
  m = umax(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xF, 0xF, true));
  m = umax(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xF, 0xF, true));
  m = umax(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x141, 0xF, 0xF, true));
  return umax(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x140, 0xF, 0xF, true));
}
// ... over the four rows of 16 lanes of a wave: lanes 16 apart.
__device__ __forceinline__ uint32_t rows_max(uint32_t m) {
  const auto a = __builtin_amdgcn_permlane16_swap(m, m, false, false);
  m = umax(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(m, m, false, false);
  return umax(b[0], b[1]);
}

}  // namespace infcl

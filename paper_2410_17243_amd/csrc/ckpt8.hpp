// 8-bit checkpoint groups and the activation functions of their kernels.
#pragma once

#include "rows.hpp"

namespace infcl {

constexpr int kActNone = 0, kActGelu = 1, kActQuickGelu = 2;

// Phi(-|x|): with E = e^(-x^2/2) and t = 1 / (1 + |x| / sqrt(8)),
// the scaled complementary error function is a smooth function of t on [0, 1], and
// Phi(-|x|) = E t Q(t), Q its least relative error polynomial of degree 8 (fitted by
// reweighted least squares against erfcx in 64 bits: 4e-8; in fp32, with the
// reciprocal and exponential of the hardware, 9e-7 of the value up to |x| = 4, 2e-7
// absolute).  15 instructions and two of quarter rate; the library's erf takes
// three times as many, which showed where f is taken from 8 bits (65536 x 4096:
// 210 us with it).
__device__ __forceinline__ float phi_tail(float x, float& E) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.35355339f, fabsf(x), 1.f));
  float q = -2.959678322e-02f;
  q = fmaf(q, t, 1.425919682e-01f);
  q = fmaf(q, t, -2.442315370e-01f);
  q = fmaf(q, t, 1.397574842e-01f);
  q = fmaf(q, t, -1.381248608e-02f);
  q = fmaf(q, t, 1.015552655e-01f);
  q = fmaf(q, t, 1.214982346e-01f);
  q = fmaf(q, t, 1.411950439e-01f);
  q = fmaf(q, t, 1.410427839e-01f);
  E = exp2_hw(-0.5f * kLog2e * x * x);
  return q * t * E;
}

// f(x): x Phi(x), or x sigma(1.702 x).
template <int ACT>
__device__ __forceinline__ float act_value(float x) {
  if constexpr (ACT == kActGelu) {
    float E;
    const float q = phi_tail(x, E);
    return x * (x > 0.f ? 1.f - q : q);
  } else if constexpr (ACT == kActQuickGelu) {
    return x * __builtin_amdgcn_rcpf(1.f + exp2_hw(-1.702f * kLog2e * x));
  } else {
    return x;
  }
}
// f'(x): Phi(x) + x phi(x), or s (1 + 1.702 x (1 - s)) with s = sigma(1.702 x).
// Far on the negative side s is 0, and x s with it: no product there leaves fp32's
// range, as 1.702 x would below -2e38.
template <int ACT>
__device__ __forceinline__ float act_slope(float x) {
  if constexpr (ACT == kActGelu) {
    float E;
    const float q = phi_tail(x, E);
    return fmaf(x * 0.39894228040143268f, E, x > 0.f ? 1.f - q : q);
  } else {
    const float s = __builtin_amdgcn_rcpf(1.f + exp2_hw(-1.702f * kLog2e * x));
    return fmaf(1.702f * (1.f - s), x * s, s);
  }
}

// The 8 features of a lane whose quad holds the group: their 8 bytes and the
// group's exponent byte.  Bits of |x| order like the values, infinities and
// NaN above all.  In [64, 128) 2^e the maximum rounds to 128 from 127.5 on,
// where its 23 fraction bits reach 0x7F0000: adding 0x10000 carries those into
// the exponent.
__device__ __forceinline__ uint2 pack8(const float (&x)[8], uint32_t& byte) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t a = __float_as_uint(x[e]) & 0x7FFFFFFFu;
    m = a > m ? a : m;
  }
#pragma unroll
  for (int s = 1; s <= 2; s <<= 1) {  // (quad_perm [1,0,3,2], [2,3,0,1])
    const uint32_t o = s == 1 ? (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xF, 0xF, true)
                              : (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xF, 0xF, true);
    m = o > m ? o : m;
  }
  if (m >= 0x7F800000u) {
    byte = 255;
    return make_uint2(0, 0);
  }
  const int b = (int)((m + 0x10000u) >> 23) - 6;
  byte = (uint32_t)(b < 1 ? 1 : b);
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = x[e];
  if (byte > 248) {  // next to the largest float 64 2^122 would read back as infinity: 127 2^121 instead
    byte = 248;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = fminf(fmaxf(y[e], -0x1.FCp+127f), 0x1.FCp+127f);
  }
  const float inv = __uint_as_float((254u - byte) << 23);
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e >> 2] |= ((uint32_t)(int)rintf(y[e] * inv) & 0xFFu) << (8 * (e & 3));
  return make_uint2(w[0], w[1]);
}
// q 2^e; 0 x infinity = NaN for exponent byte 255.
__device__ __forceinline__ void unpack8(uint2 w, uint32_t byte, float (&x)[8]) {
  const float s = __uint_as_float(byte << 23);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t u = e < 4 ? w.x : w.y;
    x[e] = (float)((int)(u << (24 - 8 * (e & 3))) >> 24) * s;
  }
}

}  // namespace infcl

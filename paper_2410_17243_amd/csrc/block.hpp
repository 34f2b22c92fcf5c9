// Shared helpers of the block operators' kernels (gfx950): rows in chunks of 8
// features, sums over groups of lanes, and the counter-based generator.
#pragma once

#include "infcl_block.h"
#include "rows.hpp"

namespace infcl {

// 8 features of type T from element `at` of p (16-byte aligned).
template <int T>
__device__ __forceinline__ void load8(const void* p, int64_t at, float (&x)[8]) {
  if constexpr (T == kF32) {
    const f32x4* q = (const f32x4*)((const float*)p + at);
    const f32x4 a = q[0], b = q[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = a[e], x[4 + e] = b[e];
  } else {
    Chunk<T>::load(*(const u32x4*)((const uint16_t*)p + at), x);
  }
}
// The bits of a chunk, for loads that are to be under way together before the first is used.
template <int T>
struct Raw8 {
  u32x4 w[T == kF32 ? 2 : 1];
  __device__ __forceinline__ void load(const void* p, int64_t at) {
    const u32x4* q = (const u32x4*)((const char*)p + at * (T == kF32 ? 4 : 2));
#pragma unroll
    for (int i = 0; i < (T == kF32 ? 2 : 1); ++i) w[i] = q[i];
  }
  // (zeros where the chunk is not there)
  __device__ __forceinline__ void get(bool there, float (&x)[8]) const {
    if constexpr (T == kF32) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = there ? __uint_as_float(w[e >> 2][e & 3]) : 0.f;
    } else {
      u32x4 c = w[0];
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = there ? c[i] : 0;
      Chunk<T>::load(c, x);
    }
  }
};
template <int T>
__device__ __forceinline__ void store8(void* p, int64_t at, const float (&x)[8]) {
  if constexpr (T == kF32) {
    f32x4* q = (f32x4*)((float*)p + at);
    q[0] = f32x4{x[0], x[1], x[2], x[3]};
    q[1] = f32x4{x[4], x[5], x[6], x[7]};
  } else {
    *(u32x4*)((uint16_t*)p + at) = Chunk<T>::store(x);
  }
}
// ... past the caches with FAR: outputs larger than the L2s only push out what is read
// (dropout of 65536 x 4096 both ways 384 us, 397 through them; 50001 x 16 heads of 80 turned both ways
// 115 and 118; smaller outputs are left for who reads them next).
constexpr int64_t kL2Bytes = (int64_t)32 << 20;
template <int T, bool FAR>
__device__ __forceinline__ void store8(void* p, int64_t at, const float (&x)[8]) {
  if constexpr (!FAR) {
    store8<T>(p, at, x);
  } else if constexpr (T == kF32) {
    f32x4* q = (f32x4*)((float*)p + at);
    __builtin_nontemporal_store(f32x4{x[0], x[1], x[2], x[3]}, q);
    __builtin_nontemporal_store(f32x4{x[4], x[5], x[6], x[7]}, q + 1);
  } else {
    __builtin_nontemporal_store(Chunk<T>::store(x), (u32x4*)((uint16_t*)p + at));
  }
}
// The same where the type is one of two at run time: fp32, or T.
template <int T>
__device__ __forceinline__ void load8_or_f32(const void* p, int64_t at, bool f32, float (&x)[8]) {
  if (T == kF32 || f32)
    load8<kF32>(p, at, x);
  else
    load8<T>(p, at, x);
}

// x plus that of the lane of the other half of 2, 4, ... 64 lanes (after the same of all
// smaller groups): the four steps inside 16 lanes by DPP, the others by exchanging rows.
template <int STEP>
__device__ __forceinline__ float other_half(float x) {
  const int i = __float_as_int(x);
  if constexpr (STEP == 1)
    return __int_as_float(__builtin_amdgcn_mov_dpp(i, 0xB1, 0xF, 0xF, true));  // quad_perm [1,0,3,2]
  else if constexpr (STEP == 2)
    return __int_as_float(__builtin_amdgcn_mov_dpp(i, 0x4E, 0xF, 0xF, true));  // quad_perm [2,3,0,1]
  else if constexpr (STEP == 4)
    return __int_as_float(__builtin_amdgcn_mov_dpp(i, 0x141, 0xF, 0xF, true));  // row_half_mirror
  else
    return __int_as_float(__builtin_amdgcn_mov_dpp(i, 0x140, 0xF, 0xF, true));  // row_mirror
}
// (both halves' values, in the order of the halves, in every lane)
__device__ __forceinline__ void both16(float x, float& a, float& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  a = __uint_as_float(r[0]), b = __uint_as_float(r[1]);
}
__device__ __forceinline__ void both32(float x, float& a, float& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  a = __uint_as_float(r[0]), b = __uint_as_float(r[1]);
}
// The sum over groups of 2^ls lanes (3 to 6), in every lane of the group.
__device__ __forceinline__ float group_sum(float x, int ls) {
  x += other_half<1>(x);
  x += other_half<2>(x);
  x += other_half<4>(x);
  float a, b;
  if (ls >= 4) x += other_half<8>(x);
  if (ls >= 5) both16(x, a, b), x = a + b;
  if (ls >= 6) both32(x, a, b), x = a + b;
  return x;
}

// 128 random bits: Philox 4x32 in ten rounds (Salmon et al. 2011).  A round is two
// 32 x 32 -> 64 products; element e of a chunk of 8 takes bits 16 e and up.
struct Random128 {
  uint32_t w[4];
  __device__ __forceinline__ uint32_t bits16(int e) const { return (e & 1) ? w[e >> 1] >> 16 : w[e >> 1] & 0xFFFFu; }
};
__device__ __forceinline__ Random128 philox(uint64_t index, uint32_t site, uint64_t seed) {
  uint32_t c0 = (uint32_t)index, c1 = (uint32_t)(index >> 32), c2 = site, c3 = 0;
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p = (uint64_t)c0 * 0xD2511F53u, q = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(q >> 32) ^ c1 ^ k0;
    c2 = (uint32_t)(p >> 32) ^ c3 ^ k1;
    c1 = (uint32_t)q;
    c3 = (uint32_t)p;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{c0, c1, c2, c3}};
}

// Dropout as the kernels take it: an entry is kept where its 16 bits reach `cut`
// (65536: nothing is), and multiplied with `unit`.
struct Drop {
  const uint64_t* ptr;
  uint64_t seed, first;  // first: the chunk index of row 0
  uint32_t site, cut;
  float unit;
  __device__ __forceinline__ uint64_t the_seed() const { return ptr ? *ptr : seed; }
};
inline bool drop_ok(const infcl_drop& d) {
  return d.p >= 0.f && d.p <= 1.f && d.row0 >= 0 && ((uintptr_t)d.seed_ptr % 8) == 0;
}
inline Drop drop_of(const infcl_drop& d, int64_t width) {
  Drop r;
  r.ptr = d.seed_ptr, r.seed = d.seed, r.site = d.site;
  r.first = (uint64_t)d.row0 * (uint64_t)(width / 8);
  r.cut = (uint32_t)__builtin_rint((double)d.p * 65536.0);
  r.unit = r.cut < 65536 ? (float)(65536.0 / (65536.0 - r.cut)) : 0.f;
  return r;
}

inline bool block_aligned(const void* p, size_t a) { return p != nullptr && ((uintptr_t)p % a) == 0; }
inline bool type_known(int t) { return t == INFCL_BF16 || t == INFCL_F32 || t == INFCL_F16; }
inline infcl_status launch_status() { return hipGetLastError() == hipSuccess ? INFCL_OK : INFCL_ERR_HIP; }

}  // namespace infcl

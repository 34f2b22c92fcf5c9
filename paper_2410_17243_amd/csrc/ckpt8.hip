// Activation checkpoints in 8 bits: packing, reading back, and the activation
// functions that write and read them.
//
// 32 features of a row share a power of two 2^e, the least (e >= -126) with
// rint(max|x| 2^-e) <= 127; a feature is kept as q = rint(x 2^-e), the exponent
// as the byte e + 127.  Both scalings are exact, so the checkpoint is a
// function of x's bits alone, and q 2^e has at most seven significant bits: it
// is exact in bf16 and in fp32 and the matrix products of the backward read it
// without a second rounding.  (A free fp32 scale would save half a bit of the
// step on average and lose that.)  A group with an infinity or a NaN gets
// exponent byte 255 and q = 0, and reads back as NaN.
//
// All kernels here move each byte once and are bound by memory: 65536 x 4096 in bf16,
// packing 138 us (814 MB at 5.9 TB/s, a share of it from the last-level cache), gelu
// with the checkpoint 239 us (1.35 GB, 5.6 TB/s), its backward 259 us (5.2 TB/s).  A lane holds
// 8 features, a quad of lanes a group; a row is shared by 4 to 64 lanes.
#include "ckpt8.hpp"
#include "infcl_tower.h"

namespace infcl {
namespace {

// 8 features of type T at row r, chunk i (of 8 features): loads and stores.
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

// Packs x (and writes the activation's value, ACT != none).  Lanes past the
// row's last chunk still take part in their group's maximum, with zeros.
template <int T, int ACT>
__global__ void __launch_bounds__(256) pack_kernel(const void* __restrict__ x, int64_t stride, int64_t n, int c,
                                                   int ls, int32_t ng, uint2* __restrict__ q,
                                                   uint8_t* __restrict__ ex, void* __restrict__ out) {
  const int gl = threadIdx.x & ((1 << ls) - 1), cp = (c + 3) & ~3;
  const int64_t r0 = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> ls, nr = (int64_t)gridDim.x * 256 >> ls;
  for (int64_t r = r0; r < n; r += nr) {
    for (int i = gl; i < cp; i += 1 << ls) {
      float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (i < c) load8<T>(x, r * stride + 8 * i, v);
      uint32_t byte;
      const uint2 w = pack8(v, byte);
      if (i >= c) continue;
      q[r * c + i] = w;
      if ((i & 3) == 0) ex[r * ng + (i >> 2)] = (uint8_t)byte;
      if constexpr (ACT != kActNone) {
        float a[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] = act_value<ACT>(v[e]);
        store8<T>(out, (r * c + i) * 8, a);
      }
    }
  }
}

// Reads checkpoints back: q 2^e (MODE 0), the activation's value at it (1), or
// dy times its slope there (2).
template <int T, int ACT, int MODE>
__global__ void __launch_bounds__(256) unpack_kernel(const uint2* __restrict__ q, const uint8_t* __restrict__ ex,
                                                     const void* __restrict__ dy, int64_t stride, int64_t n, int c,
                                                     int ls, int32_t ng, void* __restrict__ out) {
  const int gl = threadIdx.x & ((1 << ls) - 1);
  const int64_t r0 = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> ls, nr = (int64_t)gridDim.x * 256 >> ls;
  for (int64_t r = r0; r < n; r += nr) {
#pragma unroll 2
    for (int i = gl; i < c; i += 1 << ls) {
      float v[8], g[8];
      if constexpr (MODE == 2) load8<T>(dy, r * stride + 8 * i, g);
      unpack8(q[r * c + i], ex[r * ng + (i >> 2)], v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (MODE == 1) v[e] = act_value<ACT>(v[e]);
        if constexpr (MODE == 2) v[e] = g[e] * act_slope<ACT>(v[e]);
        // fp16 entries above 65024 round to 65536 in 8 bits, which fp16 does not have
        if constexpr (T == kF16 && MODE != 2) v[e] = v[e] > 65504.f ? 65504.f : v[e] < -65504.f ? -65504.f : v[e];
      }
      store8<T>(out, (r * c + i) * 8, v);
    }
  }
}

struct Grid {
  int c, ls;
  int32_t ng;
  unsigned blocks;
};
Grid grid_of(int64_t n, int64_t d) {
  Grid g;
  g.c = (int)(d / 8);
  g.ls = row_lanes_log2(g.c, 4);
  g.ng = (int32_t)((d + 31) / 32);
  const int64_t b = ((n << g.ls) + 255) / 256;
  g.blocks = (unsigned)(b < 16384 ? b : 16384);
  return g;
}

template <int T>
void pack_t(const void* x, int64_t stride, int64_t n, int64_t d, int act, void* q, void* ex, void* out,
            hipStream_t st) {
  const Grid g = grid_of(n, d);
#define INFCL_PACK(A)                                                                                             \
  hipLaunchKernelGGL((pack_kernel<T, A>), dim3(g.blocks), dim3(256), 0, st, x, stride, n, g.c, g.ls, g.ng, (uint2*)q, \
                     (uint8_t*)ex, out)
  if (act == kActNone)
    INFCL_PACK(kActNone);
  else if (act == kActGelu)
    INFCL_PACK(kActGelu);
  else
    INFCL_PACK(kActQuickGelu);
#undef INFCL_PACK
}

template <int T, int MODE>
void unpack_t(const void* q, const void* ex, int64_t n, int64_t d, int act, const void* dy, int64_t stride, void* out,
              hipStream_t st) {
  const Grid g = grid_of(n, d);
#define INFCL_UNPACK(A)                                                                                           \
  hipLaunchKernelGGL((unpack_kernel<T, A, MODE>), dim3(g.blocks), dim3(256), 0, st, (const uint2*)q,              \
                     (const uint8_t*)ex, dy, stride, n, g.c, g.ls, g.ng, out)
  if constexpr (MODE == 0)
    INFCL_UNPACK(kActNone);
  else if (act == kActGelu)
    INFCL_UNPACK(kActGelu);
  else
    INFCL_UNPACK(kActQuickGelu);
#undef INFCL_UNPACK
}

bool aligned(const void* p, size_t a) { return p != nullptr && ((uintptr_t)p % a) == 0; }
bool known(int t) { return t == INFCL_BF16 || t == INFCL_F32 || t == INFCL_F16; }
bool act_known(int a) { return a == kActNone || a == kActGelu || a == kActQuickGelu; }

// Checks that every call here makes of its rows: INFCL_OK, or what is wrong.
infcl_status check(int64_t n, int64_t d, int dtype, int act, int64_t stride) {
  if (n < 0 || d < 1 || !known(dtype) || !act_known(act) || stride < d) return INFCL_ERR_INVALID;
  if (d % 8 != 0 || stride % 8 != 0 || d > ((int64_t)1 << 20) || n > ((int64_t)1 << 40) / d ||
      stride > ((int64_t)1 << 32))
    return INFCL_ERR_UNSUPPORTED;
  return INFCL_OK;
}
infcl_status launched() { return hipGetLastError() == hipSuccess ? INFCL_OK : INFCL_ERR_HIP; }

template <int MODE>
infcl_status unpack_any(const void* q, const void* ex, int64_t n, int64_t d, int dtype, int act, const void* dy,
                        int64_t stride, void* out, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  if (dtype == INFCL_BF16)
    unpack_t<kBF16, MODE>(q, ex, n, d, act, dy, stride, out, st);
  else if (dtype == INFCL_F16)
    unpack_t<kF16, MODE>(q, ex, n, d, act, dy, stride, out, st);
  else
    unpack_t<kF32, MODE>(q, ex, n, d, act, dy, stride, out, st);
  return launched();
}

}  // namespace

// f(x^) in a 16-bit type, for the weight gradient.
int launch_ckpt8_expand(const void* q, const void* ex, int64_t n, int64_t d, int dtype, int act, void* out,
                        hipStream_t st) {
  if (act == kActNone) return unpack_any<0>(q, ex, n, d, dtype, act, nullptr, d, out, st);
  return unpack_any<1>(q, ex, n, d, dtype, act, nullptr, d, out, st);
}

}  // namespace infcl

using namespace infcl;

extern "C" infcl_status infcl_ckpt8_pack(const void* x, int64_t x_stride, int64_t n, int64_t d, int dtype, void* q,
                                         void* exps, void* stream) {
  const infcl_status s = check(n, d, dtype, kActNone, x_stride);
  if (s != INFCL_OK || n == 0) return s;
  if (!aligned(x, 16) || !aligned(q, 16) || exps == nullptr) return INFCL_ERR_INVALID;
  hipStream_t st = (hipStream_t)stream;
  if (dtype == INFCL_BF16)
    pack_t<kBF16>(x, x_stride, n, d, kActNone, q, exps, nullptr, st);
  else if (dtype == INFCL_F16)
    pack_t<kF16>(x, x_stride, n, d, kActNone, q, exps, nullptr, st);
  else
    pack_t<kF32>(x, x_stride, n, d, kActNone, q, exps, nullptr, st);
  return launched();
}

extern "C" infcl_status infcl_ckpt8_unpack(const void* q, const void* exps, int64_t n, int64_t d, int dtype, void* out,
                                           void* stream) {
  const infcl_status s = check(n, d, dtype, kActNone, d);
  if (s != INFCL_OK || n == 0) return s;
  if (!aligned(q, 16) || exps == nullptr || !aligned(out, 16)) return INFCL_ERR_INVALID;
  return unpack_any<0>(q, exps, n, d, dtype, kActNone, nullptr, d, out, stream);
}

extern "C" infcl_status infcl_ckpt8_act_fwd(const void* x, int64_t x_stride, int64_t n, int64_t d, int dtype, int act,
                                            void* out, void* q, void* exps, void* stream) {
  const infcl_status s = check(n, d, dtype, act, x_stride);
  if (s != INFCL_OK) return s;
  if (act == kActNone) return INFCL_ERR_INVALID;
  if (n == 0) return INFCL_OK;
  if (!aligned(x, 16) || !aligned(q, 16) || exps == nullptr || !aligned(out, 16)) return INFCL_ERR_INVALID;
  hipStream_t st = (hipStream_t)stream;
  if (dtype == INFCL_BF16)
    pack_t<kBF16>(x, x_stride, n, d, act, q, exps, out, st);
  else if (dtype == INFCL_F16)
    pack_t<kF16>(x, x_stride, n, d, act, q, exps, out, st);
  else
    pack_t<kF32>(x, x_stride, n, d, act, q, exps, out, st);
  return launched();
}

extern "C" infcl_status infcl_ckpt8_act_bwd(const void* dy, int64_t dy_stride, const void* q, const void* exps,
                                            int64_t n, int64_t d, int dtype, int act, void* dx, void* stream) {
  const infcl_status s = check(n, d, dtype, act, dy_stride);
  if (s != INFCL_OK) return s;
  if (act == kActNone) return INFCL_ERR_INVALID;
  if (n == 0) return INFCL_OK;
  if (!aligned(dy, 16) || !aligned(q, 16) || exps == nullptr || !aligned(dx, 16)) return INFCL_ERR_INVALID;
  return unpack_any<2>(q, exps, n, d, dtype, act, dy, dy_stride, dx, stream);
}

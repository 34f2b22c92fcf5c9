// Dropout from a counter-based generator.
//
// The 128 bits of one Philox call are the 16 bits of 8 entries, a lane's chunk; the
// chunk's number is the counter, so that nothing is stored and the backward pass is
// the forward on the gradient.  (16 bits put p on multiples of 2^-16; the factor is
// the inverse of the share that is kept in earnest, so sums keep their expectation.)
// Twenty 32 x 32 products a chunk, at a quarter of the vector unit's rate: about half
// of what the chunk's bytes leave time for in 16 bits, so bound by them: 65536 x 4096 in
// bf16 (1.07 GB) 183 to 190 us, 5.7 TB/s; 2001 x 512 in fp32 3.4 us.
#include "block.hpp"

namespace infcl {
namespace {

template <int T, bool FAR>
__global__ void __launch_bounds__(256) dropout_kernel(const void* __restrict__ x, int64_t stride, int64_t chunks,
                                                      uint32_t c, const Drop drop, void* __restrict__ out) {
  const uint64_t seed = drop.the_seed();
  const int64_t step = (int64_t)gridDim.x * 256;
  const bool packed = stride == (int64_t)c * 8;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < chunks; i += step) {
    int64_t at = i * 8;
    if (!packed) {
      const int64_t r = i / c;
      at = r * stride + (i - r * c) * 8;
    }
    float v[8];
    load8<T>(x, at, v);
    const Random128 r = philox(drop.first + (uint64_t)i, drop.site, seed);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = r.bits16(e) >= drop.cut ? v[e] * drop.unit : 0.f;
    store8<T, FAR>(out, i * 8, v);
  }
}

template <int T>
void dropout_t(const void* x, int64_t stride, int64_t n, int64_t d, const Drop& r, void* out, hipStream_t st) {
  const int64_t chunks = n * (d / 8), blocks = (chunks + 255) / 256;
  const dim3 grid((unsigned)(blocks < 16384 ? blocks : 16384));
  if (n * d * (T == kF32 ? 4 : 2) > kL2Bytes)
    hipLaunchKernelGGL((dropout_kernel<T, true>), grid, dim3(256), 0, st, x, stride, chunks, (uint32_t)(d / 8), r, out);
  else
    hipLaunchKernelGGL((dropout_kernel<T, false>), grid, dim3(256), 0, st, x, stride, chunks, (uint32_t)(d / 8), r, out);
}

}  // namespace
}  // namespace infcl

using namespace infcl;

extern "C" infcl_status infcl_dropout(const void* x, int64_t x_stride, int64_t n, int64_t d, int dtype, infcl_drop drop,
                                      void* out, void* stream) {
  if (n < 0 || d < 1 || !type_known(dtype) || x_stride < d || !drop_ok(drop)) return INFCL_ERR_INVALID;
  if (d % 8 != 0 || x_stride % 8 != 0 || d > ((int64_t)1 << 31) || n > ((int64_t)1 << 40) / d ||
      x_stride > ((int64_t)1 << 32) || drop.row0 > ((int64_t)1 << 62) / d)
    return INFCL_ERR_UNSUPPORTED;
  if (n == 0) return INFCL_OK;
  if (!block_aligned(x, 16) || !block_aligned(out, 16)) return INFCL_ERR_INVALID;
  const Drop r = drop_of(drop, d);
  const int64_t stride = n == 1 ? d : x_stride;
  if (dtype == INFCL_BF16)
    dropout_t<kBF16>(x, stride, n, d, r, out, (hipStream_t)stream);
  else if (dtype == INFCL_F16)
    dropout_t<kF16>(x, stride, n, d, r, out, (hipStream_t)stream);
  else
    dropout_t<kF32>(x, stride, n, d, r, out, (hipStream_t)stream);
  return launch_status();
}

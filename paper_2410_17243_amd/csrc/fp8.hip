// Operands in 8-bit floats: packing along rows, along columns, or both in one pass;
// reading back.
//
// 128 entries in a row of the contraction share a power of two 2^e, the least that
// brings the largest of them to 448 or below; an entry is kept as the nearest 8-bit
// float (E4M3) of x 2^-e.  Both scalings are exact, so a packed operand is a function of
// x's bits alone, and the matrix unit takes e as a byte with each block: a product of
// two packed operands needs no multiplication by scales of its own.
//
// A layer's gradients contract along the rows of the same arrays that its forward
// contracts along the features of, so x (and dy, and the weights) is wanted in blocks
// along both, the second transposed.  One workgroup takes a tile of 128 rows and 128
// features, a lane 8 of each: the tile stays in registers while both kinds of maxima
// are taken, so x is read once.  Bound by the bytes: 65536 x 4096 both ways with column
// sums (1.09 GB) 207 to 210 us, 65536 x 1024 with 4096 x 1024 (278 MB) 55 to 57, 5.0 to 5.3 TB/s;
// 10007 x 776 with 1000 x 776 14 us; 4096 x 2048 along rows 7.3.
#include "fp8.hpp"

namespace infcl {
namespace {

struct PackArgs {
  const void* x;
  int64_t xs, n, d, blocks, kp, ep, tp, tep;  // blocks and pitches of a row; tp, tep: of the transpose
  uint8_t *q, *ex, *qt, *ext;
  float* sums;  // [ceil(n / 128)][d]
};

// The exponent of block b of a row; after the last block, 127 to the end of its word.
__device__ __forceinline__ void put_exponent(uint8_t* row, int64_t b, int64_t blocks, uint32_t byte) {
  row[b] = (uint8_t)byte;
  if (b == blocks - 1)
    for (int64_t i = blocks; i & 3; ++i) row[i] = 127;
}

// Along rows alone: 16 lanes take a block.
template <int T>
__global__ void __launch_bounds__(256) pack_rows(const PackArgs a) {
  const uint32_t blocks = (uint32_t)a.blocks, total = (uint32_t)a.n * blocks, step = gridDim.x * 16;  // (below 2^31)
  const int lane = threadIdx.x & 15;
  for (uint32_t i = blockIdx.x * 16 + (threadIdx.x >> 4); i < total; i += step) {
    const uint32_t at = i / blocks, block = i - at * blocks;
    const int64_t r = at, b = block, col = b * 128 + 8 * lane;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (col < a.d) load8<T>(a.x, r * a.xs + col, v);
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = umax(m, top_bits(v[e]));
    const uint32_t byte = fp8_exponent(row16_max(m));
    const float inv = fp8_inverse(byte);
    uint2 w = make_uint2(fp8_pack4(v[0], v[1], v[2], v[3], inv), fp8_pack4(v[4], v[5], v[6], v[7], inv));
    if (byte == 255) w = make_uint2(kFp8Nan, kFp8Nan);
    *(uint2*)(a.q + r * a.kp + col) = w;
    if (lane == 0) put_exponent(a.ex + r * a.ep, b, blocks, byte);
  }
}

// Both, or along columns alone, of one array or of two: a tile of 128 x 128.  Lane (g, c), c = 0..15, of the
// workgroup's 16 groups: rows 8 g .. 8 g + 7, features 8 c .. 8 c + 7.
template <int T>
__global__ void __launch_bounds__(256, 2) pack_tile(const PackArgs one, const PackArgs two, unsigned first) {
  const PackArgs& a = blockIdx.x < first ? one : two;
  __shared__ uint32_t top[4][128];
  __shared__ float sum[4][128];
  __shared__ __attribute__((aligned(16))) uint8_t tile[128 * 144];  // [feature][row], 16 bytes between rows of it
  const int c = threadIdx.x & 15, g = threadIdx.x >> 4, wave = threadIdx.x >> 6;
  const uint32_t at = blockIdx.x < first ? blockIdx.x : blockIdx.x - first, across = (uint32_t)a.blocks;
  const int64_t tiles = a.blocks, rt = at / across, ct = at % across;
  const int64_t row0 = rt * 128 + 8 * g, col = ct * 128 + 8 * c;
  const int rows = a.n - row0 < 8 ? (int)(a.n - row0) : 8;  // (none or fewer: this lane's rows are not there)
  const int cols = a.d - ct * 128 < 128 ? (int)(a.d - ct * 128) : 128;  // of the tile
  // Addresses go from row to row by additions (with products of 64 bits for each, 1366
  // instructions instead of 1147, a hundred of them at a quarter of the rate).  All loads first, of some other row
  // or chunk where there is none (one at a time, each in a branch of its own, 10007 x 776 took 16 us
  // instead of 10).
  constexpr int kSize = T == kF32 ? 4 : 2;
  Raw8<T> raw[8];
  const char* from = (const char*)a.x + ((row0 < a.n ? row0 : a.n - 1) * a.xs + (col < a.d ? col : 0)) * kSize;
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    raw[r].load(from, 0);
    from += r + 1 < rows ? a.xs * kSize : 0;
  }
  float v[8][8];
#pragma unroll
  for (int r = 0; r < 8; ++r) raw[r].get(r < rows && col < a.d, v[r]);
  if (a.q) {
    uint8_t *to = a.q + row0 * a.kp + col, *ex = a.ex + row0 * a.ep + ct;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      uint32_t m = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) m = umax(m, top_bits(v[r][e]));
      const uint32_t byte = fp8_exponent(row16_max(m));
      const float inv = fp8_inverse(byte);
      uint2 w = make_uint2(fp8_pack4(v[r][0], v[r][1], v[r][2], v[r][3], inv), fp8_pack4(v[r][4], v[r][5], v[r][6], v[r][7], inv));
      if (byte == 255) w = make_uint2(kFp8Nan, kFp8Nan);
      if (r < rows) {
        *(uint2*)to = w;
        if (c == 0) *ex = (uint8_t)byte;
      }
      to += a.kp, ex += a.ep;
    }
    if (ct == tiles - 1 && threadIdx.x < 128 && rt * 128 + threadIdx.x < a.n)  // 127 to the end of the last word
      for (int64_t i = tiles; i & 3; ++i) a.ex[(rt * 128 + threadIdx.x) * a.ep + i] = 127;
  }
  if (a.qt) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint32_t m = 0;
#pragma unroll
      for (int r = 0; r < 8; ++r) m = umax(m, top_bits(v[r][e]));
      m = rows_max(m);
      if ((threadIdx.x & 63) < 16) top[wave][8 * c + e] = m;
    }
  }
  if (a.sums) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float s = 0.f, p, q;
#pragma unroll
      for (int r = 0; r < 8; ++r) s += v[r][e];
      both16(s, p, q), s = p + q;
      both32(s, p, q), s = p + q;
      if ((threadIdx.x & 63) < 16) sum[wave][8 * c + e] = s;
    }
  }
  __syncthreads();
  if (a.sums && threadIdx.x < 128 && ct * 128 + threadIdx.x < a.d) {
    const int i = threadIdx.x;
    a.sums[rt * a.d + ct * 128 + i] = sum[0][i] + sum[1][i] + sum[2][i] + sum[3][i];
  }
  if (!a.qt) return;
  uint8_t* ext = a.ext + col * a.tep + rt;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int f = 8 * c + e;
    const uint32_t byte = fp8_exponent(umax(umax(top[0][f], top[1][f]), umax(top[2][f], top[3][f])));
    const float inv = fp8_inverse(byte);
    uint2 w = make_uint2(fp8_pack4(v[0][e], v[1][e], v[2][e], v[3][e], inv), fp8_pack4(v[4][e], v[5][e], v[6][e], v[7][e], inv));
    if (byte == 255) w = make_uint2(kFp8Nan, kFp8Nan);
    *(uint2*)(tile + f * 144 + 8 * g) = w;
    if (g == 0 && f < cols) *ext = (uint8_t)byte;
    ext += a.tep;
  }
  const int64_t down = (a.n + 127) / 128;
  if (rt == down - 1 && (int)threadIdx.x < cols)
    for (int64_t i = down; i & 3; ++i) a.ext[(ct * 128 + threadIdx.x) * a.tep + i] = 127;
  __syncthreads();
  const int f0 = threadIdx.x >> 3, byte0 = 16 * (threadIdx.x & 7);
  uint8_t* to = a.qt + (ct * 128 + f0) * a.tp + rt * 128 + byte0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {  // 8 lanes write the 128 bytes of a feature
    if (32 * i + f0 < cols) *(u32x4*)to = *(const u32x4*)(tile + (32 * i + f0) * 144 + byte0);
    to += 32 * a.tp;
  }
}

// The tiles' column sums in order, 32 columns and 16 slices to a workgroup.
template <int T>
__global__ void __launch_bounds__(512) join_columns(const float* __restrict__ part, int64_t parts, int64_t d, void* out) {
  __shared__ float lds[16][33];
  const int64_t col = (int64_t)blockIdx.x * 32 + (threadIdx.x & 31);
  const int slice = threadIdx.x >> 5;
  float s = 0.f;
  if (col < d) {
    int64_t i = slice;
    for (; i + 16 * 7 < parts; i += 16 * 8) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = part[(i + 16 * j) * d + col];
#pragma unroll
      for (int j = 0; j < 8; ++j) s += v[j];
    }
    for (; i < parts; i += 16) s += part[i * d + col];
  }
  lds[slice][threadIdx.x & 31] = s;
  __syncthreads();
  if (slice == 0 && col < d) {
    float t = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) t += lds[j][threadIdx.x];
    if constexpr (T == kF32)
      ((float*)out)[col] = t;
    else if constexpr (T == kF16)
      ((_Float16*)out)[col] = (_Float16)t;
    else
      ((__bf16*)out)[col] = (__bf16)t;
  }
}

template <int T>
__global__ void __launch_bounds__(256) unpack_rows(const uint8_t* __restrict__ q, const uint8_t* __restrict__ ex,
                                                   int64_t kp, int64_t ep, int64_t rows, int64_t k, void* out) {
  const int64_t words = (k + 3) / 4, total = rows * words, step = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += step) {
    const int64_t r = i / words, c = 4 * (i - r * words);
    const uint32_t w = *(const uint32_t*)(q + r * kp + c), byte = ex[r * ep + c / 128];
    const float s = __uint_as_float(byte << 23);  // (0 is not used: e >= -126)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (c + e >= k) break;
      const uint32_t b = w >> (8 * e) & 0xFFu, m = b & 0x7Fu;
      // 4 exponent bits from -7, 3 fraction bits: the value is that of fp32's fields with the bias moved by 120
      float x = __uint_as_float(m << 20) * 0x1p120f;
      x = m == 0x7Fu ? __uint_as_float(0x7FC00000u) : b & 0x80u ? -x : x;
      x *= s;
      // an entry next to the type's largest may round to the next power of two in 8 bits
      const float most = T == kF32 ? 0x1.fffffep127f : T == kF16 ? 65504.f : 0x1.fep127f;
      x = x > most ? most : x < -most ? -most : x;
      if constexpr (T == kF32)
        ((float*)out)[r * k + c + e] = x;
      else if constexpr (T == kF16)
        ((_Float16*)out)[r * k + c + e] = (_Float16)x;
      else
        ((__bf16*)out)[r * k + c + e] = (__bf16)x;
    }
  }
}

unsigned tiles_of(const PackArgs& a) { return (unsigned)((a.n + 127) / 128 * a.blocks); }

template <int T>
void pack_t(const PackArgs& a, void* colsum, hipStream_t st) {
  if (!a.qt && !a.sums) {
    const int64_t need = (a.n * a.blocks + 15) / 16;
    hipLaunchKernelGGL((pack_rows<T>), dim3((unsigned)(need < 16384 ? need : 16384)), dim3(256), 0, st, a);
    return;
  }
  const unsigned tiles = tiles_of(a);
  if (tiles > 0) hipLaunchKernelGGL((pack_tile<T>), dim3(tiles), dim3(256), 0, st, a, a, tiles);
  if (a.sums)
    hipLaunchKernelGGL((join_columns<T>), dim3((unsigned)((a.d + 31) / 32)), dim3(512), 0, st, (const float*)a.sums,
                       (a.n + 127) / 128, a.d, colsum);
}

bool sizes_ok(int64_t n, int64_t d) {
  return d % 8 == 0 && d <= ((int64_t)1 << 23) && n <= ((int64_t)1 << 27) && n <= ((int64_t)1 << 37) / d;
}

PackArgs args_of(const void* x, int64_t x_stride, int64_t n, int64_t d, void* q, void* exps, void* qt, void* expst) {
  PackArgs a;
  a.x = x, a.xs = x_stride, a.n = n, a.d = d, a.blocks = fp8_blocks(d), a.kp = fp8_pitch(d), a.ep = fp8_ep(d);
  a.tp = fp8_pitch(n), a.tep = fp8_ep(n);
  a.q = (uint8_t*)q, a.ex = (uint8_t*)exps, a.qt = (uint8_t*)qt, a.ext = (uint8_t*)expst, a.sums = nullptr;
  return a;
}

}  // namespace

// Two arrays, each along its rows and (qt) along its columns, in one launch; 16 bits.
infcl_status fp8_pack_two(const void* x, int64_t x_stride, int64_t n, const void* w, int64_t w_stride, int64_t m, int64_t k,
                          int dtype, void* xq, void* xe, void* xqt, void* xet, void* wq, void* we, void* wqt, void* wet,
                          hipStream_t st) {
  const PackArgs a = args_of(x, x_stride, n, k, xq, xe, xqt, xet), b = args_of(w, w_stride, m, k, wq, we, wqt, wet);
  const unsigned first = tiles_of(a), all = first + tiles_of(b);
  if (dtype == INFCL_BF16)
    hipLaunchKernelGGL((pack_tile<kBF16>), dim3(all), dim3(256), 0, st, a, b, first);
  else
    hipLaunchKernelGGL((pack_tile<kF16>), dim3(all), dim3(256), 0, st, a, b, first);
  return launch_status();
}

}  // namespace infcl

using namespace infcl;

extern "C" infcl_status infcl_fp8_pack_workspace(int64_t n, int64_t d, size_t* bytes) {
  if (!bytes || n < 0 || d < 1) return INFCL_ERR_INVALID;
  if (!sizes_ok(n, d)) return INFCL_ERR_UNSUPPORTED;
  const size_t b = (size_t)((n + 127) / 128) * (size_t)d * 4;
  *bytes = b < 256 ? 256 : (b + 255) & ~(size_t)255;
  return INFCL_OK;
}

extern "C" infcl_status infcl_fp8_pack(const void* x, int64_t x_stride, int64_t n, int64_t d, int dtype, void* q,
                                       void* exps, void* qt, void* expst, void* colsum, void* workspace,
                                       size_t ws_bytes, void* stream) {
  if (n < 0 || d < 1 || !type_known(dtype) || x_stride < d || (q != nullptr) != (exps != nullptr) ||
      (qt != nullptr) != (expst != nullptr) || (!q && !qt && !colsum))
    return INFCL_ERR_INVALID;
  if (!sizes_ok(n, d) || x_stride % 8 != 0 || x_stride > ((int64_t)1 << 32)) return INFCL_ERR_UNSUPPORTED;
  if ((n > 0 && !block_aligned(x, 16)) || ((uintptr_t)q % 16) != 0 || ((uintptr_t)exps % 4) != 0 ||
      ((uintptr_t)qt % 16) != 0 || ((uintptr_t)expst % 4) != 0 || ((uintptr_t)colsum % 4) != 0)
    return INFCL_ERR_INVALID;
  if (colsum) {
    size_t need = 0;
    infcl_fp8_pack_workspace(n, d, &need);
    if (!block_aligned(workspace, 256)) return INFCL_ERR_INVALID;
    if (ws_bytes < need) return INFCL_ERR_WORKSPACE;
  }
  if (n == 0 && !colsum) return INFCL_OK;
  PackArgs a = args_of(x, x_stride, n, d, q, exps, qt, expst);
  a.sums = colsum ? (float*)workspace : nullptr;
  hipStream_t st = (hipStream_t)stream;
  if (dtype == INFCL_BF16)
    pack_t<kBF16>(a, colsum, st);
  else if (dtype == INFCL_F16)
    pack_t<kF16>(a, colsum, st);
  else
    pack_t<kF32>(a, colsum, st);
  return launch_status();
}

extern "C" infcl_status infcl_fp8_unpack(const void* q, const void* exps, int64_t rows, int64_t k, int dtype, void* out,
                                         void* stream) {
  if (rows < 0 || k < 0 || !type_known(dtype)) return INFCL_ERR_INVALID;
  if (k > ((int64_t)1 << 27) || rows > ((int64_t)1 << 27) || (k > 0 && rows > ((int64_t)1 << 38) / k)) return INFCL_ERR_UNSUPPORTED;
  if (rows == 0 || k == 0) return INFCL_OK;
  if (!block_aligned(q, 16) || !block_aligned(exps, 4) || !block_aligned(out, 4)) return INFCL_ERR_INVALID;
  const int64_t need = (rows * ((k + 3) / 4) + 255) / 256;
  const dim3 grid((unsigned)(need < 16384 ? need : 16384));
  hipStream_t st = (hipStream_t)stream;
  const int64_t kp = fp8_pitch(k), ep = fp8_ep(k);
  const uint8_t *b = (const uint8_t*)q, *e = (const uint8_t*)exps;
  if (dtype == INFCL_BF16)
    hipLaunchKernelGGL((unpack_rows<kBF16>), grid, dim3(256), 0, st, b, e, kp, ep, rows, k, out);
  else if (dtype == INFCL_F16)
    hipLaunchKernelGGL((unpack_rows<kF16>), grid, dim3(256), 0, st, b, e, kp, ep, rows, k, out);
  else
    hipLaunchKernelGGL((unpack_rows<kF32>), grid, dim3(256), 0, st, b, e, kp, ep, rows, k, out);
  return launch_status();
}

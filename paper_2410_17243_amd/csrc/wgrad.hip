// Weight gradient from an 8-bit checkpoint: dW [m, d] = dy^T f(x^), the sum over
// n tokens of products of a row of dy and a row of f(x^).
//
// A matrix product whose two operands are both read across their rows: tiles
// of 32 tokens are copied to LDS as they lie in memory and the fragments of
// the 32x32x16 MFMA come from transposing LDS reads.  The segments of 128
// features and their chunk order are those of the loss's swept tiles
// (sweep.hpp): copies and transposing reads without bank conflicts.
// Four stages of tiles are in flight by asynchronous copies; a stage is waited
// for by the number of copies issued after it, so that copies run three steps
// ahead of the products.
//
// The tokens are cut into parts where the tiles of dW alone would leave
// compute units idle; the parts' sums are added in order by a second launch.
//
// f(x^) is first written out in 16 bits: taken in the loader, f would be taken
// again for every tile of dW that a row meets (35 instructions an element with
// gelu, nine times what the products of a 256-wide tile leave time for).
//
// 65536 tokens, 4096 x 1024, gelu: the product 501 us (1097 TFLOP/s; the library's
// product of the same operands in 16 bits 592 us), f(x^) 175 us (805 MB at 4.6
// TB/s), the sums 12 us.  2002 tokens, 512 x 512: 18 us in three launches, each
// near the time of an empty one.
#include "ckpt8.hpp"
#include "grid.hpp"
#include "infcl_tower.h"
#include "sweep.hpp"

namespace infcl {
int launch_ckpt8_expand(const void* q, const void* ex, int64_t n, int64_t d, int dtype, int act, void* out,
                        hipStream_t st);
namespace {

constexpr int kBK = kSweepBN;  // tokens of a stage
constexpr int kStages = 4;

// Waves WM x WN, each FM x FN blocks of 32 x 32; WM WN is 4 or 8, and every wave
// issues four copies a stage.
template <int WM, int WN, int FM, int FN>
struct WTile {
  static constexpr int BM = 32 * WM * FM, BN = 32 * WN * FN;
  static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
  static constexpr int kSegs = (BM + BN) / 128;
  static constexpr int kCopies = kSegs * 8 / kWaves;
  static constexpr int kStage = kSegs * kSeg;
  static_assert(kCopies == 4 && BM % 128 == 0 && BN % 128 == 0, "layout");
};

__device__ __forceinline__ bf16x8 join8(s16x4 a, s16x4 b) {
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

template <class W, int WN, int FM, int FN, bool F16, int OUT>
__global__ void __launch_bounds__(W::kThreads, 2)
    wgrad_kernel(const uint16_t* __restrict__ dy, int64_t ldy, const uint16_t* __restrict__ x, int64_t ldx, int64_t n,
                 int m, int d, int tn, int tiles, int64_t steps, void* __restrict__ out) {
  __shared__ __attribute__((aligned(1024))) char lds[kStages * W::kStage];
  const uint32_t slot = xcd_slot(blockIdx.x, gridDim.x);  // a part's tiles on neighbouring slots: shared rows
  const int part = (int)(slot / (uint32_t)tiles), tile = (int)(slot % (uint32_t)tiles);
  const int m0 = tile / tn * W::BM, d0 = tile % tn * W::BN;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t t0 = part * steps * kBK, left = n - t0;  // tokens of this part
  const int ns = (int)((left + kBK - 1) / kBK < steps ? (left + kBK - 1) / kBK : steps);

  const uint32_t yb = (uint32_t)(ldy * 2), xb = (uint32_t)(ldx * 2);
  const uint32_t vy = sweep_dma_lane_off(lane, wave & 3, (int)yb), vx = sweep_dma_lane_off(lane, wave & 3, (int)xb);
  const uint16_t* py = dy + t0 * ldy + m0;
  const uint16_t* px = x + t0 * ldx + d0;
  const uint32_t ycols = (uint32_t)(m - m0) * 2, xcols = (uint32_t)(d - d0) * 2;
  auto issue = [&](int s) {  // stage s of this part; past the part's tokens: zeros
    const int64_t rows64 = left - (int64_t)s * kBK;
    const int rows = s >= ns || rows64 <= 0 ? 0 : rows64 > kBK ? kBK : (int)rows64;
    u32x4 ry, rx;
    const uint64_t ay = (uint64_t)(py + (int64_t)s * kBK * ldy), ax = (uint64_t)(px + (int64_t)s * kBK * ldx);
    ry[0] = (uint32_t)ay, ry[1] = (uint32_t)(ay >> 32) & 0xFFFFu, ry[3] = 0x00020000u;
    rx[0] = (uint32_t)ax, rx[1] = (uint32_t)(ax >> 32) & 0xFFFFu, rx[3] = 0x00020000u;
    ry[2] = rows ? (uint32_t)(rows - 1) * yb + ycols : 0;
    rx[2] = rows ? (uint32_t)(rows - 1) * xb + xcols : 0;
    INFCL_LDS char* base = (INFCL_LDS char*)lds + (s % kStages) * W::kStage;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      const int k = wave + W::kWaves * kk, seg = k >> 3;
      const bool isy = W::kWaves * kk / 8 < W::BM / 128;  // (the segment, which the wave does not change)
      const int sc = isy ? seg : seg - W::BM / 128;
      if (isy)
        dma16_asm(ry, base + 1024 * k, vy, (uint32_t)(4 * (k & 7)) * yb + 256 * sc);
      else
        dma16_asm(rx, base + 1024 * k, vx, (uint32_t)(4 * (k & 7)) * xb + 256 * sc);
    }
  };

  const int wm = wave / WN, wn = wave % WN;
  f32x16 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  int offm[FM][2], offn[FN][2];
#pragma unroll
  for (int tt = 0; tt < 2; ++tt) {
#pragma unroll
    for (int i = 0; i < FM; ++i) offm[i][tt] = sweep_tr_off(lane, tt, wm * FM + i);
#pragma unroll
    for (int j = 0; j < FN; ++j) offn[j][tt] = sweep_tr_off(lane, tt, W::BM / 32 + wn * FN + j);
  }
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) issue(s);
  for (int s = 0; s < ns; ++s) {
    // this wave's copies of stage s are done (eight later ones may not be), and
    // with the barrier every wave's; all reads of the stage before are done too
    asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    issue(s + kStages - 1);
    const INFCL_LDS char* cur = (const INFCL_LDS char*)lds + (s % kStages) * W::kStage;
#pragma unroll
    for (int k2 = 0; k2 < kBK / 16; ++k2) {
      bf16x8 a[FM], b[FN];
#pragma unroll
      for (int i = 0; i < FM; ++i)
        a[i] = join8(__builtin_amdgcn_ds_read_tr16_b64_v4i16((INFCL_LDS s16x4*)(cur + offm[i][0] + 16 * kSegRow * k2)),
                     __builtin_amdgcn_ds_read_tr16_b64_v4i16((INFCL_LDS s16x4*)(cur + offm[i][1] + 16 * kSegRow * k2)));
#pragma unroll
      for (int j = 0; j < FN; ++j)
        b[j] = join8(__builtin_amdgcn_ds_read_tr16_b64_v4i16((INFCL_LDS s16x4*)(cur + offn[j][0] + 16 * kSegRow * k2)),
                     __builtin_amdgcn_ds_read_tr16_b64_v4i16((INFCL_LDS s16x4*)(cur + offn[j][1] + 16 * kSegRow * k2)));
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = mfma16<F16>(a[i], b[j], acc[i][j]);
    }
  }
  // Copies past the last stage wrote zeros or nothing into stages no one reads;
  // they must have landed before the workgroup's LDS is given away.
  wait_dma();

  const int h = lane >> 5, col0 = d0 + 32 * wn * FN + (lane & 31);
  const int64_t base = OUT == 0 ? (int64_t)part * m * d : 0;
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int row = m0 + 32 * (wm * FM + i) + 8 * (r >> 2) + 4 * h + (r & 3), col = col0 + 32 * j;
        if (row >= m || col >= d) continue;
        const int64_t at = base + (int64_t)row * d + col;
        if constexpr (OUT == 0)
          ((float*)out)[at] = acc[i][j][r];
        else
          ((__bf16*)out)[at] = to16<F16>(acc[i][j][r]);
      }
}

// The parts' sums in order.  OUT: kF32, kBF16 or kF16.
template <int OUT>
__global__ void __launch_bounds__(256) wgrad_sum(const f32x4* __restrict__ part, int parts, int64_t n4,
                                                 void* __restrict__ out) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 2;  // 8 values
  if (i >= n4) return;
  float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int p0 = 0; p0 < parts; p0 += 8) {  // eight parts' loads at a time
    f32x4 x[8][2];
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const int64_t at = (int64_t)(p0 + p < parts ? p0 + p : p0) * n4 + i;
      x[p][0] = part[at], x[p][1] = part[at + 1];
    }
#pragma unroll
    for (int p = 0; p < 8; ++p)
      if (p0 + p < parts)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += x[p][0][e], s[4 + e] += x[p][1][e];
  }
  if constexpr (OUT == kF32) {
    ((f32x4*)out)[i] = f32x4{s[0], s[1], s[2], s[3]};
    ((f32x4*)out)[i + 1] = f32x4{s[4], s[5], s[6], s[7]};
  } else {
    ((u32x4*)out)[i / 2] = Chunk<OUT>::store(s);
  }
}

// Large tiles read each operand half as often, small ones start sooner and fill the
// chip with less to sum (2002 tokens, 512 x 512: 11 us small, 18 large; 10007 tokens,
// 776 x 1000: 28 and 34, with more parts to add; 65536 tokens, 4096 x 1024: 501 large,
// twice the rate that the small ones reach).
typedef WTile<2, 4, 4, 2> Big;    // 256 x 256, 8 waves of 128 x 64
typedef WTile<2, 2, 2, 2> Small;  // 128 x 128, 4 waves of 64 x 64

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

struct WPlan {
  bool big;
  int tm, tn, parts;
  int64_t steps;  // stages of a part
  size_t x16, part, total;
};

WPlan wgrad_plan(int64_t n, int64_t d, int64_t m) {
  WPlan w;
  const int64_t stages = (n + kBK - 1) / kBK;
  w.big = m >= 256 && d >= 256 && ((m + 255) / 256) * ((d + 255) / 256) * stages >= 256 * 32;
  const int bm = w.big ? 256 : 128;
  w.tm = (int)((m + bm - 1) / bm), w.tn = (int)((d + bm - 1) / bm);
  const int64_t tiles = (int64_t)w.tm * w.tn, slots = w.big ? 256 : 512;
  int64_t parts = slots / tiles;
  if (parts > stages / 8) parts = stages / 8;  // a part worth its sums
  if (parts > 64) parts = 64;
  if (parts < 1) parts = 1;
  w.steps = (stages + parts - 1) / parts;
  if (w.steps < 1) w.steps = 1;
  w.parts = (int)((stages + w.steps - 1) / w.steps);
  if (w.parts < 1) w.parts = 1;
  size_t off = 0;
  w.x16 = off; off = up256(off + (size_t)n * (size_t)d * 2);
  w.part = off; off = up256(off + (w.parts > 1 ? (size_t)w.parts * (size_t)m * (size_t)d * 4 : 0));
  w.total = off < 256 ? 256 : off;
  return w;
}

template <class W, int WN, int FM, int FN, bool F16>
void launch_tiles(const WPlan& w, const void* dy, int64_t ldy, const void* x, int64_t n, int64_t d, int64_t m, int out,
                  void* to, hipStream_t st) {
  const int tiles = w.tm * w.tn;
  const dim3 grid((unsigned)((int64_t)tiles * w.parts));
  if (out == 0)
    hipLaunchKernelGGL((wgrad_kernel<W, WN, FM, FN, F16, 0>), grid, dim3(W::kThreads), 0, st, (const uint16_t*)dy, ldy,
                       (const uint16_t*)x, d, n, (int)m, (int)d, w.tn, tiles, w.steps, to);
  else
    hipLaunchKernelGGL((wgrad_kernel<W, WN, FM, FN, F16, 1>), grid, dim3(W::kThreads), 0, st, (const uint16_t*)dy, ldy,
                       (const uint16_t*)x, d, n, (int)m, (int)d, w.tn, tiles, w.steps, to);
}

template <bool F16>
int wgrad_t(const WPlan& w, const void* dy, int64_t ldy, const void* q, const void* ex, int64_t n, int64_t d, int64_t m,
            int act, void* dw, int grad, char* ws, hipStream_t st) {
  const int t = F16 ? INFCL_F16 : INFCL_BF16;
  if (n > 0) {
    const int rc = launch_ckpt8_expand(q, ex, n, d, t, act, ws + w.x16, st);
    if (rc != INFCL_OK) return rc;
  }
  const bool direct = w.parts == 1;
  void* to = direct ? dw : (void*)(ws + w.part);
  const int out = direct && grad != INFCL_F32 ? 1 : 0;
  if (w.big)
    launch_tiles<Big, 4, 4, 2, F16>(w, dy, ldy, ws + w.x16, n, d, m, out, to, st);
  else
    launch_tiles<Small, 2, 2, 2, F16>(w, dy, ldy, ws + w.x16, n, d, m, out, to, st);
  if (hipGetLastError() != hipSuccess) return INFCL_ERR_HIP;
  if (!direct) {
    const int64_t n4 = m * d / 4;
    const dim3 grid((unsigned)((n4 / 2 + 255) / 256));
    if (grad == INFCL_F32)
      hipLaunchKernelGGL((wgrad_sum<kF32>), grid, dim3(256), 0, st, (const f32x4*)to, w.parts, n4, dw);
    else
      hipLaunchKernelGGL((wgrad_sum<F16 ? kF16 : kBF16>), grid, dim3(256), 0, st, (const f32x4*)to, w.parts, n4, dw);
    if (hipGetLastError() != hipSuccess) return INFCL_ERR_HIP;
  }
  return INFCL_OK;
}

bool aligned(const void* p, size_t a) { return p != nullptr && ((uintptr_t)p % a) == 0; }
bool known(int t) { return t == INFCL_BF16 || t == INFCL_F32 || t == INFCL_F16; }
constexpr int64_t kMaxW = 1 << 20;  // widths
bool sizes_ok(int64_t n, int64_t d, int64_t m) {
  return d % 8 == 0 && m % 8 == 0 && d <= kMaxW && m <= kMaxW && n <= ((int64_t)1 << 36) / (d > m ? d : m) &&
         m * d <= ((int64_t)1 << 36);
}

}  // namespace
}  // namespace infcl

using namespace infcl;

extern "C" infcl_status infcl_ckpt8_wgrad_workspace(int64_t n, int64_t d, int64_t m, size_t* bytes) {
  if (!bytes || n < 0 || d < 1 || m < 1) return INFCL_ERR_INVALID;
  if (!sizes_ok(n, d, m)) return INFCL_ERR_UNSUPPORTED;
  *bytes = wgrad_plan(n, d, m).total;
  return INFCL_OK;
}

extern "C" infcl_status infcl_ckpt8_wgrad(const void* dy, int64_t dy_stride, const void* q, const void* exps, int64_t n,
                                          int64_t d, int64_t m, int dtype, int act, void* dw, int grad_dtype,
                                          void* workspace, size_t ws_bytes, void* stream) {
  if (n < 0 || d < 1 || m < 1 || !known(dtype) || !known(grad_dtype) || act < kActNone || act > kActQuickGelu ||
      dy_stride < m)
    return INFCL_ERR_INVALID;
  if (dtype == INFCL_F32 || (grad_dtype != INFCL_F32 && grad_dtype != dtype) || !sizes_ok(n, d, m) ||
      dy_stride % 8 != 0 || dy_stride > ((int64_t)1 << 24))
    return INFCL_ERR_UNSUPPORTED;
  if (!aligned(dw, 16) || !aligned(workspace, 256)) return INFCL_ERR_INVALID;
  if (n > 0 && (!aligned(dy, 16) || !aligned(q, 16) || exps == nullptr)) return INFCL_ERR_INVALID;
  const WPlan w = wgrad_plan(n, d, m);
  if (ws_bytes < w.total) return INFCL_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  const int rc = dtype == INFCL_BF16
                     ? wgrad_t<false>(w, dy, dy_stride, q, exps, n, d, m, act, dw, grad_dtype, (char*)workspace, st)
                     : wgrad_t<true>(w, dy, dy_stride, q, exps, n, d, m, act, dw, grad_dtype, (char*)workspace, st);
  return (infcl_status)rc;
}

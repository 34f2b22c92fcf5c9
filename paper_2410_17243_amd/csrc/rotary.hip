// Rotary positions of one to four axes.
//
// Pair f of a token is a point (u, v) of the plane, turned by the angle
// pos freqs[f]: (u cos - v sin, v cos + u sin).  The angle in turns is one fp64
// product and its distance to the nearest whole number, so positions far out lose
// nothing; sine and cosine of what is left are fp32.
//
// The angles are those of all heads of a token: a workgroup takes some tokens,
// writes their sines and cosines to LDS, and then streams the heads past them, so
// that the 100 instructions of an angle are paid once for `heads` pairs and the
// kernel is bound by the bytes it moves: 17408 tokens x 24 heads of 64 (107 MB both ways)
// 20 to 21 us, 50001 x 16 heads of 80 on three axes (256 MB) 49 us, 5.1 to 5.3 TB/s; one
// token 2.2 us, the latency of an angle and of a row.
#include "block.hpp"

namespace infcl {
namespace {

constexpr int kTable = 2048;  // angles of a workgroup

struct RotaryArgs {
  const void* x;
  void* out;
  int64_t xs, xh, os, oh;  // strides of tokens and heads, elements
  const void* pos;
  const float* freqs;
  int64_t ps, n;
  int heads, turned, hd, pairs, e1, e2, e3;  // pairs before the second, third, fourth axis
  int pos_f32;
  float sign;
  int tokens;                 // of a workgroup
  int items;                  // of a head
  uint32_t by_items, by_heads;  // 2^32 over them, rounded up (0 for 1)
};

// i / d from by = 2^32 / d rounded up: exact where i d < 2^32.
__device__ __forceinline__ uint32_t over(uint32_t i, uint32_t by) { return by ? __umulhi(i, by) : i; }

// One element.
template <int T>
__device__ __forceinline__ float load1(const void* p, int64_t at) {
  if constexpr (T == kF32)
    return ((const float*)p)[at];
  else if constexpr (T == kF16)
    return (float)((const _Float16*)p)[at];
  else
    return (float)((const __bf16*)p)[at];
}

// WHOLE: pairs are halves and a multiple of 8, an item is 8 pairs (two chunks), or a
// chunk that is copied.  Otherwise an item is one chunk of 8 features.
template <int T, bool HALVES, bool WHOLE, bool FAR>
__global__ void __launch_bounds__(256) rotary_kernel(const RotaryArgs a) {
  __shared__ float2 table[kTable];
  const int64_t t0 = (int64_t)blockIdx.x * a.tokens;
  const int nt = (int)(a.n - t0 < a.tokens ? a.n - t0 : a.tokens);
  for (int i = threadIdx.x; i < nt * a.pairs; i += 256) {
    const int t = i / a.pairs, f = i - t * a.pairs;
    const int axis = (f >= a.e1) + (f >= a.e2) + (f >= a.e3);
    const int64_t at = (t0 + t) * a.ps + axis;
    const double pos = a.pos_f32 ? (double)((const float*)a.pos)[at] : (double)((const int32_t*)a.pos)[at];
    const double turns = pos * (double)a.freqs[f] * 0.15915494309189533577;
    const float r = (float)(turns - __builtin_rint(turns));
    float s, c;
    sincospif(2.f * r, &s, &c);
    table[i] = make_float2(c, a.sign * s);
  }
  __syncthreads();
  const int total = nt * a.heads * a.items;
  for (int i = threadIdx.x; i < total; i += 256) {
    const uint32_t row = over((uint32_t)i, a.by_items), t = over(row, a.by_heads);
    const int c = i - (int)row * a.items, head = (int)row - (int)t * a.heads;
    const int64_t xi = (t0 + t) * a.xs + head * a.xh, oi = (t0 + t) * a.os + head * a.oh;
    const float2* cs = table + t * a.pairs;
    if constexpr (WHOLE) {
      const int half = a.pairs / 8;
      if (c >= half) {  // past the pairs: copied
        float u[8];
        load8<T>(a.x, xi + 8 * (c + half), u);
        store8<T, FAR>(a.out, oi + 8 * (c + half), u);
        continue;
      }
      float u[8], v[8];
      load8<T>(a.x, xi + 8 * c, u);
      load8<T>(a.x, xi + 8 * c + a.pairs, v);
      if (head < a.turned) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float2 w = cs[8 * c + e];
          const float p = u[e] * w.x - v[e] * w.y, q = v[e] * w.x + u[e] * w.y;
          u[e] = p, v[e] = q;
        }
      }
      store8<T, FAR>(a.out, oi + 8 * c, u);
      store8<T, FAR>(a.out, oi + 8 * c + a.pairs, v);
    } else {
      float u[8];
      load8<T>(a.x, xi + 8 * c, u);
      if (head < a.turned) {
        if constexpr (HALVES) {
          float y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int f = 8 * c + e, first = f < a.pairs;
            y[e] = u[e];
            if (f >= 2 * a.pairs) continue;
            const float2 w = cs[first ? f : f - a.pairs];
            const float v = load1<T>(a.x, xi + (first ? f + a.pairs : f - a.pairs));
            y[e] = first ? u[e] * w.x - v * w.y : u[e] * w.x + v * w.y;
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) u[e] = y[e];
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (4 * c + e >= a.pairs) continue;
            const float2 w = cs[4 * c + e];
            const float p = u[2 * e] * w.x - u[2 * e + 1] * w.y, q = u[2 * e + 1] * w.x + u[2 * e] * w.y;
            u[2 * e] = p, u[2 * e + 1] = q;
          }
        }
      }
      store8<T, FAR>(a.out, oi + 8 * c, u);
    }
  }
}

template <int T, bool FAR>
void rotary_far(const RotaryArgs& a, int paired, bool whole, unsigned grid, hipStream_t st) {
  if (paired == INFCL_PAIRED_NEIGHBOURS)
    hipLaunchKernelGGL((rotary_kernel<T, false, false, FAR>), dim3(grid), dim3(256), 0, st, a);
  else if (whole)
    hipLaunchKernelGGL((rotary_kernel<T, true, true, FAR>), dim3(grid), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((rotary_kernel<T, true, false, FAR>), dim3(grid), dim3(256), 0, st, a);
}
template <int T>
void rotary_t(const RotaryArgs& a, int paired, bool whole, unsigned grid, hipStream_t st) {
  if (a.n * a.heads * a.hd * (T == kF32 ? 4 : 2) > kL2Bytes)
    rotary_far<T, true>(a, paired, whole, grid, st);
  else
    rotary_far<T, false>(a, paired, whole, grid, st);
}

uint32_t by(int d) { return d == 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + d - 1) / d); }

bool view_ok(const infcl_attn_view& v, int64_t hd) { return block_aligned(v.data, 16) && v.token_stride >= hd && v.head_stride >= 0; }
bool view_supported(const infcl_attn_view& v) {
  return v.token_stride % 8 == 0 && v.head_stride % 8 == 0 && v.token_stride <= ((int64_t)1 << 32) &&
         v.head_stride <= ((int64_t)1 << 40);
}

}  // namespace
}  // namespace infcl

using namespace infcl;

extern "C" infcl_status infcl_rotary(const infcl_rotary_shape* s, infcl_attn_view x, infcl_attn_view out,
                                     const void* pos, const float* freqs, void* stream) {
  if (!s || s->n < 0 || s->heads < 1 || s->turned < 0 || s->turned > s->heads || s->head_dim < 1 ||
      !type_known(s->dtype) || (s->paired != INFCL_PAIRED_HALVES && s->paired != INFCL_PAIRED_NEIGHBOURS) ||
      (s->back != 0 && s->back != 1) || s->axes < 1 || s->axes > 4 || (s->pos_dtype != 0 && s->pos_dtype != 1) ||
      s->pos_stride < 0)
    return INFCL_ERR_INVALID;
  int64_t pairs = 0, ends[4] = {0, 0, 0, 0};
  for (int i = 0; i < 4; ++i) {
    if (i < s->axes && s->sections[i] < 1) return INFCL_ERR_INVALID;
    if (i < s->axes) pairs += s->sections[i];
    ends[i] = i + 1 < s->axes ? pairs : INT32_MAX;
  }
  if (2 * pairs > s->head_dim) return INFCL_ERR_INVALID;
  if (s->head_dim % 8 != 0 || s->head_dim > 1024 || s->heads > 4096 || s->n > ((int64_t)1 << 31) ||
      s->pos_stride > ((int64_t)1 << 31))
    return INFCL_ERR_UNSUPPORTED;
  if (s->n == 0) return INFCL_OK;
  if (!view_ok(x, s->head_dim) || !view_ok(out, s->head_dim) || !block_aligned(pos, 4) || !block_aligned(freqs, 4) ||
      x.data == out.data)
    return INFCL_ERR_INVALID;
  if (!view_supported(x) || !view_supported(out)) return INFCL_ERR_UNSUPPORTED;
  RotaryArgs a;
  a.x = x.data, a.out = out.data, a.xs = x.token_stride, a.xh = x.head_stride, a.os = out.token_stride;
  a.oh = out.head_stride, a.pos = pos, a.freqs = freqs, a.ps = s->pos_stride, a.n = s->n;
  a.heads = s->heads, a.turned = s->turned, a.hd = s->head_dim, a.pairs = (int)pairs;
  a.e1 = (int)ends[0], a.e2 = (int)ends[1], a.e3 = (int)ends[2];
  a.pos_f32 = s->pos_dtype, a.sign = s->back ? -1.f : 1.f;
  const bool whole = s->paired == INFCL_PAIRED_HALVES && pairs % 8 == 0;
  a.items = whole ? (int)(s->head_dim / 8 - pairs / 8) : s->head_dim / 8;
  a.by_items = by(a.items), a.by_heads = by(a.heads);
  // Some 4096 items of work for a workgroup, as long as there are several for every
  // compute unit; the table holds the angles of at least two tokens.
  const int64_t row = (int64_t)a.heads * a.items;
  int64_t tokens = 4096 / row;
  if (tokens > kTable / pairs) tokens = kTable / pairs;
  if (tokens > s->n / 1024) tokens = s->n / 1024;
  if (tokens < 1) tokens = 1;
  a.tokens = (int)tokens;
  const int64_t grid = (s->n + tokens - 1) / tokens;
  if (grid > (((int64_t)1 << 32) - 1) / 256) return INFCL_ERR_UNSUPPORTED;
  hipStream_t st = (hipStream_t)stream;
  if (s->dtype == INFCL_BF16)
    rotary_t<kBF16>(a, s->paired, whole, (unsigned)grid, st);
  else if (s->dtype == INFCL_F16)
    rotary_t<kF16>(a, s->paired, whole, (unsigned)grid, st);
  else
    rotary_t<kF32>(a, s->paired, whole, (unsigned)grid, st);
  return launch_status();
}

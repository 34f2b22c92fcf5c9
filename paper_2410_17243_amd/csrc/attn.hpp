// Shared parts of the packed-attention kernels (gfx950).
//
// Every kernel keeps 32 rows of one side per wave in registers as the column
// operand of the 32x32x16 MFMA and sweeps tiles of the other side through LDS.
// A product of swept rows (A) with own rows (B) leaves in lane L the own row
// L % 32 and, in register r of a 32-row block, the swept row
// 8 (r / 4) + 4 (L / 32) + r % 4: softmax statistics of own rows are sums over a
// lane's registers and one exchange with lane L ^ 32, and registers 8t .. 8t + 7,
// rounded to 16 bits, are the column operand of the next product over swept
// rows 16t .. 16t + 15 as they stand, if the transposing LDS reads of its row
// operand take those rows in the same order (lane half h, slot e:
// 16t + 8 (e / 4) + 4h + e % 4).
//
// Tiles in LDS: rows of DP features (64 or 128; heads of fewer features are
// filled up with zeros), 16-byte chunks at chunk ^ attn_sw(row), so that reads
// of one chunk of 16 rows, and the 4 rows x 4 chunks of a half-wave's
// transposing reads, each touch all 64 banks once.
#pragma once

#include "common.hpp"
#include "infcl_tower.h"

namespace infcl {

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

// What the kernels get of a call.  Strides in elements.
struct AttnArgs {
  const uint16_t *q, *k, *v;
  int64_t qs, qh, ks, kh, vs, vh;  // from token to token, from head to head
  const int32_t *cu_q, *cu_k, *len_k;  // (len_k: may be null)
  int64_t tq, tk;
  int32_t nseq, heads, kvh, group, hd, causal;
  float scale, sl2;  // of the scores; times log2(e)
};

// How a forward call is cut up, and its workspace.
struct AttnFwdPlan {
  int nw, tiles, parts;  // waves of a workgroup; row tiles of a sequence; parts of its keys
  size_t o, ml, total;
};

// ... and a backward call.
struct AttnBwdPlan {
  bool few;
  int parts, parts_q;  // of the sweeps over queries, over keys
  int64_t trow;        // pairs of a head in stat
  size_t stat, part, part_q, total;
};

// A launch has less than 2^32 work-items (past that its grid would wrap, without an
// error).  So many of `tiles` tiles for each of `others` workgroups at once: the
// kernels go on to the rest in steps of that number.
constexpr int64_t kAttnItems = ((int64_t)1 << 32) - 1;
inline int64_t attn_at_once(int64_t tiles, int64_t others, int threads) {
  const int64_t most = kAttnItems / threads / others;
  return tiles < most ? tiles : most < 1 ? 1 : most;
}
// Pairs of sequence (and the rows past the last one) and key head.
inline int64_t attn_groups(const AttnArgs& a) { return ((int64_t)a.nseq + 1) * a.kvh; }

// Tiles of nseq sequences, of which none has more than `most` and all together
// about `sum`.
inline int64_t attn_tiles(int64_t nseq, int64_t most, int64_t sum) {
  const int64_t a = nseq * most, b = sum + nseq;
  return a < b ? a : b;
}
// Parts into which each of `have` sweeps is cut so that there are `want` of them,
// at most `most` and 16.
inline int attn_parts(int64_t have, int64_t want, int64_t most) {
  int64_t p = have > 0 ? (want + have - 1) / have : 1;
  p = p < most ? p : most;
  p = p < 16 ? p : 16;
  return (int)(p < 1 ? 1 : p);
}

// Sequence z's queries [q0, q0 + m) and keys [k0, k0 + n), cut to the arrays
// whatever the offsets say.  z = nseq: the rows past the last sequence, as
// queries without keys (or keys without queries).
struct AttnSeq {
  int64_t q0, k0;
  int32_t m, n;
};
__device__ __forceinline__ AttnSeq attn_seq(const AttnArgs& a, int z) {
  AttnSeq s;
  const int64_t q0 = a.cu_q[z], k0 = a.cu_k[z];
  const int64_t q1 = z < a.nseq ? a.cu_q[z + 1] : a.tq, k1 = z < a.nseq ? a.cu_k[z + 1] : a.tk;
  s.q0 = q0 < 0 ? 0 : q0 > a.tq ? a.tq : q0;
  s.k0 = k0 < 0 ? 0 : k0 > a.tk ? a.tk : k0;
  const int64_t e = q1 > a.tq ? a.tq : q1, f = k1 > a.tk ? a.tk : k1;
  s.m = (int32_t)(e > s.q0 ? e - s.q0 : 0);
  s.n = (int32_t)(f > s.k0 ? f - s.k0 : 0);
  if (a.len_k && z < a.nseq) {
    const int32_t used = a.len_k[z] < 0 ? 0 : a.len_k[z];
    s.n = used < s.n ? used : s.n;
  }
  return s;
}

// Workgroup idx of a grid of `tiles` tiles for each of `groups` (sequence, key head)
// pairs: tile t, 0 the first to run, of pair g.  With many pairs a pair's tiles
// follow one another on one XCD, whose L2 then holds what they share; with few,
// all first tiles come first (the longest, where lengths differ by tile), spread
// over the XCDs, so that none of them is left waiting.  (Forward of 4112 pairs of
// 257 tokens: 225 us, 267 with first tiles first; step of 20 pairs of up to 4096
// tokens, dq 223 and 228, dk and dv 320 and 335 the other way round.)
constexpr uint32_t kAttnManyGroups = 64;
struct AttnPlace {
  uint32_t t, g;
};
__host__ __device__ __forceinline__ AttnPlace attn_place(uint32_t idx, uint32_t tiles, uint32_t groups) {
  if (groups < kAttnManyGroups) return AttnPlace{idx / groups, idx % groups};
  const uint32_t even = groups & ~7u;
  if (idx < even * tiles) return AttnPlace{(idx >> 3) % tiles, (idx >> 3) / tiles * 8 + (idx & 7)};
  return AttnPlace{(idx - even * tiles) % tiles, even + (idx - even * tiles) / tiles};
}

template <int DP>
__host__ __device__ __forceinline__ int attn_sw(int r) {
  return DP == 128 ? 4 * (r & 3) + ((r >> 2) & 3) : 4 * ((r >> 1) & 1) + ((r >> 2) & 3);
}

// Copies of a tile of KT rows to LDS by NW waves: instruction k = wave + NW kk
// fills 1024 bytes.  The chunk order depends on k only modulo kPeriod, so a
// lane keeps one source offset for each of kVar instructions.  Chunks past the
// head's features have an offset past every tile: zeros.
template <int DP, int NW, int KT>
struct AttnTile {
  static constexpr int kCh = DP / 8, kRows = 64 / kCh, kInstr = KT / kRows, kPer = kInstr / NW;
  static constexpr int kPeriod = DP == 128 ? 4 : 2, kVar = kPeriod / NW > 1 ? kPeriod / NW : 1;
  static constexpr int kBytes = KT * DP * 2, kRow = DP * 2;
  static_assert(kPer >= 1 && kInstr % NW == 0, "layout");

  static __host__ __device__ __forceinline__ void offsets(uint32_t (&off)[kVar], int wave, int lane, uint32_t stride, int hd) {
#pragma unroll
    for (int i = 0; i < kVar; ++i) {
      const int r = ((wave + NW * i) % kPeriod) * kRows + lane / kCh, c = (lane % kCh) ^ attn_sw<DP>(r);
      off[i] = 8 * c < hd ? (uint32_t)(lane / kCh) * stride + 16 * c : 0x80000000u;
    }
  }
  // rows: how many there are from base on (any number; at most KT are read).
  static __device__ __forceinline__ void issue(const uint16_t* base, int rows, uint32_t stride, int hd,
                                               INFCL_LDS char* lds, const uint32_t (&off)[kVar], int wave) {
    int n = rows > KT ? KT : rows;
    n = n < 0 ? 0 : n;
    const uint64_t at = (uint64_t)base;
    u32x4 rs;
    rs[0] = (uint32_t)at, rs[1] = (uint32_t)(at >> 32) & 0xFFFFu, rs[3] = 0x00020000u;
    rs[2] = n ? (uint32_t)(n - 1) * stride + 2 * hd : 0;
#pragma unroll
    for (int kk = 0; kk < kPer; ++kk) {
      const int k = wave + NW * kk;
      dma16_asm(rs, lds + 1024 * k, off[kk % kVar], (uint32_t)(k * kRows) * stride);
    }
  }
};

// Addresses in a tile: row fragments (swept rows as A operand: row L % 32, chunk
// 2i + h) and transposed ones (32-feature block fb, rows 16t + 8tt + 4h + e).
template <int DP>
struct AttnLanes {
  static constexpr int kI = DP / 16, kFb = DP / 32;
  int row[kI], tr[2][kFb];
  __host__ __device__ __forceinline__ void init(int lane) {
    const int r = lane & 31, h = lane >> 5;
#pragma unroll
    for (int i = 0; i < kI; ++i) row[i] = r * DP * 2 + 16 * ((2 * i + h) ^ attn_sw<DP>(r));
    const int l16 = lane & 15, e = l16 >> 2, qq = l16 & 3, nb = (lane >> 4) & 1;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const int tr_row = 8 * tt + 4 * h + e;
#pragma unroll
      for (int fb = 0; fb < kFb; ++fb)
        tr[tt][fb] =
            tr_row * DP * 2 + 16 * ((4 * fb + 2 * nb + (qq >> 1)) ^ attn_sw<DP>(tr_row)) + 8 * (qq & 1);
    }
  }
};

__device__ __forceinline__ bf16x8 attn_row(const INFCL_LDS char* p) { return *(const INFCL_LDS bf16x8*)p; }
__device__ __forceinline__ bf16x8 attn_tr(const INFCL_LDS char* p0, const INFCL_LDS char* p1) {
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((INFCL_LDS s16x4*)p0);
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((INFCL_LDS s16x4*)p1);
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Registers 8t .. 8t + 7 of a 32-row block as the column operand of step t.
template <bool F16>
__device__ __forceinline__ bf16x8 attn_pack(const f32x16& x, int t) {
  bf16x8 r;
  if constexpr (F16) {
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = to16<true>(x[8 * t + e]);
  } else {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = pk_bf16(x[8 * t + 2 * e], x[8 * t + 2 * e + 1]);
    r = __builtin_bit_cast(bf16x8, w);
  }
  return r;
}

// x, as a value the compiler knows nothing of (a comparison with it is one
// instruction, not one for each of the conditions it came from).
__device__ __forceinline__ int attn_opaque(int x) {
  asm("" : "+v"(x));
  return x;
}

// Waits for fragments loaded from memory: here, once, and not at their first use
// in a sweep, where the wait would be for the copies under way as well, every time
// around.
template <int N>
__device__ __forceinline__ void attn_settle(bf16x8 (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(x[i]));
}

// x of this lane and of lane ^ 32.
__device__ __forceinline__ void attn_both(float x, float& a, float& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  a = __uint_as_float(r[0]);
  b = __uint_as_float(r[1]);
}
__device__ __forceinline__ float attn_max2(float x) {
  float a, b;
  attn_both(x, a, b);
  return fmaxf(a, b);
}
__device__ __forceinline__ float attn_sum2(float x) {
  float a, b;
  attn_both(x, a, b);
  return a + b;
}

__device__ __forceinline__ f32x16 f32x16_zero() {
  f32x16 z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.f;
  return z;
}

// Swept row of register r in lane half h, within its 32-row block.
__host__ __device__ __forceinline__ int attn_reg_row(int r, int h) { return 8 * (r >> 2) + 4 * h + (r & 3); }

// One own row's 16-byte chunk 2i + h (of hd / 8), or zeros.
__device__ __forceinline__ bf16x8 attn_own(const uint16_t* row, int i, int h, int hd, bool live) {
  u32x4 c = {0, 0, 0, 0};
  if (live && 8 * (2 * i + h) < hd) c = *(const u32x4*)(row + 8 * (2 * i + h));
  return __builtin_bit_cast(bf16x8, c);
}

// Stores a transposed accumulator (own row in the lane, features in the
// registers) times f as 16-bit elements.
template <bool F16, int FB>
__device__ __forceinline__ void attn_store(uint16_t* row, const f32x16 (&acc)[FB], float f, int h, int hd) {
#pragma unroll
  for (int fb = 0; fb < FB; ++fb)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int d = 32 * fb + 8 * j + 4 * h;
      if (d >= hd) continue;
      u32x2 w;
      if constexpr (F16) {
        typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
        f16x4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (_Float16)(acc[fb][4 * j + e] * f);
        w = __builtin_bit_cast(u32x2, x);
      } else {
        w[0] = pk_bf16(acc[fb][4 * j] * f, acc[fb][4 * j + 1] * f);
        w[1] = pk_bf16(acc[fb][4 * j + 2] * f, acc[fb][4 * j + 3] * f);
      }
      *(u32x2*)(row + d) = w;
    }
}

// ---- Masked rows that hold infinities or NaN.  A masked weight is zero, but zero
// times such an entry is NaN, and a product's swept rows are common to own rows
// that see them and own rows that do not.  Only the tiles that a causal mask cuts
// have rows of both kinds (past a sequence's end the copies leave zeros), and they
// are a sweep's last ones.  A wave whose sums are not finite looks at the rows of
// these tiles; where those are all finite its results stand.  Else its workgroup
// sweeps again without them (CUT), and then takes them one by one on the vector
// unit, in fp32, from memory, each for the own rows that see it: two tiles' rows
// and a wave's 32 at most (times the heads of a group for keys), whatever the
// length and whoever sees them.

// Whether an accumulator holds a NaN (x 0 is NaN for infinities too).
template <int FB>
__device__ __forceinline__ bool attn_bad(const f32x16 (&acc)[FB]) {
  float t = 0.f;
#pragma unroll
  for (int fb = 0; fb < FB; ++fb)
#pragma unroll
    for (int r = 0; r < 16; ++r) t = fmaf(acc[fb][r], 0.f, t);
  return !(t == 0.f);
}
// Whether rows [0, n) of x hold an entry that is not finite (the wave together).
// Adding the exponent's last bit to |x| carries into the sign's place from the
// exponent of all ones on.
template <bool F16>
__device__ __forceinline__ bool attn_odd(const uint16_t* x, int n, int64_t stride, int hd, int lane) {
  uint32_t odd = 0;
#pragma unroll 1
  for (int r = lane >> 4; r < n; r += 4)
    if (8 * (lane & 15) < hd) {
      const u32x4 w = *(const u32x4*)(x + r * stride + 8 * (lane & 15));
#pragma unroll
      for (int i = 0; i < 4; ++i) odd |= (w[i] & 0x7FFF7FFFu) + (F16 ? 0x04000400u : 0x00800080u);
    }
  return wave_any((odd & 0x80008000u) != 0);
}
// ... the keys x of sequence sq's key head in the tiles that the mask of a wave's
// rows [rw, rw + 32) of (query, head of the group) cuts.
template <bool F16>
__device__ __forceinline__ bool attn_odd_keys(const uint16_t* x, int64_t stride, int hd, const AttnSeq& sq, int group,
                                              uint32_t rw, uint32_t rows, int tile) {
  const uint32_t rv = rw + 31 < rows ? rw + 31 : rows - 1;
  int lo = (int)(rw / (uint32_t)group) + sq.n - sq.m + 1, hi = (int)(rv / (uint32_t)group) + sq.n - sq.m + 1 + tile;
  lo = lo < 0 ? 0 : lo, hi = hi < sq.n ? hi : sq.n;
  return attn_odd<F16>(x + lo * stride, hi - lo, stride, hd, (int)threadIdx.x & 63);
}
// Whether one of the workgroup's waves says so; `flags`: NW words that were not read
// since the last barrier.
template <int NW>
__device__ __forceinline__ bool attn_vote(bool x, INFCL_LDS int* flags, int wave) {
  if constexpr (NW == 1) return x;
  flags[wave] = x;
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  int any = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) any |= flags[i];
  return __builtin_amdgcn_readfirstlane(any) != 0;
}

// Lanes L and L ^ 32 share an own row and take every other 8 features of it.

// <x, y>, over both lanes' features.
template <bool F16>
__device__ __forceinline__ float attn_dot(const uint16_t* x, const uint16_t* y, int h, int hd) {
  float s = 0.f;
#pragma unroll 1
  for (int d = 8 * h; d < hd; d += 16) {
    const bf16x8 a = *(const bf16x8*)(x + d), b = *(const bf16x8*)(y + d);
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(from16<F16>(a[e]), from16<F16>(b[e]), s);
  }
  return attn_sum2(s);
}
// acc += w x, acc as the products leave it.
template <bool F16, int FB>
__device__ __forceinline__ void attn_axpy(f32x16 (&acc)[FB], float w, const uint16_t* x, int h, int hd) {
#pragma unroll
  for (int fb = 0; fb < FB; ++fb)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int d = 32 * fb + 8 * j + 4 * h;
      if (d >= hd) continue;
      const u32x2 a = *(const u32x2*)(x + d);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint16_t b = (uint16_t)(a[e >> 1] >> (16 * (e & 1)));
        acc[fb][4 * j + e] = fmaf(w, from16<F16>(__builtin_bit_cast(__bf16, b)), acc[fb][4 * j + e]);
      }
    }
}
// 8 sums times f as 16-bit elements.
template <bool F16>
__device__ __forceinline__ void attn_store8(uint16_t* x, const float (&acc)[8], float f) {
  bf16x8 a;
#pragma unroll
  for (int e = 0; e < 8; ++e) a[e] = to16<F16>(acc[e] * f);
  *(bf16x8*)x = a;
}

// Barrier of the workgroup after all of this wave's copies and LDS reads.
__device__ __forceinline__ void attn_barrier() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// A kernel's arguments (all of them, as a struct) read again: code after a sweep
// that is seldom run then does not hold them in registers through the sweep.
template <typename Args>
__device__ __forceinline__ Args attn_reload() {
  typedef const __attribute__((address_space(4))) char Kernarg;
  Kernarg* p = (Kernarg*)__builtin_amdgcn_kernarg_segment_ptr();
  asm("" : "+s"(p));
  return *(const Args*)p;
}

}  // namespace infcl

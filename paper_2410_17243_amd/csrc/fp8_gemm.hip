// Products of operands in 8-bit floats: out [n, m] = a b^T + bias, a [n, k] and b [m, k]
// with a power of two for each 128 entries of a row.
//
// The scaled 32 x 32 x 64 MFMA takes the powers of two as bytes, one for each row of
// its operands, so the products run at the matrix unit's 8-bit rate (twice that of 16
// bits) and accumulate in fp32 without a multiplication by scales.  The unit adds its
// products in groups of eight with 13 bits below the largest of a group, and the groups
// in fp32; on entries of one scale that is 2^-17 of the result in the root mean square, a
// small part of what 16-bit outputs round off.
//
// b's rows are the MFMA's rows and a's its columns, so that a lane holds four entries in
// a row of the output next to each other.  Tiles of 64 bytes of the contraction go to LDS
// by asynchronous copies, four stages in flight: a stage is waited for by the number of
// copies issued after it, with one barrier a stage.  A row's four chunks of 16 bytes are
// XORed with bits 2 and 3 of the row, which spreads both the copies and the row reads
// over all banks.  The exponent bytes of 4096 entries of the contraction are kept in LDS
// as words of four blocks and shifted along.
//
// The contraction is cut into parts where the output's tiles alone would leave compute
// units idle; their sums are added in order by a second launch, with the bias.
//
// 8192^3 takes 427 to 505 us with the clock of the card at hand (2575 to 2180 TFLOP/s): a stage's
// LDS traffic, 96 KiB read and 32 written, is about as long as its products.  65536 x 1024 x 4096
// takes 235 to 260, 4096 x 1024 x 65536 241 to 260 in four parts and their join.  Short contractions
// are further from the unit's rate (65536 x 4096 x 1024 300 to 372 us of 197, 17408 x 2048 x 512 34 of
// 13); a workgroup's start and end are some 8 us, but that is not all of it: two workgroups of 256 x
// 128 to a compute unit, one's end beside the other's products, do not gain (8192^3 536 us for 427,
// 65536 x 4096 x 1024 304 for 300), nor does a stream of stages over several tiles.
#include "fp8.hpp"
#include "grid.hpp"

namespace infcl {
infcl_status fp8_pack_two(const void* x, int64_t x_stride, int64_t n, const void* w, int64_t w_stride, int64_t m, int64_t k,
                          int dtype, void* xq, void* xe, void* xqt, void* xet, void* wq, void* we, void* wqt, void* wet,
                          hipStream_t st);
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4v __attribute__((ext_vector_type(4)));

constexpr int kStep = 64;    // entries of a stage
constexpr int kStages = 4;
constexpr int kGroups = 8;   // words of exponents in LDS: 512 entries each

// Waves WM x WN of FM x FN blocks of 32 x 32: BM rows of b, BN rows of a.
template <int WM_, int WN_, int FM_, int FN_>
struct Tile {
  static constexpr int WM = WM_, WN = WN_, FM = FM_, FN = FN_;
  static constexpr int BM = 32 * WM * FM, BN = 32 * WN * FN, kRows = BM + BN;
  static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
  static constexpr int kCopies = kRows / 16 / kWaves;  // 16 rows of 64 bytes each
  static constexpr int kStage = kRows * kStep;
  static_assert(kRows % (16 * kWaves) == 0 && BM % (16 * kCopies) == 0, "layout");
};

struct MatmulArgs {
  const uint8_t *a, *ae, *b, *be;
  const void* bias;
  void* out;
  float* part;
  int64_t n, m, kp, ep, nm;  // nm: elements of one part
  int tm, tn, tiles, stages, steps;  // tiles along m and n; stages in all, of a part
};

// OUT: sums of a part, the output, or the output past the caches.
enum Out { kParts, kOutput, kPastCaches };
template <class W, bool F16, Out OUT>
__global__ void __launch_bounds__(W::kThreads, 2) matmul_kernel(const MatmulArgs p) {
  constexpr bool PARTS = OUT == kParts;
  __shared__ __attribute__((aligned(1024))) char lds[kStages * W::kStage];
  __shared__ uint32_t exps[kGroups * W::kRows];
  const uint32_t slot = xcd_slot(blockIdx.x, gridDim.x);
  const int part = (int)(slot / (uint32_t)p.tiles), tile = (int)(slot % (uint32_t)p.tiles);
  // eight tiles along m for each along n, so that the workgroups of an XCD share rows of both
  const int band = tile / (8 * p.tn), in = tile - band * 8 * p.tn, wide = p.tm - 8 * band < 8 ? p.tm - 8 * band : 8;
  const int64_t m0 = (int64_t)(8 * band + in % wide) * W::BM, n0 = (int64_t)(in / wide) * W::BN;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int s0 = part * p.steps, ns = p.stages - s0 < p.steps ? p.stages - s0 : p.steps;
  const int rows_b = (int)(p.m - m0 < W::BM ? p.m - m0 : W::BM), rows_a = (int)(p.n - n0 < W::BN ? p.n - n0 : W::BN);

  // A wave's copies are of one operand: 16 rows each, from row `first` of its tile on.
  const uint32_t kp = (uint32_t)p.kp;
  const bool of_b = 16 * W::kCopies * wave < W::BM;
  const int first = 16 * W::kCopies * wave - (of_b ? 0 : W::BM);
  const uint32_t voff = (uint32_t)(first + (lane >> 2)) * kp + 16 * ((lane & 3) ^ ((lane >> 4) & 3));
  const uint64_t base = (uint64_t)(of_b ? p.b + m0 * p.kp : p.a + n0 * p.kp) + (uint64_t)s0 * kStep;
  const uint32_t limit = (uint32_t)((of_b ? rows_b : rows_a) - 1) * kp + kStep;
  auto source = [&](int s) {  // stage s of this part; past its end: zeros
    const uint64_t at = base + (uint64_t)s * kStep;
    u32x4 r;
    r[0] = (uint32_t)at, r[1] = (uint32_t)(at >> 32) & 0xFFFFu, r[2] = s < ns ? limit : 0, r[3] = 0x00020000u;
    return r;
  };
  auto copy = [&](const u32x4& r, int s, int i) {  // the i-th of a wave's copies
    dma16_asm(r, (INFCL_LDS char*)lds + (s % kStages) * W::kStage + 1024 * (W::kCopies * wave + i), voff, (uint32_t)(16 * i) * kp);
  };
  auto exponents = [&](int s) {  // of 64 stages from s (a multiple of 64) on: a row for each thread, all loads at once
    static_assert(W::kRows == W::kThreads, "a row for each thread");
    const int r = threadIdx.x;
    const bool isb = r < W::BM;
    const int row = isb ? r : r - W::BM, rows = isb ? rows_b : rows_a;
    const int64_t word0 = (int64_t)(s0 + s) / 8, words = p.ep / 4;
    const uint32_t* e = (const uint32_t*)(isb ? p.be : p.ae) + ((isb ? m0 : n0) + (row < rows ? row : rows - 1)) * words;
    uint32_t w[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) w[g] = e[word0 + g < words ? word0 + g : words - 1];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) exps[g * W::kRows + r] = w[g];
  };

  const int wm = wave / W::WN, wn = wave % W::WN, h = lane >> 5;
  f32x16 acc[W::FM][W::FN];
#pragma unroll
  for (int i = 0; i < W::FM; ++i)
#pragma unroll
    for (int j = 0; j < W::FN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  const int row = lane & 31, swz = (row >> 2) & 3;
  const int off0 = row * kStep + 16 * ((2 * h) ^ swz), off1 = row * kStep + 16 * ((2 * h + 1) ^ swz);
  const int bm = wm * W::FM * 32, bn = W::BM + wn * W::FN * 32;  // first rows of this wave's blocks
  i32x8 b[W::FM], a0[W::FN], a1[W::FN];
  auto frag = [&](int s, int first) {
    const INFCL_LDS char* cur = (const INFCL_LDS char*)lds + (s % kStages) * W::kStage + first * kStep;
    const i32x4 lo = *(const INFCL_LDS i32x4*)(cur + off0), hi = *(const INFCL_LDS i32x4*)(cur + off1);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  uint32_t eb[W::FM], ea[W::FN];
  auto words = [&](int s) {  // the exponents of eight stages from s on
    const uint32_t* e = exps + (s / 8 % kGroups) * W::kRows + row;
#pragma unroll
    for (int i = 0; i < W::FM; ++i) eb[i] = e[bm + 32 * i];
#pragma unroll
    for (int j = 0; j < W::FN; ++j) ea[j] = e[bn + 32 * j];
  };
  static_assert(W::kCopies == 4, "waits");
  // One stage: its fragments are in registers, those of the next one are read beside its
  // products, b's into the registers that a product has just read.  At the barrier this
  // wave's copies of stage s + 1 are done (those of two later ones may not be) and with it
  // every wave's; all reads of stage s are done too, so its place takes stage s + 4, whose
  // copies go out between the products (right after the barrier they cost 2 to 4 percent).
  auto step = [&](int s, const i32x8 (&a)[W::FN], i32x8 (&next)[W::FN]) {
    asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const u32x4 later = source(s + kStages);
#pragma unroll
    for (int j = 0; j < W::FN; ++j) next[j] = frag(s + 1, bn + 32 * j);
#pragma unroll
    for (int i = 0; i < W::FM; ++i) {
#pragma unroll
      for (int j = 0; j < W::FN; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b[i], a[j], acc[i][j], 0, 0, 0, (int)eb[i], 0, (int)ea[j]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int c = i * W::kCopies / W::FM; c < (i + 1) * W::kCopies / W::FM; ++c) copy(later, s + kStages, c);
      b[i] = frag(s + 1, bm + 32 * i);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
#pragma unroll
  for (int s = 0; s < kStages; ++s) {
    const u32x4 r = source(s);
#pragma unroll
    for (int i = 0; i < W::kCopies; ++i) copy(r, s, i);
  }
  if (ns > 0) exponents(0);  // (no blocks, no words)
  asm volatile("s_waitcnt vmcnt(12) lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
  for (int j = 0; j < W::FN; ++j) a0[j] = frag(0, bn + 32 * j);
#pragma unroll
  for (int i = 0; i < W::FM; ++i) b[i] = frag(0, bm + 32 * i);
  for (int s = 0; s < ns;) {  // (128 entries at least: an even number of stages)
    if (s > 0 && s % 64 == 0) {
      __syncthreads();
      exponents(s);
      __syncthreads();
    }
    words(s);
    const int end = s + 8 < ns ? s + 8 : ns;
#pragma unroll 1
    for (; s < end; s += 2) {
      step(s, a0, a1);
      step(s + 1, a1, a0);
#pragma unroll
      for (int i = 0; i < W::FM; ++i) eb[i] >>= 8;  // the next block's bytes
#pragma unroll
      for (int j = 0; j < W::FN; ++j) ea[j] >>= 8;
    }
  }
  // Copies past the last stage wrote zeros into stages no one reads; they must have
  // landed before the workgroup's LDS is given away.
  wait_dma();

  // Rows of a lane's own entries would be 8 bytes of 32 rows in one store.  Where rows are
  // 16-byte aligned, a wave's block goes through its share of the LDS instead and comes out
  // in whole rows of it: PARTS 32 rows of a at a time, in fp32, else all in 16 bits.
  constexpr int kSize = PARTS ? 4 : 2, kAcross = W::FM * 32 * kSize / 16;  // chunks of a row
  if (p.m % (16 / kSize) == 0) {
    constexpr int kJ = PARTS ? 1 : W::FN, kRowsOut = 32 * kJ;
    static_assert(kRowsOut * kAcross * 16 * W::kWaves <= kStages * W::kStage, "LDS of the output");
    INFCL_LDS char* mine = (INFCL_LDS char*)lds + wave * (kRowsOut * kAcross * 16);
    const int64_t c0 = m0 + bm, r0 = n0 + 32 * wn * W::FN;
    __syncthreads();  // every wave's reads of the last stage are done
#pragma unroll
    for (int j0 = 0; j0 < W::FN; j0 += kJ) {
#pragma unroll
      for (int i = 0; i < W::FM; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int at = 32 * i + 8 * g + 4 * h;  // of this wave's entries along m
          float bias[4] = {0.f, 0.f, 0.f, 0.f};
          if (!PARTS && p.bias && c0 + at < p.m) {
            typedef __attribute__((__vector_size__(8), __aligned__(2))) __bf16 quad;
            const quad y = *(const quad*)((const __bf16*)p.bias + c0 + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) bias[e] = from16<F16>(y[e]);
          }
#pragma unroll
          for (int jj = 0; jj < kJ; ++jj) {
            const int j = j0 + jj, r = 32 * jj + (lane & 31), c = at * kSize / 16;
            INFCL_LDS char* to = mine + (r * kAcross + (c ^ (r & (kAcross - 1)))) * 16 + (at * kSize & 15);
            f32x4v v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              v[e] = acc[i][j][4 * g + e] + bias[e];
            }
            if constexpr (PARTS) {
              *(INFCL_LDS f32x4v*)to = v;
            } else {
              __bf16 y[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) y[e] = to16<F16>(v[e]);
              *(INFCL_LDS uint64_t*)to = __builtin_bit_cast(uint64_t, y);
            }
          }
        }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 4
      for (int t = 0; t < kRowsOut * kAcross / 64; ++t) {
        const int r = t * (64 / kAcross) + lane / kAcross, c = lane % kAcross;
        const i32x4 v = *(const INFCL_LDS i32x4*)(mine + (r * kAcross + (c ^ (r & (kAcross - 1)))) * 16);
        const int64_t row = r0 + 32 * j0 + r, col = c0 + c * (16 / kSize);
        if (row >= p.n || col >= p.m) continue;
        i32x4* out = (i32x4*)((char*)(PARTS ? (void*)(p.part + part * p.nm) : p.out) + (row * p.m + col) * kSize);
        if constexpr (OUT == kPastCaches)
          __builtin_nontemporal_store(v, out);
        else
          *out = v;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < W::FN; ++j) {
    const int64_t col = n0 + 32 * (wn * W::FN + j) + (lane & 31);
    if (col >= p.n) continue;
#pragma unroll
    for (int i = 0; i < W::FM; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int64_t at = m0 + bm + 32 * i + 8 * (r >> 2) + 4 * h + (r & 3);
        if (at >= p.m) continue;
        if constexpr (PARTS)
          p.part[part * p.nm + col * p.m + at] = acc[i][j][r];
        else
          ((__bf16*)p.out)[col * p.m + at] = to16<F16>(acc[i][j][r] + (p.bias ? from16<F16>(((const __bf16*)p.bias)[at]) : 0.f));
      }
  }
}

// The parts' sums in order, and the bias: four entries a lane.
template <bool F16>
__global__ void __launch_bounds__(256) matmul_join(const float* __restrict__ part, int parts, int64_t nm, int64_t total,
                                                   int64_t m, const __bf16* __restrict__ bias, __bf16* __restrict__ out) {
  const int64_t i = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x);
  if (i >= total) return;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0; p0 < parts; p0 += 8) {  // eight parts' loads at a time
    f32x4 x[8];
#pragma unroll
    for (int p = 0; p < 8; ++p) x[p] = *(const f32x4*)(part + (int64_t)(p0 + p < parts ? p0 + p : p0) * nm + i);
#pragma unroll
    for (int p = 0; p < 8; ++p)
      if (p0 + p < parts) s += x[p];
  }
  int64_t c = bias ? i % m : 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (i + e >= total) break;
    if (c >= m) c -= m;
    out[i + e] = to16<F16>(s[e] + (bias ? from16<F16>(bias[c]) : 0.f));
    ++c;
  }
}

// Up to 16 rows of x: a workgroup takes 16 rows of the weights, its waves every eighth
// block of the contraction, straight from memory; the waves' sums meet in LDS.  Every
// workgroup packs x itself (as infcl_fp8_pack does), 4096 entries of the contraction at a
// time, into LDS while the weights for them are on their way.  Bound by the weights' bytes
// and the latency of one such pass: 4 x 4096 -> 4096 7.1 us, 16 rows 10.7.  (Where each wave packs what
// it needs in its operand's layout, 16 rows whatever n, 9.3 and 9.4: better near 16 rows only, and
// not kept as a second form.)
constexpr int kFewWaves = 8, kFewBlocks = 4, kFewSpan = 128 * kFewWaves * kFewBlocks, kFewPitch = kFewSpan + 16;
template <bool F16>
__global__ void __launch_bounds__(64 * kFewWaves) few_kernel(const uint16_t* __restrict__ x, int64_t xs, int n, int64_t k,
                                                             const uint8_t* __restrict__ w, const uint8_t* __restrict__ we,
                                                             int64_t m, int64_t kp, int64_t ep,
                                                             const __bf16* __restrict__ bias, __bf16* __restrict__ out) {
  __shared__ f32x4v sums[kFewWaves][64];
  __shared__ __attribute__((aligned(16))) uint8_t xq[16 * kFewPitch];
  __shared__ uint8_t xe[16][kFewSpan / 128];
  constexpr int T = F16 ? kF16 : kBF16;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
  const int64_t m0 = (int64_t)blockIdx.x * 16, wrow = m0 + r < m ? m0 + r : m - 1;
  const uint8_t *wp = w + wrow * kp + 32 * q, *wep = we + wrow * ep;
  f32x4v acc = {0.f, 0.f, 0.f, 0.f};
  const int blocks = (int)((k + 127) / 128);
  for (int c0 = 0; c0 < blocks; c0 += kFewSpan / 128) {
    i32x4 lo[kFewBlocks], hi[kFewBlocks];
    uint32_t byte[kFewBlocks];
#pragma unroll
    for (int i = 0; i < kFewBlocks; ++i) {  // (past the last block: that one again)
      const int b = c0 + wave + kFewWaves * i, at = b < blocks ? b : blocks - 1;
      lo[i] = *(const i32x4*)(wp + 128 * (int64_t)at), hi[i] = *(const i32x4*)(wp + 128 * (int64_t)at + 16);
      byte[i] = wep[at];
    }
    if (c0 > 0) __syncthreads();  // (the packed entries of before have been read)
    const int here = blocks - c0 < kFewSpan / 128 ? blocks - c0 : kFewSpan / 128;
    // 16 lanes take a block of every row, eight rows at a time
    static_assert(4 * kFewWaves == kFewSpan / 128, "a block for each 16 lanes");
    const int b = threadIdx.x >> 4;
    const int64_t at = 128 * (int64_t)(c0 + b) + 8 * r;
    for (int j0 = 0; j0 < n && b < here; j0 += 8) {
      Raw8<T> raw[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j0 + j < n) raw[j].load(x, (j0 + j) * xs + (at < k ? at : 0));
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (j0 + j >= n) break;
        float v[8];
        raw[j].get(at < k, v);
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = umax(top, top_bits(v[e]));
        const uint32_t xb = fp8_exponent(row16_max(top));
        const float inv = fp8_inverse(xb);
        uint2 y = make_uint2(fp8_pack4(v[0], v[1], v[2], v[3], inv), fp8_pack4(v[4], v[5], v[6], v[7], inv));
        if (xb == 255) y = make_uint2(kFp8Nan, kFp8Nan);
        *(uint2*)(xq + (j0 + j) * kFewPitch + 128 * b + 8 * r) = y;
        if (r == 0) xe[j0 + j][b] = (uint8_t)xb;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kFewBlocks; ++i) {
      const int b = wave + kFewWaves * i;
      if (b >= here) break;
      // (columns of rows that are not there come to nothing, whatever their operand holds)
      const i32x4 a0 = *(const i32x4*)(xq + r * kFewPitch + 128 * b + 32 * q), a1 = *(const i32x4*)(xq + r * kFewPitch + 128 * b + 32 * q + 16);
      acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
          __builtin_shufflevector(lo[i], hi[i], 0, 1, 2, 3, 4, 5, 6, 7), __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7), acc, 0,
          0, 0, (int)byte[i], 0, (int)xe[r][b]);
    }
  }
  sums[wave][lane] = acc;
  __syncthreads();
  if (wave != 0 || r >= n) return;
#pragma unroll
  for (int i = 1; i < kFewWaves; ++i) acc += sums[i][lane];
  const int64_t row = m0 + 4 * q;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (row + e < m) out[r * m + row + e] = to16<F16>(acc[e] + (bias ? from16<F16>(bias[row + e]) : 0.f));
}

typedef Tile<2, 4, 4, 2> Big;    // 256 x 256, 8 waves of 128 x 64
typedef Tile<2, 2, 2, 2> Small;  // 128 x 128, 4 waves of 64 x 64

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

struct MatmulPlan {
  bool big;
  int64_t tm, tn;
  int parts, stages, steps;
  size_t total;
};
// What a form of the product takes, in us, from the times of some thirty shapes: a round of
// workgroups is as long as its stages (of the small tiles 0.3 us with one to a compute
// unit, 0.6 with two; of the large ones 0.65 to 0.87 with what the chip's clock then is)
// and a start and an end; parts cost a launch and the traffic of their sums.  Measured, chosen and
// left: 4096 x 1024 x 1024 9.8 in small tiles, 16.5 in large ones, 28.5 in two parts; 776 x 1000 x
// 10007 22 in four parts of small tiles, 50 in one, 32 in large ones; 8192^3 454 in large
// tiles, 4096 x 4096 x 2048 37 and 51; 512 x 512 x 65536 31 in 16 parts, 39 in 32, 244 in one.
double estimate(bool big, int64_t tiles, int64_t parts, int64_t steps, int64_t nm) {
  const int64_t slots = big ? 256 : 512, wgs = tiles * parts, rest = wgs % slots;
  const double start = big ? 8. : 4., full = steps * (big ? 0.87 : 0.6) + start;
  double t = (double)(wgs / slots) * full;
  if (rest > slots / 2)
    t += full;
  else if (rest > 0)
    t += steps * (big ? 0.65 : 0.3) + start;
  return parts > 1 ? t + 6. + (double)parts * (double)nm * 8. / 3.5e6 : t;
}
MatmulPlan plan_of(int64_t n, int64_t m, int64_t k) {
  MatmulPlan p = {};
  p.stages = (int)(fp8_blocks(k) * (kFp8Block / kStep));
  const int64_t groups = (p.stages + 7) / 8;  // parts begin with a word of exponents
  double best = 0.;
  for (int big = 0; big < 2; ++big) {
    const int64_t b = big ? 256 : 128, tm = (m + b - 1) / b, tn = (n + b - 1) / b, tiles = tm * tn;
    for (int64_t asked : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
      if (asked > 1 && (asked > groups || tiles * asked > 2048)) break;
      const int64_t steps = groups < 1 ? 8 : (groups + asked - 1) / asked * 8;
      const int64_t parts = p.stages < 1 ? 1 : (p.stages + steps - 1) / steps;
      const double t = estimate(big, tiles, parts, steps < p.stages ? steps : p.stages, n * m);
      if (p.parts > 0 && t >= best) continue;
      best = t;
      p.big = big, p.tm = tm, p.tn = tn, p.parts = (int)parts, p.steps = (int)steps;
    }
  }
  p.total = p.parts > 1 ? up256((size_t)p.parts * ((size_t)(n * m + 3) & ~(size_t)3) * 4) : 0;
  return p;
}

// An output larger than the L2s would push the operands out of them (65536 x 4096 x 1024: 370 us
// past them, 415 through); a smaller one is left for who reads it next (10007 x 1000 x 776: 20 us,
// 21 past them).
constexpr int64_t kCaches = (int64_t)32 << 20;

template <class W, bool F16>
void launch_tiles(const MatmulPlan& p, const MatmulArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)(p.tm * p.tn * p.parts));
  if (p.parts > 1)
    hipLaunchKernelGGL((matmul_kernel<W, F16, kParts>), grid, dim3(W::kThreads), 0, st, a);
  else if (a.n * a.m * 2 > kCaches)
    hipLaunchKernelGGL((matmul_kernel<W, F16, kPastCaches>), grid, dim3(W::kThreads), 0, st, a);
  else
    hipLaunchKernelGGL((matmul_kernel<W, F16, kOutput>), grid, dim3(W::kThreads), 0, st, a);
}

template <bool F16>
infcl_status matmul_t(const uint8_t* aq, const uint8_t* ae, int64_t n, const uint8_t* bq, const uint8_t* be, int64_t m,
                      int64_t k, const void* bias, void* out, char* ws, hipStream_t st) {
  const MatmulPlan p = plan_of(n, m, k);
  MatmulArgs a;
  a.a = aq, a.ae = ae, a.b = bq, a.be = be, a.bias = bias, a.out = out, a.part = (float*)ws, a.n = n, a.m = m;
  a.kp = fp8_pitch(k), a.ep = fp8_ep(k), a.nm = (n * m + 3) & ~(int64_t)3;
  a.tm = (int)p.tm, a.tn = (int)p.tn, a.tiles = (int)(p.tm * p.tn), a.stages = p.stages, a.steps = p.steps;
  if (p.big)
    launch_tiles<Big, F16>(p, a, st);
  else
    launch_tiles<Small, F16>(p, a, st);
  if (p.parts > 1) {
    if (hipGetLastError() != hipSuccess) return INFCL_ERR_HIP;
    const int64_t total = n * m;
    hipLaunchKernelGGL((matmul_join<F16>), dim3((unsigned)((total + 1023) / 1024)), dim3(256), 0, st, (const float*)ws, p.parts,
                       a.nm, total, m, (const __bf16*)bias, (__bf16*)out);
  }
  return launch_status();
}

infcl_status sizes_status(int64_t n, int64_t m, int64_t k) {
  if (n < 0 || m < 1 || k < 0) return INFCL_ERR_INVALID;
  const int64_t most = (int64_t)1 << 27;
  if (n > most || m > ((int64_t)1 << 24) || k > ((int64_t)1 << 23) || (n > 0 && m > ((int64_t)1 << 38) / n) ||
      ((n + 127) / 128) * ((m + 127) / 128) > ((int64_t)1 << 22))
    return INFCL_ERR_UNSUPPORTED;
  return INFCL_OK;
}
bool few(int64_t n) { return n <= 16; }

// Packed operands one after the other in a block of memory: rows x k, values and exponents.
struct Places {
  char* at;
  size_t used = 0;
  explicit Places(void* p) : at((char*)p) {}
  void* take(size_t bytes) {
    void* p = at + used;
    used += up256(bytes);
    return p;
  }
  void operand(int64_t rows, int64_t k, void*& q, void*& e) {
    q = take((size_t)rows * (size_t)fp8_pitch(k));
    e = take((size_t)rows * (size_t)fp8_ep(k));
  }
};
struct LayerPlaces {
  void *xt = nullptr, *xte = nullptr, *wt = nullptr, *wte = nullptr;  // kept
  void *x, *xe, *w, *we, *fwd;                                        // the forward's
  void *dy = nullptr, *dye = nullptr, *dyt = nullptr, *dyte = nullptr, *sums, *bwd;  // the backward's
  size_t kept, fwd_bytes, bwd_bytes;
};
LayerPlaces layer_places(int64_t n, int64_t k, int64_t m, int keeps, void* kept, void* ws) {
  LayerPlaces r;
  Places p(kept), f(ws), b(ws);
  if (keeps & INFCL_KEEP_X) p.operand(k, n, r.xt, r.xte);
  if (keeps & INFCL_KEEP_W) p.operand(k, m, r.wt, r.wte);
  f.operand(n, k, r.x, r.xe);
  f.operand(m, k, r.w, r.we);
  r.fwd = f.take(plan_of(n, m, k).total);
  if (keeps & INFCL_KEEP_W) b.operand(n, m, r.dy, r.dye);
  if (keeps & INFCL_KEEP_X) b.operand(m, n, r.dyt, r.dyte);
  size_t sums = 0;
  infcl_fp8_pack_workspace(n, m, &sums);
  r.sums = b.take(sums);
  const size_t dx = keeps & INFCL_KEEP_W ? plan_of(n, k, m).total : 0, dw = keeps & INFCL_KEEP_X ? plan_of(m, k, n).total : 0;
  r.bwd = b.take(dx > dw ? dx : dw);
  r.kept = p.used, r.fwd_bytes = f.used, r.bwd_bytes = b.used;
  return r;
}
// The limits of the products that there are: the rows are a contraction for dw alone.
infcl_status layer_status(int64_t n, int64_t k, int64_t m, int keeps) {
  if (n < 0 || k < 1 || m < 1 || keeps < 0 || keeps > 3) return INFCL_ERR_INVALID;
  if (k % 8 != 0 || m % 8 != 0 || m > ((int64_t)1 << 23) || m > ((int64_t)1 << 36) / k ||
      n > ((int64_t)1 << 37) / (k > m ? k : m))
    return INFCL_ERR_UNSUPPORTED;
  infcl_status s = sizes_status(n, m, k);
  if (s == INFCL_OK && keeps & INFCL_KEEP_W) s = sizes_status(n, k, m);
  return s == INFCL_OK && keeps & INFCL_KEEP_X ? sizes_status(m, k, n) : s;
}

}  // namespace
}  // namespace infcl

using namespace infcl;

extern "C" infcl_status infcl_fp8_matmul_workspace(int64_t n, int64_t m, int64_t k, size_t* bytes) {
  if (!bytes) return INFCL_ERR_INVALID;
  const infcl_status s = sizes_status(n, m, k);
  if (s == INFCL_OK) *bytes = plan_of(n, m, k).total;
  return s;
}

extern "C" infcl_status infcl_fp8_matmul(const void* aq, const void* aexps, int64_t n, const void* bq,
                                         const void* bexps, int64_t m, int64_t k, const void* bias, int dtype,
                                         void* out, void* workspace, size_t ws_bytes, void* stream) {
  infcl_status s = sizes_status(n, m, k);
  if (s != INFCL_OK) return s;
  if (!type_known(dtype)) return INFCL_ERR_INVALID;
  if (dtype == INFCL_F32) return INFCL_ERR_UNSUPPORTED;
  if (n == 0) return INFCL_OK;
  if ((k > 0 && (!block_aligned(aq, 16) || !block_aligned(aexps, 4) || !block_aligned(bq, 16) || !block_aligned(bexps, 4))) ||
      ((uintptr_t)bias % 4) != 0 || !block_aligned(out, 16))
    return INFCL_ERR_INVALID;
  const size_t need = plan_of(n, m, k).total;
  if (need > 0 && !block_aligned(workspace, 256)) return INFCL_ERR_INVALID;
  if (ws_bytes < need) return INFCL_ERR_WORKSPACE;
  const uint8_t *a = (const uint8_t*)aq, *ae = (const uint8_t*)aexps, *b = (const uint8_t*)bq, *be = (const uint8_t*)bexps;
  return dtype == INFCL_BF16 ? matmul_t<false>(a, ae, n, b, be, m, k, bias, out, (char*)workspace, (hipStream_t)stream)
                             : matmul_t<true>(a, ae, n, b, be, m, k, bias, out, (char*)workspace, (hipStream_t)stream);
}

extern "C" infcl_status infcl_fp8_linear_workspace(int64_t n, int64_t m, int64_t k, size_t* bytes) {
  if (!bytes) return INFCL_ERR_INVALID;
  const infcl_status s = sizes_status(n, m, k);
  if (s != INFCL_OK) return s;
  *bytes = few(n) ? 0 : up256((size_t)n * (size_t)fp8_pitch(k)) + up256((size_t)n * (size_t)fp8_ep(k)) + plan_of(n, m, k).total;
  return INFCL_OK;
}

extern "C" infcl_status infcl_fp8_linear(const void* x, int64_t x_stride, int64_t n, int64_t k, const void* wq,
                                         const void* wexps, int64_t m, const void* bias, int dtype, void* out,
                                         void* workspace, size_t ws_bytes, void* stream) {
  infcl_status s = sizes_status(n, m, k);
  if (s != INFCL_OK) return s;
  if (k < 1 || !type_known(dtype) || x_stride < k) return INFCL_ERR_INVALID;
  if (dtype == INFCL_F32 || k % 8 != 0 || x_stride % 8 != 0 || x_stride > ((int64_t)1 << 32) || n > ((int64_t)1 << 37) / k)
    return INFCL_ERR_UNSUPPORTED;
  if (n == 0) return INFCL_OK;
  if (!block_aligned(x, 16) || !block_aligned(wq, 16) || !block_aligned(wexps, 4) || ((uintptr_t)bias % 4) != 0 ||
      !block_aligned(out, 16))
    return INFCL_ERR_INVALID;
  size_t need = 0;
  infcl_fp8_linear_workspace(n, m, k, &need);
  if (need > 0 && !block_aligned(workspace, 256)) return INFCL_ERR_INVALID;
  if (ws_bytes < need) return INFCL_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  if (few(n)) {
    const dim3 grid((unsigned)((m + 15) / 16)), block(64 * kFewWaves);
    if (dtype == INFCL_BF16)
      hipLaunchKernelGGL((few_kernel<false>), grid, block, 0, st, (const uint16_t*)x, x_stride, (int)n, k, (const uint8_t*)wq,
                         (const uint8_t*)wexps, m, fp8_pitch(k), fp8_ep(k), (const __bf16*)bias, (__bf16*)out);
    else
      hipLaunchKernelGGL((few_kernel<true>), grid, block, 0, st, (const uint16_t*)x, x_stride, (int)n, k, (const uint8_t*)wq,
                         (const uint8_t*)wexps, m, fp8_pitch(k), fp8_ep(k), (const __bf16*)bias, (__bf16*)out);
    return launch_status();
  }
  char* q = (char*)workspace;
  char* e = q + up256((size_t)n * (size_t)fp8_pitch(k));
  char* rest = e + up256((size_t)n * (size_t)fp8_ep(k));
  s = infcl_fp8_pack(x, x_stride, n, k, dtype, q, e, nullptr, nullptr, nullptr, nullptr, 0, stream);
  if (s != INFCL_OK) return s;
  return infcl_fp8_matmul(q, e, n, wq, wexps, m, k, bias, dtype, out, rest, ws_bytes - (size_t)(rest - q), stream);
}

extern "C" infcl_status infcl_fp8_layer_sizes(int64_t n, int64_t k, int64_t m, int keeps, size_t* kept_bytes,
                                              size_t* fwd_bytes, size_t* bwd_bytes) {
  const infcl_status s = layer_status(n, k, m, keeps);
  if (s != INFCL_OK) return s;
  if (!kept_bytes || !fwd_bytes || !bwd_bytes) return INFCL_ERR_INVALID;
  const LayerPlaces r = layer_places(n, k, m, keeps, nullptr, nullptr);
  *kept_bytes = r.kept, *fwd_bytes = r.fwd_bytes, *bwd_bytes = r.bwd_bytes;
  return INFCL_OK;
}

extern "C" infcl_status infcl_fp8_layer_fwd(const void* x, int64_t x_stride, int64_t n, int64_t k, const void* w,
                                            int64_t w_stride, int64_t m, const void* bias, int dtype, int keeps,
                                            void* out, void* kept, void* workspace, size_t ws_bytes, void* stream) {
  infcl_status s = layer_status(n, k, m, keeps);
  if (s != INFCL_OK) return s;
  if (!type_known(dtype) || x_stride < k || w_stride < k) return INFCL_ERR_INVALID;
  if (dtype == INFCL_F32 || x_stride % 8 != 0 || w_stride % 8 != 0 || x_stride > ((int64_t)1 << 32) ||
      w_stride > ((int64_t)1 << 32))
    return INFCL_ERR_UNSUPPORTED;
  if ((n > 0 && (!block_aligned(x, 16) || !block_aligned(out, 16))) || !block_aligned(w, 16) || ((uintptr_t)bias % 4) != 0 ||
      (keeps && !block_aligned(kept, 256)) || !block_aligned(workspace, 256))
    return INFCL_ERR_INVALID;
  const LayerPlaces r = layer_places(n, k, m, keeps, kept, workspace);
  if (ws_bytes < r.fwd_bytes) return INFCL_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  s = fp8_pack_two(x, x_stride, n, w, w_stride, m, k, dtype, r.x, r.xe, r.xt, r.xte, r.w, r.we, r.wt, r.wte, st);
  if (s != INFCL_OK || n == 0) return s;
  return infcl_fp8_matmul(r.x, r.xe, n, r.w, r.we, m, k, bias, dtype, out, r.fwd, ws_bytes, stream);
}

extern "C" infcl_status infcl_fp8_layer_bwd(const void* dy, int64_t dy_stride, int64_t n, int64_t k, int64_t m,
                                            int dtype, int keeps, const void* kept, void* dx, void* dw, void* db,
                                            void* workspace, size_t ws_bytes, void* stream) {
  infcl_status s = layer_status(n, k, m, keeps);
  if (s != INFCL_OK) return s;
  if (!type_known(dtype) || dy_stride < m || (dx && !(keeps & INFCL_KEEP_W)) || (dw && !(keeps & INFCL_KEEP_X)))
    return INFCL_ERR_INVALID;
  if (dtype == INFCL_F32 || dy_stride % 8 != 0 || dy_stride > ((int64_t)1 << 32)) return INFCL_ERR_UNSUPPORTED;
  if (!dx && !dw && !db) return INFCL_OK;
  if ((n > 0 && !block_aligned(dy, 16)) || ((uintptr_t)dx % 16) != 0 || ((uintptr_t)dw % 16) != 0 || ((uintptr_t)db % 4) != 0 ||
      ((dx || dw) && !block_aligned(kept, 256)) || !block_aligned(workspace, 256))
    return INFCL_ERR_INVALID;
  const LayerPlaces r = layer_places(n, k, m, keeps, (void*)kept, workspace);
  if (ws_bytes < r.bwd_bytes) return INFCL_ERR_WORKSPACE;
  s = infcl_fp8_pack(dy, dy_stride, n, m, dtype, dx ? r.dy : nullptr, dx ? r.dye : nullptr, dw ? r.dyt : nullptr,
                     dw ? r.dyte : nullptr, db, r.sums, ws_bytes, stream);
  if (s != INFCL_OK) return s;
  if (dx && n > 0) s = infcl_fp8_matmul(r.dy, r.dye, n, r.wt, r.wte, k, m, nullptr, dtype, dx, r.bwd, ws_bytes, stream);
  if (s != INFCL_OK || !dw) return s;
  return infcl_fp8_matmul(r.dyt, r.dyte, m, r.xt, r.xte, k, n, nullptr, dtype, dw, r.bwd, ws_bytes, stream);
}

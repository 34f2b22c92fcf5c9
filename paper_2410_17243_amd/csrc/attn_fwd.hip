// Packed attention, forward: grouped heads, causal or full, sequences of any
// lengths one after another.
//
//   s_ij = scale <q_i, k_j>,  lse_i = log sum_j e^{s_ij},  o_i = sum_j e^{s_ij - lse_i} v_j
//
// over the keys j that i sees.  One pass over the keys with the running maximum
// M and sum l of each row: scores are the product of swept key rows with own
// query rows, which leaves a query's scores in the registers of two lanes; the
// weights, rounded to 16 bits (relative 2^-8 or 2^-11 of each at most, as the inputs
// are), enter the second product from the registers they are in, against the
// sum of the unrounded ones.  M follows the scores only when they pass it by
// 2^8, so that the accumulators are rarely rescaled.
//
// Own rows are (query, head of the group) pairs: the heads that share keys read
// them together, which a single query token needs most.  Where rows are few
// and keys many the keys are cut into parts; each part leaves its M, l and
// unnormalised sums in fp32, and a second launch joins them in order.
//
// 64 features, causal, 2 x 8192 tokens, 8 heads: 168 us, 818 TFLOP/s of the visible
// pairs; 128 features, up to 4096 tokens, 16 heads over 4: 168 us, 830 TFLOP/s, MFMAs
// busy 39% of the time.  Bound there by the exponentials and the other vector work of the weights (per
// 64 keys and 32 rows 130 instructions and 32 exponentials beside 16 or 32
// products), of which half runs beside the products of another wave.  256 x 257
// tokens, 16 heads of 64: 204 us, 543 MB at 2.7 TB/s: the 257th row and key cost a
// third row tile and a fifth key tile.  One token each of 64 sequences over up to
// 8192 keys, 32 heads of 128 over 8: 224 us, 4.9 TB/s, the rate of a large copy.
#include "attn.hpp"

namespace infcl {
namespace {

constexpr float kSlack = 8.f;  // log2 of how far scores may pass the running maximum

// What a part of the keys leaves, for row id token * heads + head.
struct AttnParts {
  float* o;   // [parts][rows][hd]
  float* ml;  // [parts][rows][2]: M scale log2(e), l (-1: sees keys, all of score -infinity)
  int64_t rows;
};

// One workgroup's tile t of sequence sq's rows (query, head of the group kv), over
// its part of the keys.  again: LDS is in use.  CUT: keys of the tiles that a mask
// cuts one by one (attn.hpp).  Returns whether the wave's sums were not finite.
template <int DP, int NW, int KT, bool F16, bool SPLIT, bool CUT>
__device__ __forceinline__ bool attn_fwd_tile(const AttnArgs& a, uint16_t* __restrict__ out, int64_t os, int64_t oh,
                                              float* __restrict__ lse, int parts, const AttnParts& pw,
                                              const AttnSeq& sq, int kv, int part, uint32_t t, uint32_t rows,
                                              INFCL_LDS char* lds, bool again) {
  constexpr int kFb = DP / 32, kI = DP / 16, kKb = KT / 32;
  typedef AttnTile<DP, NW, KT> Tile;
  const int wave = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int h = lane >> 5;
  AttnLanes<DP> ln;
  ln.init(lane);
  const uint32_t kst = (uint32_t)(a.ks * 2), vst = (uint32_t)(a.vs * 2);
  uint32_t koff[Tile::kVar], voff[Tile::kVar];
  Tile::offsets(koff, wave, lane, kst, a.hd);
  Tile::offsets(voff, wave, lane, vst, a.hd);
  const uint16_t* kb = a.k + sq.k0 * a.ks + kv * a.kh;
  const uint16_t* vb = a.v + sq.k0 * a.vs + kv * a.vh;
  // this part's keys
  const int per = SPLIT ? ((sq.n + parts - 1) / parts + KT - 1) / KT * KT : 0;
  const int kbeg = SPLIT ? (part * per < sq.n ? part * per : sq.n) : 0;
  const int kstop = SPLIT ? (kbeg + per < sq.n ? kbeg + per : sq.n) : sq.n;

  const uint32_t r = t * (32 * NW) + wave * 32 + (lane & 31);
  const bool live = r < rows;
  const int pos = live ? (int)(r / (uint32_t)a.group) : 0, g = live ? (int)(r % (uint32_t)a.group) : 0;
  const int head = kv * a.group + g;
  const int64_t token = sq.q0 + pos;

  // keys [0, lim) are seen by this lane's row; every row of the wave sees
  // those below wmin, none of the workgroup those from kend on
  const int shift = sq.n - sq.m + 1;
  int lim = a.causal ? pos + shift : sq.n;
  lim = lim < 0 ? 0 : lim;
  if (!live) lim = 0;
  const uint32_t rl = t * (uint64_t)(32 * NW) + 32 * NW < rows ? t * (32 * NW) + 32 * NW - 1 : rows - 1;
  int kend = a.causal ? (int)(rl / (uint32_t)a.group) + shift : sq.n;
  kend = kend < kstop ? kend : kstop;
  const uint32_t rw = t * (32 * NW) + wave * 32;  // the wave's first row, and its last
  const uint32_t rv = rw + 31 < rows ? rw + 31 : rows - 1;
  const int wmin = rw >= rows ? 0 : a.causal ? (int)(rw / (uint32_t)a.group) + shift : sq.n;
  const int wmax = rw >= rows ? 0 : a.causal ? (int)(rv / (uint32_t)a.group) + shift : sq.n;

  f32x16 acc[kFb];
#pragma unroll
  for (int fb = 0; fb < kFb; ++fb) acc[fb] = f32x16_zero();
  float M = -__builtin_inff(), l = 0.f;
  if (again) attn_barrier();
  if (kbeg < kend) {
    Tile::issue(kb + (int64_t)kbeg * a.ks, sq.n - kbeg, kst, a.hd, lds, koff, wave);
    Tile::issue(vb + (int64_t)kbeg * a.vs, sq.n - kbeg, vst, a.hd, lds + Tile::kBytes, voff, wave);
  }
  bf16x8 qf[kI];
#pragma unroll
  for (int i = 0; i < kI; ++i) qf[i] = attn_own(a.q + token * a.qs + head * a.qh, i, h, a.hd, live);
  attn_settle(qf);
  int buf = 0;
  const int kcut = kbeg + (wmin > kbeg ? (wmin - kbeg) / KT * KT : 0), wend = CUT ? kcut : wmax;
  for (int k = kbeg; k < kend; k += KT, buf ^= 1) {
    attn_barrier();
    if (k + KT < kend) {
      INFCL_LDS char* nx = lds + (buf ^ 1) * 2 * Tile::kBytes;
      Tile::issue(kb + (int64_t)(k + KT) * a.ks, sq.n - k - KT, kst, a.hd, nx, koff, wave);
      Tile::issue(vb + (int64_t)(k + KT) * a.vs, sq.n - k - KT, vst, a.hd, nx + Tile::kBytes, voff, wave);
    }
    if (k >= wend) continue;
    const INFCL_LDS char* kt = lds + buf * 2 * Tile::kBytes;
    const INFCL_LDS char* vt = kt + Tile::kBytes;
    // All row fragments first, then the products, and the transposed fragments of
    // the second product while the weights are formed: left to itself the compiler
    // waits for each LDS read right before its product.
    bf16x8 kf[kKb][kI];
#pragma unroll
    for (int b = 0; b < kKb; ++b)
#pragma unroll
      for (int i = 0; i < kI; ++i) kf[b][i] = attn_row(kt + b * 32 * Tile::kRow + ln.row[i]);
    __builtin_amdgcn_sched_barrier(0);
    f32x16 s[kKb];
#pragma unroll
    for (int b = 0; b < kKb; ++b) {
      s[b] = f32x16_zero();
#pragma unroll
      for (int i = 0; i < kI; ++i) s[b] = mfma16<F16>(kf[b][i], qf[i], s[b]);
    }
    __builtin_amdgcn_sched_barrier(0);
    bf16x8 vf[kKb][2][kFb];
#pragma unroll
    for (int b = 0; b < kKb; ++b)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int fb = 0; fb < kFb; ++fb) {
          const int ro = (32 * b + 16 * u) * Tile::kRow;
          vf[b][u][fb] = attn_tr(vt + ro + ln.tr[0][fb], vt + ro + ln.tr[1][fb]);
        }
    __builtin_amdgcn_sched_barrier(0);
    if (k + KT > wmin) {
      const int left = attn_opaque(lim - k - 4 * h);
#pragma unroll
      for (int b = 0; b < kKb; ++b)
#pragma unroll
        for (int x = 0; x < 16; ++x) s[b][x] = 32 * b + attn_reg_row(x, 0) < left ? s[b][x] : -__builtin_inff();
    }
    float top = s[0][0];
#pragma unroll
    for (int b = 0; b < kKb; ++b)
#pragma unroll
      for (int x = 0; x < 16; ++x) top = fmaxf(top, s[b][x]);
    top = attn_max2(top);
    const bool up = top * a.sl2 > M * a.sl2 + kSlack || (M == -__builtin_inff() && top > M);
    if (wave_any(up)) {
      const float Mn = up ? top : M;
      const float f = up && M != -__builtin_inff() ? exp2_hw((M - Mn) * a.sl2) : 1.f;  // (nothing summed yet: 0)
      M = Mn;
      l *= f;
#pragma unroll
      for (int fb = 0; fb < kFb; ++fb)
#pragma unroll
        for (int x = 0; x < 16; ++x) acc[fb][x] *= f;
    }
    const float ref = M == -__builtin_inff() ? 0.f : M * a.sl2;
#pragma unroll
    for (int b = 0; b < kKb; ++b)
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        s[b][x] = exp2_hw(fmaf(s[b][x], a.sl2, -ref));
        l += s[b][x];
      }
#pragma unroll
    for (int b = 0; b < kKb; ++b)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const bf16x8 p = attn_pack<F16>(s[b], u);
#pragma unroll
        for (int fb = 0; fb < kFb; ++fb) acc[fb] = mfma16<F16>(vf[b][u][fb], p, acc[fb]);
      }
  }
  if (CUT && live) {
    const uint16_t* q = a.q + token * a.qs + head * a.qh;
    const int stop = lim < kstop ? lim : kstop;
    float top = M;
#pragma unroll 1
    for (int k = kcut; k < stop; ++k) top = fmaxf(top, attn_dot<F16>(q, kb + k * a.ks, h, a.hd));
    const float f = M == -__builtin_inff() ? 1.f : exp2_hw((M - top) * a.sl2);  // (nothing summed yet: 0)
    M = top;
    l *= f;
#pragma unroll
    for (int fb = 0; fb < kFb; ++fb)
#pragma unroll
      for (int x = 0; x < 16; ++x) acc[fb][x] *= f;
    const float ref = M == -__builtin_inff() ? 0.f : M * a.sl2;
#pragma unroll 1
    for (int k = kcut; k < stop; ++k) {
      const float p = exp2_hw(fmaf(attn_dot<F16>(q, kb + k * a.ks, h, a.hd), a.sl2, -ref));
      l += h ? 0.f : p;
      attn_axpy<F16>(acc, p, vb + k * a.vs, h, a.hd);
    }
  }
  l = attn_sum2(l);
  const int64_t id = token * a.heads + head;
  float* po = SPLIT ? pw.o + ((int64_t)part * pw.rows + id) * a.hd : nullptr;
  float* ml = SPLIT ? pw.ml + ((int64_t)part * pw.rows + id) * 2 : nullptr;
  const bool bad = !CUT && a.causal && wave_any(live && attn_bad(acc));
  if (!live) return bad;
  if constexpr (SPLIT) {
#pragma unroll
    for (int fb = 0; fb < kFb; ++fb)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int d = 32 * fb + 8 * j + 4 * h;
        if (d < a.hd)
          *(f32x4*)(po + d) = f32x4{acc[fb][4 * j], acc[fb][4 * j + 1], acc[fb][4 * j + 2], acc[fb][4 * j + 3]};
      }
    if (h == 0) {
      ml[0] = l > 0.f || l != l ? M * a.sl2 : -__builtin_inff();
      ml[1] = l == 0.f && lim > kbeg && kstop > kbeg ? -1.f : l;
    }
  } else {
    if (l == 0.f && lim > 0) l = __builtin_nanf("");  // (scores of -infinity only: no weights)
    const float inv = l == 0.f ? 0.f : 1.f / l;
    attn_store<F16>(out + token * os + head * oh, acc, inv, h, a.hd);
    if (lse && h == 0) lse[(int64_t)head * a.tq + token] = l == 0.f ? -__builtin_inff() : fmaf(M, a.scale, logf(l));
  }
  return bad;
}

struct AttnFwdArgs {
  AttnArgs a;
  uint16_t* out;
  int64_t os, oh;
  float* lse;
  int tiles, parts;
  AttnParts pw;
};

// Workgroup idx takes rows [32 NW t, +32 NW) of sequence z's group of heads kv,
// t descending (with causal masks the last rows see most keys), and part
// `part` of its keys.
template <int DP, int NW, int KT, bool F16, bool SPLIT>
__global__ void __launch_bounds__(64 * NW, 2)
    attn_fwd_kernel(AttnFwdArgs c) {
  const AttnArgs& a = c.a;
  const int tiles = c.tiles, parts = c.parts;
  __shared__ __attribute__((aligned(1024))) char lds[4 * AttnTile<DP, NW, KT>::kBytes];
  __shared__ int flags[NW];
  uint32_t idx = blockIdx.x;
  const int part = SPLIT ? (int)(idx % (uint32_t)parts) : 0;
  if (SPLIT) idx /= (uint32_t)parts;
  const uint32_t groups = (uint32_t)(a.nseq + 1) * (uint32_t)a.kvh;
  const AttnPlace at = attn_place(idx, (uint32_t)tiles, groups);
  const int t0 = tiles - 1 - (int)at.t;
  const int z = (int)(at.g / (uint32_t)a.kvh), kv = (int)(at.g % (uint32_t)a.kvh);
  AttnSeq sq = attn_seq(a, z);
  if (z == a.nseq) sq.n = 0;
  const int64_t rows64 = (int64_t)sq.m * a.group;
  const uint32_t rows = rows64 > 0x7FFFFFFF ? 0x7FFFFFFFu : (uint32_t)rows64;
  // (one tile, unless sequences are longer than the caller said)
  bool bad = false;
  for (uint32_t t = (uint32_t)t0; t * (uint64_t)(32 * NW) < rows; t += (uint32_t)tiles)
    bad |= attn_fwd_tile<DP, NW, KT, F16, SPLIT, false>(a, c.out, c.os, c.oh, c.lse, parts, c.pw, sq, kv, part, t, rows,
                                                        (INFCL_LDS char*)lds, t != (uint32_t)t0);
  if (!a.causal) return;
  const int wave = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  bool odd = false;  // values of the tiles that a mask cuts
  if (bad) {
    const AttnArgs r = attn_reload<AttnFwdArgs>().a;
    for (uint32_t t = (uint32_t)t0; t * (uint64_t)(32 * NW) + 32 * wave < rows; t += (uint32_t)tiles)
      odd |= attn_odd_keys<F16>(r.v + sq.k0 * r.vs + kv * r.vh, r.vs, r.hd, sq, r.group, t * (32 * NW) + 32 * wave, rows,
                                KT);
  }
  if (!attn_vote<NW>(odd, (INFCL_LDS int*)flags, wave)) return;
  const AttnFwdArgs r = attn_reload<AttnFwdArgs>();
  for (uint32_t t = (uint32_t)t0; t * (uint64_t)(32 * NW) < rows; t += (uint32_t)tiles)
    attn_fwd_tile<DP, NW, KT, F16, SPLIT, true>(r.a, r.out, r.os, r.oh, r.lse, r.parts, r.pw, sq, kv, part, t, rows,
                                                (INFCL_LDS char*)lds, true);
}

// Joins the parts of every row: M the largest, l and o the rescaled sums.  A
// wave takes 64 / lanes rows; a lane 4 features at a time.
template <bool F16>
__global__ void __launch_bounds__(256) attn_join(AttnParts pw, int parts, int heads, int hd, int64_t tq,
                                                 uint16_t* __restrict__ out, int64_t os, int64_t oh,
                                                 float* __restrict__ lse) {
  const int d = 4 * (threadIdx.x & 31);
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 5; i < pw.rows; i += (int64_t)gridDim.x * 8) {
    float M = -__builtin_inff();
    for (int p = 0; p < parts; ++p) M = fmaxf(M, pw.ml[((int64_t)p * pw.rows + i) * 2]);
    float l = 0.f;
    bool none = true;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int p = 0; p < parts; ++p) {
      const float* ml = pw.ml + ((int64_t)p * pw.rows + i) * 2;
      none = none && ml[1] == 0.f;  // (sees nothing of this part)
      if (ml[1] <= 0.f) continue;
      const float f = exp2_hw(ml[0] - M);
      l = fmaf(ml[1], f, l);
      if (d < hd) {
        const f32x4 x = *(const f32x4*)(pw.o + ((int64_t)p * pw.rows + i) * hd + d);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf(x[e], f, o[e]);
      }
    }
    if (l == 0.f && !none) l = __builtin_nanf("");
    const int64_t token = i / heads;
    const int head = (int)(i % heads);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (d < hd) {
      uint16_t* po = out + token * os + head * oh + d;
#pragma unroll
      for (int e = 0; e < 4; ++e) po[e] = __builtin_bit_cast(uint16_t, to16<F16>(o[e] * inv));
    }
    if (lse && d == 0) lse[(int64_t)head * tq + token] = l == 0.f ? -__builtin_inff() : kLn2 * M + logf(l);
  }
}

template <int DP, bool F16, int NW, int KT>
void launch_one(const AttnArgs& a, const AttnFwdPlan& p, uint16_t* out, int64_t os, int64_t oh, float* lse, char* ws,
                hipStream_t st) {
  AttnParts pw{(float*)(ws + p.o), (float*)(ws + p.ml), a.tq * a.heads};
  const dim3 grid((unsigned)(p.tiles * attn_groups(a) * p.parts));
  const AttnFwdArgs c{a, out, os, oh, lse, p.tiles, p.parts, pw};
  if (p.parts > 1)
    hipLaunchKernelGGL((attn_fwd_kernel<DP, NW, KT, F16, true>), grid, dim3(64 * NW), 0, st, c);
  else
    hipLaunchKernelGGL((attn_fwd_kernel<DP, NW, KT, F16, false>), grid, dim3(64 * NW), 0, st, c);
}

}  // namespace

// Rows of a sequence's group of heads, the waves of a workgroup, and the parts of
// the keys.  Sequences of at most 128 rows run one wave to a workgroup: their
// waves need not wait for one another, and short ones leave no wave idle (1024
// captions of up to 77 tokens, 8 heads of 64: 25 us, four waves 42).  Near the edge
// it is the rows in the last tile that decide (32768 tokens in equal lengths, 8 heads
// of 64, causal, forward and backward, one wave | four: 64 rows 32 + 95 | 34 + 95 us,
// 96 rows 31 + 92 | 34 + 101, 128 rows 36 + 105 | 32 + 100, 160 rows 33 + 99 | 38 + 138,
// 256 rows 41 + 117 | 36 + 118).  Keys are cut
// where there are fewer workgroups than two waves for every SIMD (one token over
// 777 keys, 8 heads of 64: 12 us with the join, 18 uncut; 64 over up to 8192, 8 key
// heads of 128: 219 and 264).  Tiles of 64 keys for four waves: 2 x 8192 tokens,
// 8 heads of 64, 169 us, with 32 keys 196 (256 x 257 tokens: 201 and 194).
AttnFwdPlan attn_fwd_plan(const AttnArgs& a, int64_t max_q, int64_t max_k) {
  AttnFwdPlan p;
  const int64_t rows = (max_q < 1 ? 1 : max_q) * a.group;
  p.nw = rows <= 128 || attn_groups(a) > kAttnItems / 256 ? 1 : 4;  // (so many pairs: one wave each fits a launch)
  p.tiles = (int)((rows + 32 * p.nw - 1) / (32 * p.nw));
  const int64_t wgs = (int64_t)p.tiles * (a.nseq > 1 ? a.nseq : 1) * a.kvh, want = p.nw == 1 ? 2048 : 512;
  int64_t parts = 1;
  if (wgs < want) {
    parts = (want + wgs - 1) / wgs;
    const int64_t most = (max_k + 255) / 256;  // a part has at least 256 keys
    if (parts > most) parts = most;
    if (parts < 1) parts = 1;
  }
  p.parts = (int)parts;
  p.tiles = (int)attn_at_once(p.tiles, attn_groups(a) * parts, 64 * p.nw);
  const size_t r = (size_t)a.tq * (size_t)a.heads;
  size_t off = 0;
  p.o = off, off = (off + (parts > 1 ? r * a.hd * 4 * parts : 0) + 255) & ~(size_t)255;
  p.ml = off, off = (off + (parts > 1 ? r * 8 * parts : 0) + 255) & ~(size_t)255;
  p.total = off;
  return p;
}

template <bool F16>
static int attn_fwd_t(const AttnArgs& a, const AttnFwdPlan& p, uint16_t* out, int64_t os, int64_t oh, float* lse,
                      char* ws, hipStream_t st) {
  if (a.hd <= 64) {
    if (p.nw == 1)
      launch_one<64, F16, 1, 32>(a, p, out, os, oh, lse, ws, st);
    else
      launch_one<64, F16, 4, 64>(a, p, out, os, oh, lse, ws, st);
  } else {
    if (p.nw == 1)
      launch_one<128, F16, 1, 32>(a, p, out, os, oh, lse, ws, st);
    else
      launch_one<128, F16, 4, 64>(a, p, out, os, oh, lse, ws, st);
  }
  if (hipGetLastError() != hipSuccess) return INFCL_ERR_HIP;
  if (p.parts > 1) {
    AttnParts pw{(float*)(ws + p.o), (float*)(ws + p.ml), a.tq * a.heads};
    const dim3 grid((unsigned)attn_at_once((pw.rows + 7) / 8, 1, 256));
    hipLaunchKernelGGL((attn_join<F16>), grid, dim3(256), 0, st, pw, p.parts, a.heads, a.hd, a.tq, out, os, oh, lse);
    if (hipGetLastError() != hipSuccess) return INFCL_ERR_HIP;
  }
  return INFCL_OK;
}

int launch_attn_fwd(const AttnArgs& a, const AttnFwdPlan& p, int dtype, uint16_t* out, int64_t os, int64_t oh,
                    float* lse, char* ws, hipStream_t st) {
  return dtype == INFCL_F16 ? attn_fwd_t<true>(a, p, out, os, oh, lse, ws, st)
                            : attn_fwd_t<false>(a, p, out, os, oh, lse, ws, st);
}

}  // namespace infcl

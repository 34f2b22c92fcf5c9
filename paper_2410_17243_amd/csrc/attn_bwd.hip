// Packed attention, backward: grouped heads, causal or full.
//
//   p_ij = e^{s_ij - lse_i},  dp_ij = <do_i, v_j>,  D_i = <do_i, o_i> = sum_j p_ij dp_ij,
//   ds_ij = p_ij (dp_ij - D_i),
//   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i,
//
// the sums over i running over all heads that share key j.  Two sweeps, each of
// which recomputes the weights from lse: one owns queries and sums dq, one owns
// keys and sums dk and dv.  That is seven products where one sweep with atomic
// additions would need five, but no atomics, no zeroing, one write of every
// gradient, and sums in a fixed order.  The first sweep also writes D and
// lse log2(e), rows with no keys as 0, for the second.
//
// p and ds are rounded to 16 bits for the second products, as the inputs are.
// D comes from o as stored, except in waves none of whose rows sees past the first
// tile of keys (32 or 64): there it is the sum of p dp in the registers, which no
// rounding of o touches.  (The error of D from o's rounding, beside that of rounding
// ds, is the sum of p^2 over a row in the mean square: near 1 for a row that sees
// few keys, 3 / n over n keys of similar scores.  Which of the two a row of few keys
// gets depends on the rows beside it.)  ds is rounded as it stands: in fp16 its
// range is that of dout's products with v times p, about 1 / n over n keys of
// similar scores, so that long rows leave the normal numbers long before dout
// does, which loss scaling has to respect.
//
// 4 sequences of up to 4096 tokens, 16 heads of 128 over 4: dq 231 us (900 TFLOP/s,
// MFMAs busy 42% of the time), dk and dv 338 us (820, 39%) and 23 us to join their
// parts; bound by the latency of each tile's chain (products, weights, products) at
// two waves per SIMD, which is what 128 features' accumulators leave.  1024 captions
// of about 17 tokens, 8 heads of 64: 28 and 32 us; a wave's chain of loads for one tile
// of work, five waves to a compute unit.
#include "attn.hpp"

namespace infcl {
namespace {

// Workgroups that the sweeps over queries, and over keys, are cut into, about (4
// sequences of up to 4096 tokens, 4 key heads: dk and dv with their join 819 us
// uncut, 475, 362, 372 and 370 at 512, 768, 1024 and 1536; 3 of up to 3371 tokens, one
// key head: dq 115 us uncut, 81 so).
constexpr int64_t kBwdGroups = 768, kBwdRowGroups = 384;

struct AttnGrads {
  const uint16_t *out, *dout;
  int64_t os, oh, dos, doh;
  const float* lse;
  float* stat;  // [heads][trow][2]: lse log2(e), D; 32 entries past the tokens may be read
  int64_t trow;
  float* part;    // [parts][dk, dv][tokens][kvh][hd]: sums of parts of the sweeps over queries
  float* part_q;  // [parts][tokens][heads][hd]: ... over keys
  uint16_t *dq, *dk, *dv;
  int64_t dqs, dqh, dks, dkh, dvs, dvh;
};

// Whether dk's and dv's sweeps keep the own values in LDS (below).
constexpr bool attn_own_in_lds(int dp, int nw) { return dp == 128 && nw > 1; }  // (a lone wave's tiles leave it a SIMD's registers)

// Rows [32 NW t, +32 NW) of (query, head of the group kv); sweeps the keys they see.
// SPLIT: one of several parts of the keys, whose sums are left in fp32 for
// attn_dq_join.  again: LDS is in use.  CUT: keys of the tiles that a mask cuts one
// by one (attn.hpp).  Returns whether the wave's sums were not finite.
template <int DP, int NW, int KT, bool F16, bool SPLIT, bool CUT>
__device__ __forceinline__ bool attn_dq_tile(const AttnArgs& a, const AttnGrads& w, const AttnSeq& sq, int kv, int parts,
                                             int part, uint32_t t, uint32_t rows, INFCL_LDS char* lds, bool again) {
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

  const uint32_t r = t * (32 * NW) + wave * 32 + (lane & 31);
  const bool live = r < rows;
  const int pos = live ? (int)(r / (uint32_t)a.group) : 0, g = live ? (int)(r % (uint32_t)a.group) : 0;
  const int head = kv * a.group + g;
  const int64_t token = sq.q0 + pos;
  const int shift = sq.n - sq.m + 1;
  int lim = a.causal ? pos + shift : sq.n;
  lim = lim < 0 ? 0 : lim;
  if (!live) lim = 0;
  const uint32_t rl = t * (uint64_t)(32 * NW) + 32 * NW < rows ? t * (32 * NW) + 32 * NW - 1 : rows - 1;
  int kend = a.causal ? (int)(rl / (uint32_t)a.group) + shift : sq.n;
  kend = kend < sq.n ? kend : sq.n;
  int kbeg = 0;
  if (SPLIT) {  // shares of the keys that this tile sees
    const int share = ((kend > 0 ? kend : 0) + parts * KT - 1) / (parts * KT) * KT;
    kbeg = share * part;
    kend = kbeg + share < kend ? kbeg + share : kend;
  }
  const uint32_t rw = t * (32 * NW) + wave * 32;
  const uint32_t rv = rw + 31 < rows ? rw + 31 : rows - 1;
  const int wmin = rw >= rows ? 0 : a.causal ? (int)(rw / (uint32_t)a.group) + shift : sq.n;
  const int wmax = rw >= rows ? 0 : a.causal ? (int)(rv / (uint32_t)a.group) + shift : sq.n;

  if (again) attn_barrier();
  if (kbeg < kend) {
    Tile::issue(kb + (int64_t)kbeg * a.ks, sq.n - kbeg, kst, a.hd, lds, koff, wave);
    Tile::issue(vb + (int64_t)kbeg * a.vs, sq.n - kbeg, vst, a.hd, lds + Tile::kBytes, voff, wave);
  }
  bf16x8 qf[kI], df[kI];
  float D = 0.f;
#pragma unroll
  for (int i = 0; i < kI; ++i) {
    qf[i] = attn_own(a.q + token * a.qs + head * a.qh, i, h, a.hd, live);
    df[i] = attn_own(w.dout + token * w.dos + head * w.doh, i, h, a.hd, live);
  }
  if (wmax > KT) {
#pragma unroll
    for (int i = 0; i < kI; ++i) {
      const bf16x8 of = attn_own(w.out + token * w.os + head * w.oh, i, h, a.hd, live);
#pragma unroll
      for (int e = 0; e < 8; ++e) D = fmaf(from16<F16>(df[i][e]), from16<F16>(of[e]), D);
    }
    D = attn_sum2(D);
  }
  float lse2 = 0.f;
  if (live) lse2 = w.lse[(int64_t)head * a.tq + token] * kLog2e;
  if (lse2 == -__builtin_inff()) lse2 = 0.f, D = 0.f;
  attn_settle(qf);
  attn_settle(df);
  asm volatile("" : "+v"(lse2));
  f32x16 acc[kFb];
#pragma unroll
  for (int fb = 0; fb < kFb; ++fb) acc[fb] = f32x16_zero();
  const int kcut = kbeg + (wmin > kbeg ? (wmin - kbeg) / KT * KT : 0), wend = CUT ? kcut : wmax;
  {
    int buf = 0;
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
      f32x16 p[kKb], dp[kKb];
#pragma unroll
      for (int b = 0; b < kKb; ++b) {
        p[b] = f32x16_zero(), dp[b] = f32x16_zero();
#pragma unroll
        for (int i = 0; i < kI; ++i) {
          p[b] = mfma16<F16>(attn_row(kt + b * 32 * Tile::kRow + ln.row[i]), qf[i], p[b]);
          dp[b] = mfma16<F16>(attn_row(vt + b * 32 * Tile::kRow + ln.row[i]), df[i], dp[b]);
        }
      }
#pragma unroll
      for (int b = 0; b < kKb; ++b)
#pragma unroll
        for (int x = 0; x < 16; ++x) p[b][x] = exp2_hw(fmaf(p[b][x], a.sl2, -lse2));
      if (k + KT > wmin) {
        const int left = attn_opaque(lim - k - 4 * h);
#pragma unroll
        for (int b = 0; b < kKb; ++b)
#pragma unroll
          for (int x = 0; x < 16; ++x) {
            const bool seen = 32 * b + attn_reg_row(x, 0) < left;
            p[b][x] = seen ? p[b][x] : 0.f;
            dp[b][x] = seen ? dp[b][x] : 0.f;
          }
      }
      if (wmax <= KT) {
        float s = 0.f;
#pragma unroll
        for (int b = 0; b < kKb; ++b)
#pragma unroll
          for (int x = 0; x < 16; ++x) s = fmaf(p[b][x], dp[b][x], s);
        D = attn_sum2(s);
      }
#pragma unroll
      for (int b = 0; b < kKb; ++b) {
#pragma unroll
        for (int x = 0; x < 16; ++x) p[b][x] *= dp[b][x] - D;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const bf16x8 ds = attn_pack<F16>(p[b], u);
          const int ro = (32 * b + 16 * u) * Tile::kRow;
#pragma unroll
          for (int fb = 0; fb < kFb; ++fb)
            acc[fb] = mfma16<F16>(attn_tr(kt + ro + ln.tr[0][fb], kt + ro + ln.tr[1][fb]), ds, acc[fb]);
        }
      }
    }
  }
  const bool bad = !CUT && a.causal && wave_any(live && attn_bad(acc));
  // (the row's place made here again, not kept through the sweep)
  const int own_lane = attn_opaque(threadIdx.x & 63), oh = own_lane >> 5;
  const uint32_t own = rw + (own_lane & 31);
  if (own >= rows) return bad;
  const int own_pos = (int)(own / (uint32_t)a.group), own_head = kv * a.group + (int)(own % (uint32_t)a.group);
  const int64_t at = sq.q0 + own_pos;
  if (CUT) {
    const uint16_t *q = a.q + at * a.qs + own_head * a.qh, *dr = w.dout + at * w.dos + own_head * w.doh;
    const int lim = own_pos + shift, stop = lim < kend ? lim : kend;
    if (wmax <= KT) {
#pragma unroll 1
      for (int k = 0; k < stop; ++k)
        D = fmaf(exp2_hw(fmaf(attn_dot<F16>(q, kb + k * a.ks, oh, a.hd), a.sl2, -lse2)),
                 attn_dot<F16>(dr, vb + k * a.vs, oh, a.hd), D);
    }
#pragma unroll 1
    for (int k = kcut; k < stop; ++k) {
      const float p = exp2_hw(fmaf(attn_dot<F16>(q, kb + k * a.ks, oh, a.hd), a.sl2, -lse2));
      attn_axpy<F16>(acc, p * (attn_dot<F16>(dr, vb + k * a.vs, oh, a.hd) - D), kb + k * a.ks, oh, a.hd);
    }
  }
  if (!SPLIT || part == 0) w.stat[((int64_t)own_head * w.trow + at) * 2 + oh] = oh ? D : lse2;
  if constexpr (SPLIT) {
    float* po = w.part_q + (((int64_t)part * a.tq + at) * a.heads + own_head) * a.hd;
#pragma unroll
    for (int fb = 0; fb < kFb; ++fb)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int d = 32 * fb + 8 * j + 4 * oh;
        if (d < a.hd)
          *(f32x4*)(po + d) = f32x4{acc[fb][4 * j], acc[fb][4 * j + 1], acc[fb][4 * j + 2], acc[fb][4 * j + 3]};
      }
  } else {
    attn_store<F16>(w.dq + at * w.dqs + own_head * w.dqh, acc, a.scale, oh, a.hd);
  }
  return bad;
}

struct AttnBwdArgs {
  AttnArgs a;
  AttnGrads w;
  int tiles, parts;
};

template <int DP, int NW, int KT, bool F16, bool SPLIT>
__global__ void __launch_bounds__(64 * NW, 2) attn_dq_kernel(AttnBwdArgs c) {
  const AttnArgs& a = c.a;
  const AttnGrads& w = c.w;
  const int tiles = c.tiles, parts = c.parts;
  __shared__ __attribute__((aligned(1024))) char lds_[4 * AttnTile<DP, NW, KT>::kBytes];
  __shared__ int flags[NW];
  INFCL_LDS char* lds = (INFCL_LDS char*)lds_;
  const uint32_t groups = (uint32_t)(a.nseq + 1) * (uint32_t)a.kvh;
  const AttnPlace at = attn_place(blockIdx.x, (uint32_t)(tiles * parts), groups);
  const int t0 = tiles - 1 - (int)at.t / (SPLIT ? parts : 1), part = SPLIT ? (int)at.t % parts : 0;
  const int z = (int)(at.g / (uint32_t)a.kvh), kv = (int)(at.g % (uint32_t)a.kvh);
  AttnSeq sq = attn_seq(a, z);
  if (z == a.nseq) sq.n = 0;
  const int64_t rows64 = (int64_t)sq.m * a.group;
  const uint32_t rows = rows64 > 0x7FFFFFFF ? 0x7FFFFFFFu : (uint32_t)rows64;
  if ((int64_t)t0 * (32 * NW) >= rows) return;
  bool bad = false;
  for (uint32_t t = (uint32_t)t0; t * (uint64_t)(32 * NW) < rows; t += (uint32_t)tiles)
    bad |= attn_dq_tile<DP, NW, KT, F16, SPLIT, false>(a, w, sq, kv, parts, part, t, rows, lds, t != (uint32_t)t0);
  if (!a.causal) return;
  const int wave = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  bool odd = false;  // keys of the tiles that a mask cuts
  if (bad) {
    const AttnBwdArgs r = attn_reload<AttnBwdArgs>();
    for (uint32_t t = (uint32_t)t0; t * (uint64_t)(32 * NW) + 32 * wave < rows; t += (uint32_t)tiles)
      odd |= attn_odd_keys<F16>(r.a.k + sq.k0 * r.a.ks + kv * r.a.kh, r.a.ks, r.a.hd, sq, r.a.group,
                                t * (32 * NW) + 32 * wave, rows, KT);
  }
  if (!attn_vote<NW>(odd, (INFCL_LDS int*)flags, wave)) return;
  const AttnBwdArgs r = attn_reload<AttnBwdArgs>();
  for (uint32_t t = (uint32_t)t0; t * (uint64_t)(32 * NW) < rows; t += (uint32_t)tiles)
    attn_dq_tile<DP, NW, KT, F16, SPLIT, true>(r.a, r.w, sq, kv, r.parts, part, t, rows, lds, true);
}

// The parts' dq, in order.  A wave takes 8 rows of a sequence's key head, 16 lanes to
// a row.
template <bool F16>
__global__ void __launch_bounds__(256) attn_dq_join(AttnArgs a, AttnGrads w, int tiles, int parts) {
  const uint32_t groups = (uint32_t)(a.nseq + 1) * (uint32_t)a.kvh;
  const uint32_t gz = blockIdx.x % groups;
  const int z = (int)(gz / (uint32_t)a.kvh), kv = (int)(gz % (uint32_t)a.kvh);
  AttnSeq sq = attn_seq(a, z);
  if (z == a.nseq) sq.n = 0;
  const int64_t rows = (int64_t)sq.m * a.group, step = a.tq * a.heads * a.hd;
  const int lane = threadIdx.x & 63, d = 8 * (lane & 15);
  for (int64_t r0 = (int64_t)(blockIdx.x / groups) * 32 + (threadIdx.x >> 6) * 8; r0 < rows; r0 += (int64_t)tiles * 32) {
#pragma unroll
    for (int i = lane >> 4; i < 8; i += 4) {
      if (r0 + i >= rows || d >= a.hd) continue;
      const uint32_t r = (uint32_t)(r0 + i);
      const int64_t token = sq.q0 + r / (uint32_t)a.group;
      const int head = kv * a.group + (int)(r % (uint32_t)a.group);
      const float* src = w.part_q + (token * a.heads + head) * a.hd + d;
      float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll 4
      for (int p = 0; p < parts; ++p) {
        const f32x4* x = (const f32x4*)(src + p * step);
        const f32x4 x0 = x[0], x1 = x[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += x0[e], acc[4 + e] += x1[e];
      }
      attn_store8<F16>(w.dq + token * w.dqs + head * w.dqh + d, acc, a.scale);
    }
  }
}

// Owns 32 NW keys; sweeps the queries that see them, of all heads of the group:
// tiles from the last queries down, the heads of a tile one after another.  All
// workgroups of a sequence's key head begin with the same tiles that way and go
// through them together, so that the copies find them in L2.
// At 128 features the own rows, the two sums and a tile's weights are more than
// the registers of two waves per SIMD: the own values stay in LDS there (a fifth
// of the sweep's LDS reads), for a register spilled in the sweep costs more
// (its reload waits for the tile copies in flight); none is.
// SPLIT: a workgroup takes one of several parts of the tiles and leaves its sums in
// fp32 for attn_dkv_join.
// again: LDS is in use.  CUT: queries of the tiles that a mask cuts one by one
// (attn.hpp).  Returns whether the wave's sums were not finite.
template <int DP, int NW, bool F16, bool SPLIT, bool CUT>
__device__ __forceinline__ bool attn_dkv_tile(const AttnArgs& a, const AttnGrads& w, const AttnSeq& sq, int kv, int parts,
                                              int part, int64_t t, INFCL_LDS char* lds, INFCL_LDS float* stat, bool again) {
  constexpr int kFb = DP / 32, kI = DP / 16, QT = 32;
  constexpr bool kVLds = attn_own_in_lds(DP, NW);
  typedef AttnTile<DP, NW, QT> Tile;
  typedef AttnTile<DP, NW, 32 * NW> Own;
  const int wave = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int h = lane >> 5;
  AttnLanes<DP> ln;
  ln.init(lane);
  const uint32_t qst = (uint32_t)(a.qs * 2), dst = (uint32_t)(w.dos * 2);
  uint32_t qoff[Tile::kVar], doff[Tile::kVar];
  Tile::offsets(qoff, wave, lane, qst, a.hd);
  Tile::offsets(doff, wave, lane, dst, a.hd);

  const int key0 = (int)(t * (32 * NW)), kw = key0 + 32 * wave;
  bf16x8 kf[kI], vf[kVLds ? 1 : kI];
  const int shift = sq.n - sq.m;
  const int first = a.causal ? kw + (lane & 31) - shift : 0;  // queries from here on see this lane's key
  {
    const int key = kw + (lane & 31);
    const bool live = key < sq.n;
    const int64_t token = sq.k0 + (live ? key : 0);
#pragma unroll
    for (int i = 0; i < kI; ++i) {
      kf[i] = attn_own(a.k + token * a.ks + kv * a.kh, i, h, a.hd, live);
      if constexpr (!kVLds) vf[i] = attn_own(a.v + token * a.vs + kv * a.vh, i, h, a.hd, live);
    }
  }
  // from wall on all the wave's keys; none before qbeg sees one of the workgroup's
  const int wall = a.causal ? kw + 31 - shift : 0, wany = a.causal ? kw - shift : 0;
  int qbeg = a.causal ? key0 - shift : 0;
  qbeg = qbeg < 0 ? 0 : qbeg / QT * QT;

  f32x16 dk[kFb], dv[kFb];
  if (again) attn_barrier();
  const INFCL_LDS char* vown = lds + 4 * Tile::kBytes + wave * 32 * Tile::kRow;
  // this part's tiles [c0, c1): tile c is head c % group of queries qbeg + QT (per - 1 - c / group) on
  const int per = sq.m > qbeg ? (sq.m - qbeg + QT - 1) / QT : 0;
  int64_t c0 = 0, c1 = (int64_t)per * a.group;
  if (SPLIT) {
    const int64_t share = (c1 + parts - 1) / parts;
    c0 = share * part < c1 ? share * part : c1;
    c1 = c0 + share < c1 ? c0 + share : c1;
  }
  if constexpr (kVLds) {
    uint32_t off[Own::kVar];
    Own::offsets(off, wave, lane, (uint32_t)(a.vs * 2), a.hd);
    if (c0 < c1)  // (the first tile's barrier waits for them)
      Own::issue(a.v + (sq.k0 + key0) * a.vs + kv * a.vh, sq.n - key0, (uint32_t)(a.vs * 2), a.hd,
                 lds + 4 * Tile::kBytes, off, wave);
  }
#pragma unroll
  for (int fb = 0; fb < kFb; ++fb) dk[fb] = f32x16_zero(), dv[fb] = f32x16_zero();
  // the lanes fetch a tile's 32 pairs a tile ahead
  const float* row = w.stat + sq.q0 * 2;
  float ahead = 0.f;
  int g = (int)(c0 % a.group), i0 = qbeg + QT * (per - 1 - (int)(c0 / a.group));  // the tile in hand, then the next
  auto issue = [&](int b) {
    const int head = kv * a.group + g;
    INFCL_LDS char* to = lds + b * 2 * Tile::kBytes;
    Tile::issue(a.q + (sq.q0 + i0) * a.qs + head * a.qh, sq.m - i0, qst, a.hd, to, qoff, wave);
    Tile::issue(w.dout + (sq.q0 + i0) * w.dos + head * w.doh, sq.m - i0, dst, a.hd, to + Tile::kBytes, doff, wave);
    ahead = row[((int64_t)head * w.trow + i0) * 2 + lane];
  };
  if (c0 < c1) issue(0);
  // the first `cut` tiles of queries are seen by some of the wave's keys and not by others
  int cut = a.causal && wall > qbeg ? (wall - qbeg + QT - 1) / QT : 0;
  cut = cut < per ? cut : per;
  const int wend = CUT ? qbeg + cut * QT : wany;
  int buf = 0;
  for (int64_t c = c0; c < c1; ++c, buf ^= 1) {
    const int i1 = i0;
    const bool none = i1 + QT <= wend || kw >= sq.n;  // (no query of the tile sees a key of this wave)
    stat[lane] = ahead;
    if (++g == a.group) g = 0, i0 -= QT;
    attn_barrier();
    if (c + 1 < c1) issue(buf ^ 1);
    if (none) continue;
    const INFCL_LDS char* qt = lds + buf * 2 * Tile::kBytes;
    const INFCL_LDS char* dt = qt + Tile::kBytes;
    f32x16 p = f32x16_zero(), dp = f32x16_zero();
#pragma unroll
    for (int i = 0; i < kI; ++i) {
      p = mfma16<F16>(attn_row(qt + ln.row[i]), kf[i], p);
      dp = mfma16<F16>(attn_row(dt + ln.row[i]), kVLds ? attn_row(vown + ln.row[i]) : vf[kVLds ? 0 : i], dp);
    }
#pragma unroll
    for (int x4 = 0; x4 < 4; ++x4) {
      const f32x4 lo = *(const INFCL_LDS f32x4*)(stat + 2 * attn_reg_row(4 * x4, h));
      const f32x4 hi = *(const INFCL_LDS f32x4*)(stat + 2 * attn_reg_row(4 * x4, h) + 4);
      const float L[4] = {lo[0], lo[2], hi[0], hi[2]}, D[4] = {lo[1], lo[3], hi[1], hi[3]};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int x = 4 * x4 + e;
        p[x] = exp2_hw(fmaf(p[x], a.sl2, -L[e]));
        dp[x] = p[x] * (dp[x] - D[e]);
      }
    }
    if (i1 < wall || i1 + QT > sq.m) {
      const int lo = attn_opaque(first - i1 - 4 * h), hi = attn_opaque(sq.m - i1 - 4 * h);
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const bool seen = attn_reg_row(x, 0) >= lo && attn_reg_row(x, 0) < hi;
        p[x] = seen ? p[x] : 0.f;
        dp[x] = seen ? dp[x] : 0.f;
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const bf16x8 pw = attn_pack<F16>(p, u), ds = attn_pack<F16>(dp, u);
      const int ro = 16 * u * Tile::kRow;
#pragma unroll
      for (int fb = 0; fb < kFb; ++fb) {
        dv[fb] = mfma16<F16>(attn_tr(dt + ro + ln.tr[0][fb], dt + ro + ln.tr[1][fb]), pw, dv[fb]);
        dk[fb] = mfma16<F16>(attn_tr(qt + ro + ln.tr[0][fb], qt + ro + ln.tr[1][fb]), ds, dk[fb]);
      }
    }
  }
  int own_lane = threadIdx.x & 63;
  asm volatile("" : "+v"(own_lane));  // (addresses made here, not kept through the sweep)
  const int own_key = kw + (own_lane & 31);
  const bool mine = own_key < sq.n;
  const int64_t at = sq.k0 + own_key;
  if (CUT && mine) {
    const int64_t from = (int64_t)(per - cut) * a.group;
    const int see = own_key - shift, oh = own_lane >> 5;
    const uint16_t *kr = a.k + at * a.ks + kv * a.kh, *vr = a.v + at * a.vs + kv * a.vh;
#pragma unroll 1
    for (int64_t c = c0 > from ? c0 : from; c < c1; ++c) {
      const int head = kv * a.group + (int)(c % a.group);
      const int beg = qbeg + QT * (per - 1 - (int)(c / a.group)), end = beg + QT < sq.m ? beg + QT : sq.m;
#pragma unroll 1
      for (int i = beg > see ? beg : see; i < end; ++i) {
        const uint16_t* qr = a.q + (sq.q0 + i) * a.qs + head * a.qh;
        const uint16_t* dr = w.dout + (sq.q0 + i) * w.dos + head * w.doh;
        const float* st = w.stat + ((int64_t)head * w.trow + sq.q0 + i) * 2;
        const float p = exp2_hw(fmaf(attn_dot<F16>(kr, qr, oh, a.hd), a.sl2, -st[0]));
        attn_axpy<F16>(dk, p * (attn_dot<F16>(vr, dr, oh, a.hd) - st[1]), qr, oh, a.hd);
        attn_axpy<F16>(dv, p, dr, oh, a.hd);
      }
    }
  }
  const bool bad = !CUT && a.causal && wave_any(mine && (attn_bad(dk) || attn_bad(dv)));
  if (!mine) return bad;
  if constexpr (SPLIT) {
    const int64_t rows = a.tk * a.kvh;
    float* pk = w.part + ((int64_t)part * 2 * rows + at * a.kvh + kv) * a.hd;
#pragma unroll
    for (int fb = 0; fb < kFb; ++fb)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int d = 32 * fb + 8 * j + 4 * (own_lane >> 5);
        if (d >= a.hd) continue;
        *(f32x4*)(pk + d) = f32x4{dk[fb][4 * j], dk[fb][4 * j + 1], dk[fb][4 * j + 2], dk[fb][4 * j + 3]};
        *(f32x4*)(pk + rows * a.hd + d) = f32x4{dv[fb][4 * j], dv[fb][4 * j + 1], dv[fb][4 * j + 2], dv[fb][4 * j + 3]};
      }
  } else {
    attn_store<F16>(w.dk + at * w.dks + kv * w.dkh, dk, a.scale, own_lane >> 5, a.hd);
    attn_store<F16>(w.dv + at * w.dvs + kv * w.dvh, dv, 1.f, own_lane >> 5, a.hd);
  }
  return bad;
}

template <int DP, int NW, bool F16, bool SPLIT>
__global__ void __launch_bounds__(64 * NW, 2) attn_dkv_kernel(AttnArgs a, AttnGrads w, int tiles, int parts) {
  __shared__ __attribute__((aligned(1024))) char lds_[4 * AttnTile<DP, NW, 32>::kBytes +
                                                      (attn_own_in_lds(DP, NW) ? AttnTile<DP, NW, 32 * NW>::kBytes : 0)];
  __shared__ __attribute__((aligned(16))) float stat_[NW][64];  // a tile's pairs of lse log2(e) and D
  __shared__ int flags[NW];
  INFCL_LDS char* lds = (INFCL_LDS char*)lds_;
  const int wave = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  INFCL_LDS float* stat = (INFCL_LDS float*)stat_[wave];
  const uint32_t groups = (uint32_t)(a.nseq + 1) * (uint32_t)a.kvh;
  // (longest sweeps first: the first keys' parts)
  const AttnPlace where = attn_place(blockIdx.x, (uint32_t)(tiles * parts), groups);
  const int t0 = (int)where.t / (SPLIT ? parts : 1), part = SPLIT ? (int)where.t % parts : 0;
  const int z = (int)(where.g / (uint32_t)a.kvh), kv = (int)(where.g % (uint32_t)a.kvh);
  AttnSeq sq = attn_seq(a, z);
  if (z == a.nseq) sq.m = 0;
  if ((int64_t)t0 * (32 * NW) >= sq.n) return;

  bool bad = false;
  for (int64_t t = t0; t * (32 * NW) < sq.n; t += tiles)
    bad |= attn_dkv_tile<DP, NW, F16, SPLIT, false>(a, w, sq, kv, parts, part, t, lds, stat, t != t0);
  if (!a.causal) return;
  bool odd = false;  // queries and dout of the tiles that a mask cuts
  if (bad) {
    for (int64_t t = t0; t * (32 * NW) + 32 * wave < sq.n; t += tiles) {
      int lo = (int)t * (32 * NW) + 32 * wave - (sq.n - sq.m), hi = lo + 31 < sq.m ? lo + 31 : sq.m;
      lo = lo < 32 ? 0 : lo - 31;  // (the tile of the first query that sees one of the wave's keys)
      for (int g = 0; g < a.group; ++g) {
        const int head = kv * a.group + g;
        odd |= attn_odd<F16>(a.q + (sq.q0 + lo) * a.qs + head * a.qh, hi - lo, a.qs, a.hd, threadIdx.x & 63) ||
               attn_odd<F16>(w.dout + (sq.q0 + lo) * w.dos + head * w.doh, hi - lo, w.dos, a.hd, threadIdx.x & 63);
      }
    }
  }
  if (!attn_vote<NW>(odd, (INFCL_LDS int*)flags, wave)) return;
  for (int64_t t = t0; t * (32 * NW) < sq.n; t += tiles)
    attn_dkv_tile<DP, NW, F16, SPLIT, true>(a, w, sq, kv, parts, part, t, lds, stat, true);
}

// The parts' dk and dv, in order.  A wave takes 8 rows of one sequence's key head,
// 16 lanes to a row.
template <bool F16>
__global__ void __launch_bounds__(256) attn_dkv_join(AttnArgs a, AttnGrads w, int tiles, int parts) {
  const uint32_t groups = (uint32_t)(a.nseq + 1) * (uint32_t)a.kvh;
  const uint32_t gz = blockIdx.x % groups;
  const int z = (int)(gz / (uint32_t)a.kvh), kv = (int)(gz % (uint32_t)a.kvh);
  AttnSeq sq = attn_seq(a, z);
  if (z == a.nseq) sq.m = 0;
  const int lane = threadIdx.x & 63, d = 8 * (lane & 15);
  const int64_t step = a.tk * a.kvh * a.hd;  // from dk to dv of a part, and on to the next part's dk
  for (int64_t key0 = (int64_t)(blockIdx.x / groups) * 32 + (threadIdx.x >> 6) * 8; key0 < sq.n;
       key0 += (int64_t)tiles * 32) {
#pragma unroll
    for (int r = lane >> 4; r < 8; r += 4) {
      const int64_t token = sq.k0 + key0 + r;
      if (key0 + r >= sq.n || d >= a.hd) continue;
      const float* src = w.part + (token * a.kvh + kv) * a.hd + d;
      float ak[8] = {0, 0, 0, 0, 0, 0, 0, 0}, av[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll 4
      for (int p = 0; p < parts; ++p) {
        const f32x4 *x = (const f32x4*)(src + 2 * p * step), *y = (const f32x4*)(src + (2 * p + 1) * step);
        const f32x4 x0 = x[0], x1 = x[1], y0 = y[0], y1 = y[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) ak[e] += x0[e], ak[4 + e] += x1[e], av[e] += y0[e], av[4 + e] += y1[e];
      }
      attn_store8<F16>(w.dk + token * w.dks + kv * w.dkh + d, ak, a.scale);
      attn_store8<F16>(w.dv + token * w.dvs + kv * w.dvh + d, av, 1.f);
    }
  }
}

template <int DP, bool F16, int NW, int KT>
void launch_both(const AttnArgs& a, const AttnGrads& w, const AttnBwdPlan& p, int64_t max_q, int64_t max_k,
                 hipStream_t st) {
  const int64_t groups = attn_groups(a);
  const int64_t tq = attn_at_once(((max_q < 1 ? 1 : max_q) * a.group + 32 * NW - 1) / (32 * NW), groups * p.parts_q, 64 * NW);
  const int64_t tk = attn_at_once(((max_k < 1 ? 1 : max_k) + 32 * NW - 1) / (32 * NW), groups * p.parts, 64 * NW);
  const dim3 qgrid((unsigned)(tq * groups * p.parts_q));
  if (p.parts_q == 1) {
    hipLaunchKernelGGL((attn_dq_kernel<DP, NW, KT, F16, false>), qgrid, dim3(64 * NW), 0, st,
                       AttnBwdArgs{a, w, (int)tq, 1});
  } else if constexpr (NW > 1) {
    const int64_t tj = attn_at_once(NW * tq, groups, 256);
    hipLaunchKernelGGL((attn_dq_kernel<DP, NW, KT, F16, true>), qgrid, dim3(64 * NW), 0, st,
                       AttnBwdArgs{a, w, (int)tq, p.parts_q});
    hipLaunchKernelGGL((attn_dq_join<F16>), dim3((unsigned)(tj * groups)), dim3(256), 0, st, a, w, (int)tj, p.parts_q);
  }
  const dim3 grid((unsigned)(tk * groups * p.parts));
  if (p.parts == 1) {
    hipLaunchKernelGGL((attn_dkv_kernel<DP, NW, F16, false>), grid, dim3(64 * NW), 0, st, a, w, (int)tk, 1);
  } else if constexpr (NW > 1) {
    const int64_t tj = attn_at_once(4 * tk, groups, 256);
    hipLaunchKernelGGL((attn_dkv_kernel<DP, NW, F16, true>), grid, dim3(64 * NW), 0, st, a, w, (int)tk, p.parts);
    hipLaunchKernelGGL((attn_dkv_join<F16>), dim3((unsigned)(tj * groups)), dim3(256), 0, st, a, w, (int)tj, p.parts);
  }
}

template <bool F16>
void launch_t(const AttnArgs& a, const AttnGrads& w, const AttnBwdPlan& p, int64_t max_q, int64_t max_k,
              hipStream_t st) {
  if (a.hd <= 64) {
    if (p.few)
      launch_both<64, F16, 1, 32>(a, w, p, max_q, max_k, st);
    else
      launch_both<64, F16, 4, 64>(a, w, p, max_q, max_k, st);
  } else {
    if (p.few)
      launch_both<128, F16, 1, 32>(a, w, p, max_q, max_k, st);
    else
      launch_both<128, F16, 4, 32>(a, w, p, max_q, max_k, st);
  }
}

}  // namespace

// As in the forward, short sequences run one wave to a workgroup.  Otherwise the
// sweeps are cut into parts where there are fewer workgroups than it takes to
// fill the chip evenly: their lengths differ (with causal masks from none to all
// of the other side), and one long sweep would be waited for.
AttnBwdPlan attn_bwd_plan(const AttnArgs& a, int64_t max_q, int64_t max_k) {
  AttnBwdPlan p;
  p.few = (max_q * a.group <= 128 && max_k <= 128) || attn_groups(a) > kAttnItems / 256;  // (as in the forward)
  p.parts = p.parts_q = 1;
  if (!p.few) {
    const int64_t tiles = max_k > 0 ? attn_tiles(a.nseq, (max_k + 127) / 128, a.tk / 128) * a.kvh : 0;
    p.parts = attn_parts(tiles, kBwdGroups, (max_q + 31) / 32 * a.group / 16);  // at least 16 tiles a part
    const int64_t rows = (max_q * a.group + 127) / 128;
    p.parts_q = attn_parts(attn_tiles(a.nseq, rows, a.tq * a.group / 128) * a.kvh, kBwdRowGroups, max_k / 256);
  }
  const size_t row = ((size_t)a.tq + 32 + 63) / 64 * 64;
  size_t off = 0;
  p.trow = (int64_t)row;
  p.stat = off, off = (off + 2 * row * (size_t)a.heads * sizeof(float) + 255) & ~(size_t)255;
  p.part = off;
  if (p.parts > 1) off += 2 * (size_t)p.parts * (size_t)a.tk * (size_t)a.kvh * (size_t)a.hd * sizeof(float);
  p.part_q = p.part;  // (joined before the other sweep begins)
  if (p.parts_q > 1) {
    const size_t end = p.part + (size_t)p.parts_q * (size_t)a.tq * (size_t)a.heads * (size_t)a.hd * sizeof(float);
    off = off > end ? off : end;
  }
  p.total = (off + 255) & ~(size_t)255;
  return p;
}

int launch_attn_bwd(const AttnArgs& a, const AttnBwdPlan& p, int dtype, int64_t max_q, int64_t max_k,
                    const uint16_t* out, int64_t os, int64_t oh, const float* lse, const uint16_t* dout, int64_t dos,
                    int64_t doh, uint16_t* dq, int64_t dqs, int64_t dqh, uint16_t* dk, int64_t dks, int64_t dkh,
                    uint16_t* dv, int64_t dvs, int64_t dvh, char* ws, hipStream_t st) {
  AttnGrads w;
  w.out = out, w.os = os, w.oh = oh, w.lse = lse, w.dout = dout, w.dos = dos, w.doh = doh;
  w.dq = dq, w.dqs = dqs, w.dqh = dqh, w.dk = dk, w.dks = dks, w.dkh = dkh, w.dv = dv, w.dvs = dvs, w.dvh = dvh;
  w.trow = p.trow;
  w.stat = (float*)(ws + p.stat);
  w.part = (float*)(ws + p.part);
  w.part_q = (float*)(ws + p.part_q);
  if (dtype == INFCL_F16)
    launch_t<true>(a, w, p, max_q, max_k, st);
  else
    launch_t<false>(a, w, p, max_q, max_k, st);
  return hipGetLastError() == hipSuccess ? INFCL_OK : INFCL_ERR_HIP;
}

}  // namespace infcl

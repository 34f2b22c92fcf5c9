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
// D comes from o as stored, except where all keys of a sequence are in one
// tile: there it is the sum of p dp in the registers, which no rounding of o
// touches (with few keys o is not small beside dp, and its rounding would show).
#include "attn.hpp"

namespace infcl {
namespace {

struct AttnGrads {
  const uint16_t *out, *dout;
  int64_t os, oh, dos, doh;
  const float* lse;
  float *lse2, *dlt;  // [heads][trow]: 64 entries past the tokens may be read
  int64_t trow;
  uint16_t *dq, *dk, *dv;
  int64_t dqs, dqh, dks, dkh, dvs, dvh;
};

// Owns rows (query, head of the group); sweeps the keys they see.
template <int DP, int NW, int KT, bool F16>
__global__ void __launch_bounds__(64 * NW) attn_dq_kernel(AttnArgs a, AttnGrads w, int tiles) {
  constexpr int kFb = DP / 32, kI = DP / 16, kKb = KT / 32;
  typedef AttnTile<DP, NW, KT> Tile;
  __shared__ __attribute__((aligned(1024))) char lds_[4 * Tile::kBytes];
  __shared__ int redo;
  INFCL_LDS char* lds = (INFCL_LDS char*)lds_;
  const int wave = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int h = lane >> 5;
  const uint32_t groups = (uint32_t)(a.nseq + 1) * (uint32_t)a.kvh;
  const int t0 = tiles - 1 - (int)(blockIdx.x / groups);
  const uint32_t gz = blockIdx.x % groups;
  const int z = (int)(gz / (uint32_t)a.kvh), kv = (int)(gz % (uint32_t)a.kvh);
  AttnSeq sq = attn_seq(a, z);
  if (z == a.nseq) sq.n = 0;
  const int64_t rows64 = (int64_t)sq.m * a.group;
  const uint32_t rows = rows64 > 0x7FFFFFFF ? 0x7FFFFFFFu : (uint32_t)rows64;
  if ((int64_t)t0 * (32 * NW) >= rows) return;

  AttnLanes<DP> ln;
  ln.init(lane);
  const uint32_t kst = (uint32_t)(a.ks * 2), vst = (uint32_t)(a.vs * 2);
  uint32_t koff[Tile::kVar], voff[Tile::kVar];
  Tile::offsets(koff, wave, lane, kst, a.hd);
  Tile::offsets(voff, wave, lane, vst, a.hd);
  const uint16_t* kb = a.k + sq.k0 * a.ks + kv * a.kh;
  const uint16_t* vb = a.v + sq.k0 * a.vs + kv * a.vh;

  for (uint32_t t = (uint32_t)t0; t * (uint64_t)(32 * NW) < rows; t += (uint32_t)tiles) {
    const uint32_t r = t * (32 * NW) + wave * 32 + (lane & 31);
    const bool live = r < rows;
    const int pos = live ? (int)(r / (uint32_t)a.group) : 0, g = live ? (int)(r % (uint32_t)a.group) : 0;
    const int head = kv * a.group + g;
    const int64_t token = sq.q0 + pos;
    bf16x8 qf[kI], df[kI];
    float D = 0.f;
#pragma unroll
    for (int i = 0; i < kI; ++i) {
      qf[i] = attn_own(a.q + token * a.qs + head * a.qh, i, h, a.hd, live);
      df[i] = attn_own(w.dout + token * w.dos + head * w.doh, i, h, a.hd, live);
      const bf16x8 of = attn_own(w.out + token * w.os + head * w.oh, i, h, a.hd, live);
#pragma unroll
      for (int e = 0; e < 8; ++e) D = fmaf(from16<F16>(df[i][e]), from16<F16>(of[e]), D);
    }
    D = attn_sum2(D);
    float lse2 = 0.f;
    if (live) lse2 = w.lse[(int64_t)head * a.tq + token] * kLog2e;
    if (lse2 == -__builtin_inff()) lse2 = 0.f, D = 0.f;

    const int shift = sq.n - sq.m + 1;
    int lim = a.causal ? pos + shift : sq.n;
    lim = lim < 0 ? 0 : lim;
    if (!live) lim = 0;
    const uint32_t rl = t * (uint64_t)(32 * NW) + 32 * NW < rows ? t * (32 * NW) + 32 * NW - 1 : rows - 1;
    int kend = a.causal ? (int)(rl / (uint32_t)a.group) + shift : sq.n;
    kend = kend < sq.n ? kend : sq.n;
    const uint32_t rw = t * (32 * NW) + wave * 32;
    const uint32_t rv = rw + 31 < rows ? rw + 31 : rows - 1;
    const int wmin = rw >= rows ? 0 : a.causal ? (int)(rw / (uint32_t)a.group) + shift : sq.n;
    const int wmax = rw >= rows ? 0 : a.causal ? (int)(rv / (uint32_t)a.group) + shift : sq.n;

    f32x16 acc[kFb];
    attn_barrier();
    if (threadIdx.x == 0) redo = 0;
    for (int exact = 0;; exact = 1) {
#pragma unroll
      for (int fb = 0; fb < kFb; ++fb) acc[fb] = f32x16_zero();
      if (0 < kend) {
        Tile::issue(kb, sq.n, kst, a.hd, lds, koff, wave);
        Tile::issue(vb, sq.n, vst, a.hd, lds + Tile::kBytes, voff, wave);
      }
      int buf = 0;
      for (int k = 0; k < kend; k += KT, buf ^= 1) {
        attn_barrier();
        if (k + KT < kend) {
          INFCL_LDS char* nx = lds + (buf ^ 1) * 2 * Tile::kBytes;
          Tile::issue(kb + (int64_t)(k + KT) * a.ks, sq.n - k - KT, kst, a.hd, nx, koff, wave);
          Tile::issue(vb + (int64_t)(k + KT) * a.vs, sq.n - k - KT, vst, a.hd, nx + Tile::kBytes, voff, wave);
        }
        if (k >= wmax) continue;
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
        const bool masked = k + KT > wmin;
#pragma unroll
        for (int b = 0; b < kKb; ++b)
#pragma unroll
          for (int x = 0; x < 16; ++x) {
            p[b][x] = exp2_hw(fmaf(p[b][x], a.sl2, -lse2));
            if (masked && k + 32 * b + attn_reg_row(x, h) >= lim) p[b][x] = 0.f, dp[b][x] = 0.f;
          }
        if (sq.n <= KT) {
          float s = 0.f;
#pragma unroll
          for (int b = 0; b < kKb; ++b)
#pragma unroll
            for (int x = 0; x < 16; ++x) s = fmaf(p[b][x], dp[b][x], s);
          D = attn_sum2(s);
        }
        if (exact && masked) {
          for (int j = 0; j < KT && k + j < kend; ++j) {
            const float pj = exp2_hw(fmaf(attn_dot<DP, F16>(qf, kt, j, h), a.sl2, -lse2));
            const float ds = pj * (attn_dot<DP, F16>(df, vt, j, h) - D);
            attn_axpy<DP, F16>(acc, ds, k + j < lim, kt, j, h);
          }
          continue;
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
      if (!a.causal || exact) break;
      attn_barrier();
      if (wave_any(attn_bad(acc)) && lane == 0) redo = 1;
      attn_barrier();
      if (!redo) break;
    }
    if (!live) continue;
    attn_store<F16>(w.dq + token * w.dqs + head * w.dqh, acc, a.scale, h, a.hd);
    if (h == 0) {
      w.lse2[(int64_t)head * w.trow + token] = lse2;
      w.dlt[(int64_t)head * w.trow + token] = D;
    }
  }
}

// Owns keys; sweeps the queries that see them, one head of the group after
// another.
template <int DP, int NW, bool F16>
__global__ void __launch_bounds__(64 * NW) attn_dkv_kernel(AttnArgs a, AttnGrads w, int tiles) {
  constexpr int kFb = DP / 32, kI = DP / 16, QT = 32;
  typedef AttnTile<DP, NW, QT> Tile;
  __shared__ __attribute__((aligned(1024))) char lds_[4 * Tile::kBytes];
  __shared__ int redo;
  INFCL_LDS char* lds = (INFCL_LDS char*)lds_;
  const int wave = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int h = lane >> 5;
  const uint32_t groups = (uint32_t)(a.nseq + 1) * (uint32_t)a.kvh;
  const int t0 = (int)(blockIdx.x / groups);
  const uint32_t gz = blockIdx.x % groups;
  const int z = (int)(gz / (uint32_t)a.kvh), kv = (int)(gz % (uint32_t)a.kvh);
  AttnSeq sq = attn_seq(a, z);
  if (z == a.nseq) sq.m = 0;
  if ((int64_t)t0 * (32 * NW) >= sq.n) return;

  AttnLanes<DP> ln;
  ln.init(lane);
  const uint32_t qst = (uint32_t)(a.qs * 2), dst = (uint32_t)(w.dos * 2);
  uint32_t qoff[Tile::kVar], doff[Tile::kVar];
  Tile::offsets(qoff, wave, lane, qst, a.hd);
  Tile::offsets(doff, wave, lane, dst, a.hd);

  for (int64_t t = t0; t * (32 * NW) < sq.n; t += tiles) {
    const int key0 = (int)(t * (32 * NW)), kw = key0 + 32 * wave, key = kw + (lane & 31);
    const bool live = key < sq.n;
    const int64_t token = sq.k0 + key;
    bf16x8 kf[kI], vf[kI];
#pragma unroll
    for (int i = 0; i < kI; ++i) {
      kf[i] = attn_own(a.k + (live ? token * a.ks : 0) + kv * a.kh, i, h, a.hd, live);
      vf[i] = attn_own(a.v + (live ? token * a.vs : 0) + kv * a.vh, i, h, a.hd, live);
    }
    // queries from `first` on see this lane's key, from wall on all the wave's;
    // none before qbeg sees one of the workgroup's
    const int shift = sq.n - sq.m;
    const int first = a.causal ? key - shift : 0;
    const int wall = a.causal ? kw + 31 - shift : 0, wany = a.causal ? kw - shift : 0;
    int qbeg = a.causal ? key0 - shift : 0;
    qbeg = qbeg < 0 ? 0 : qbeg / QT * QT;

    f32x16 dk[kFb], dv[kFb];
    attn_barrier();
    if (threadIdx.x == 0) redo = 0;
    for (int exact = 0;; exact = 1) {
#pragma unroll
      for (int fb = 0; fb < kFb; ++fb) dk[fb] = f32x16_zero(), dv[fb] = f32x16_zero();
      // tiles of all heads of the group, as one sequence
      const int per = sq.m > qbeg ? (sq.m - qbeg + QT - 1) / QT : 0;
      const int64_t count = (int64_t)per * a.group;
      auto issue = [&](int g, int i, int b) {
        const int head = kv * a.group + g;
        INFCL_LDS char* to = lds + b * 2 * Tile::kBytes;
        Tile::issue(a.q + (sq.q0 + i) * a.qs + head * a.qh, sq.m - i, qst, a.hd, to, qoff, wave);
        Tile::issue(w.dout + (sq.q0 + i) * w.dos + head * w.doh, sq.m - i, dst, a.hd, to + Tile::kBytes, doff, wave);
      };
      if (count) issue(0, qbeg, 0);
      int g = 0, i0 = qbeg, buf = 0;
      for (int64_t c = 0; c < count; ++c, buf ^= 1) {
        int gn = g, in = i0 + QT;
        if (in >= sq.m) ++gn, in = qbeg;
        attn_barrier();
        if (c + 1 < count) issue(gn, in, buf ^ 1);
        const int head = kv * a.group + g, i1 = i0;
        g = gn, i0 = in;
        if (i1 + QT <= wany || kw >= sq.n) continue;  // (no query of the tile sees a key of this wave)
        const float* pl = w.lse2 + (int64_t)head * w.trow + sq.q0 + i1;
        const float* pd = w.dlt + (int64_t)head * w.trow + sq.q0 + i1;
        const INFCL_LDS char* qt = lds + buf * 2 * Tile::kBytes;
        const INFCL_LDS char* dt = qt + Tile::kBytes;
        f32x16 p = f32x16_zero(), dp = f32x16_zero(), L, Dv;
#pragma unroll
        for (int x = 0; x < 16; ++x) L[x] = pl[attn_reg_row(x, h)], Dv[x] = pd[attn_reg_row(x, h)];
#pragma unroll
        for (int i = 0; i < kI; ++i) {
          p = mfma16<F16>(attn_row(qt + ln.row[i]), kf[i], p);
          dp = mfma16<F16>(attn_row(dt + ln.row[i]), vf[i], dp);
        }
        const bool masked = i1 < wall || i1 + QT > sq.m;
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          p[x] = exp2_hw(fmaf(p[x], a.sl2, -L[x]));
          dp[x] -= Dv[x];
          const int i = i1 + attn_reg_row(x, h);
          if (masked && (i < first || i >= sq.m)) p[x] = 0.f, dp[x] = 0.f;
          dp[x] *= p[x];
        }
        if (exact && masked) {
          for (int j = 0; j < QT && i1 + j < sq.m; ++j) {
            const float pj = exp2_hw(fmaf(attn_dot<DP, F16>(kf, qt, j, h), a.sl2, -pl[j]));
            const float ds = pj * (attn_dot<DP, F16>(vf, dt, j, h) - pd[j]);
            attn_axpy<DP, F16>(dv, pj, i1 + j >= first, dt, j, h);
            attn_axpy<DP, F16>(dk, ds, i1 + j >= first, qt, j, h);
          }
          continue;
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
      if (!a.causal || exact) break;
      attn_barrier();
      if ((wave_any(attn_bad(dk)) || wave_any(attn_bad(dv))) && lane == 0) redo = 1;
      attn_barrier();
      if (!redo) break;
    }
    if (!live) continue;
    attn_store<F16>(w.dk + token * w.dks + kv * w.dkh, dk, a.scale, h, a.hd);
    attn_store<F16>(w.dv + token * w.dvs + kv * w.dvh, dv, 1.f, h, a.hd);
  }
}

template <int DP, bool F16, int NW, int KT>
void launch_both(const AttnArgs& a, const AttnGrads& w, int64_t max_q, int64_t max_k, hipStream_t st) {
  const int64_t groups = (int64_t)(a.nseq + 1) * a.kvh, own = 32 * NW;
  const int64_t tq = ((max_q < 1 ? 1 : max_q) * a.group + own - 1) / own, tk = ((max_k < 1 ? 1 : max_k) + own - 1) / own;
  hipLaunchKernelGGL((attn_dq_kernel<DP, NW, KT, F16>), dim3((unsigned)(tq * groups)), dim3(64 * NW), 0, st, a, w,
                     (int)tq);
  hipLaunchKernelGGL((attn_dkv_kernel<DP, NW, F16>), dim3((unsigned)(tk * groups)), dim3(64 * NW), 0, st, a, w,
                     (int)tk);
}

template <bool F16>
void launch_t(const AttnArgs& a, const AttnGrads& w, int64_t max_q, int64_t max_k, hipStream_t st) {
  // as in the forward: short sequences run one wave to a workgroup
  const bool few = max_q * a.group <= 128 && max_k <= 128;
  if (a.hd <= 64) {
    if (few)
      launch_both<64, F16, 1, 32>(a, w, max_q, max_k, st);
    else
      launch_both<64, F16, 4, 64>(a, w, max_q, max_k, st);
  } else {
    if (few)
      launch_both<128, F16, 1, 32>(a, w, max_q, max_k, st);
    else
      launch_both<128, F16, 4, 32>(a, w, max_q, max_k, st);
  }
}

}  // namespace

size_t attn_bwd_bytes(const AttnArgs& a) {
  const size_t row = ((size_t)a.tq + 64 + 63) / 64 * 64;
  return 2 * row * (size_t)a.heads * sizeof(float) + 256;
}

int launch_attn_bwd(const AttnArgs& a, int dtype, int64_t max_q, int64_t max_k, const uint16_t* out, int64_t os,
                    int64_t oh, const float* lse, const uint16_t* dout, int64_t dos, int64_t doh, uint16_t* dq,
                    int64_t dqs, int64_t dqh, uint16_t* dk, int64_t dks, int64_t dkh, uint16_t* dv, int64_t dvs,
                    int64_t dvh, char* ws, hipStream_t st) {
  AttnGrads w;
  w.out = out, w.os = os, w.oh = oh, w.lse = lse, w.dout = dout, w.dos = dos, w.doh = doh;
  w.dq = dq, w.dqs = dqs, w.dqh = dqh, w.dk = dk, w.dks = dks, w.dkh = dkh, w.dv = dv, w.dvs = dvs, w.dvh = dvh;
  w.trow = (int64_t)(((size_t)a.tq + 64 + 63) / 64 * 64);
  w.lse2 = (float*)ws;
  w.dlt = w.lse2 + w.trow * a.heads;
  if (dtype == INFCL_F16)
    launch_t<true>(a, w, max_q, max_k, st);
  else
    launch_t<false>(a, w, max_q, max_k, st);
  return hipGetLastError() == hipSuccess ? INFCL_OK : INFCL_ERR_HIP;
}

}  // namespace infcl

// A block's output normed, dropped out, gated and added to the residual rows, and
// the norm of the sum:
//   t = gate D(N(y) post_w + post_b),  h = alpha x + t,  z = N(h) pre_w + pre_b
// and all gradients in one pass over x, y, dh and dz.
//
// With v = N(y), r1 its factor, k = N(h), r2 its factor, D = 0 or 1 / (1 - p), and for
// a norm's rows <.> the mean over features (second terms: layer norms only):
//   g = dz pre_w,  e = dh + r2 (g - k <g k> - <g>)
//   dx = alpha e,  s = e gate D,  q = s post_w,  dy = r1 (q - v <q v> - <q>)
//   dpre_w = sum dz k, dpre_b = sum dz, dgate = sum e D (v post_w + post_b),
//   dpost_w = sum s v, dpost_b = sum s
//
// A row is 8 features in each of up to 1024 lanes: a group of 8 to 64 lanes of one
// wave, or several waves.  It stays in registers from its load to its last use, so the
// variance is that of the centred row and the backward reads each input once; h is
// taken again from x and y there (as many bytes as reading it back, and not rounded).
// What a lane adds up for its features over all its rows are 32 registers at most (40 with gate
// and biases; some of them in LDS where rows take several waves), then
// one row of partial sums for each workgroup, joined in order by a second launch.
// Bound by the rows' bytes without gate, first norm and dropout (17408 x 512: 13 us forward and 21
// backward for 71 and 107 MB; 50001 x 1160: 77 and 138 for 464 and 696 MB, part of them from the
// last-level cache).  With everything the vector unit has about as much to do, some 400 instructions
// for 8 features: 50001 x 1160 108 to 116 and 154 to 171 us, 20001 x 2568 117 and 134, of 82 and 122 at a
// copy's 5.04 TB/s.  8 rows of 4096 forward: 4.2 to 4.8 us.
#include "block.hpp"

namespace infcl {
namespace {

struct NormArgs {
  const void *x, *y, *gate, *post_w, *post_b, *pre_w, *pre_b, *dh, *dz;
  void *h, *z, *dx, *dy;
  float4* stats;
  float* part;  // [workgroups][sums][d]
  int64_t n, xs, ys, dhs, dzs;
  int c, ls;  // chunks of a row; log2 of the lanes of a row within a wave
  int rms, wf32;
  int want_gate, want_post, want_post_b, want_pre, want_pre_b;  // sums that are taken, in this order
  float eps, alpha, by_d;
  Drop drop;
};

// Sums over a row of K values of each lane: over its group of lanes, or over all waves
// of the workgroup (WIDE) through one of two buffers in turn, so that one barrier
// does for each: 16 lanes read the 16 waves' sums (zeros of waves that are not there) and
// add them up as they do their own.
template <bool WIDE, int K>
__device__ __forceinline__ void row_sums(float (&s)[K], int ls, float (*buf)[16][2], int& turn) {
#pragma unroll
  for (int i = 0; i < K; ++i) s[i] = group_sum(s[i], WIDE ? 6 : ls);
  if constexpr (WIDE) {
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < K; ++i) buf[turn][threadIdx.x >> 6][i] = s[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < K; ++i) s[i] = buf[turn][threadIdx.x & 15][i];
#pragma unroll
    for (int i = 0; i < K; ++i) s[i] = group_sum(s[i], 4);
    turn ^= 1;
  }
}
__device__ __forceinline__ void clear(float (*buf)[16][2]) {
  if (threadIdx.x < 64) ((float*)buf)[threadIdx.x] = 0.f;
  __syncthreads();
}

// N(t): the mean and factor of the row, t becomes the normed row.  Lanes past the row
// (`in` false) hold zeros before and after.
template <bool WIDE>
__device__ __forceinline__ void norm_row(float (&t)[8], bool in, const NormArgs& a, float& mean, float& r,
                                         float (*buf)[16][2], int& turn) {
  mean = 0.f;
  if (!a.rms) {
    float s[1] = {0.f};
#pragma unroll
    for (int e = 0; e < 8; ++e) s[0] += t[e];
    row_sums<WIDE, 1>(s, a.ls, buf, turn);
    mean = s[0] * a.by_d;
    const float here = in ? mean : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] -= here;
  }
  float s[1] = {0.f};
#pragma unroll
  for (int e = 0; e < 8; ++e) s[0] += t[e] * t[e];
  row_sums<WIDE, 1>(s, a.ls, buf, turn);
  r = 1.f / sqrtf(s[0] * a.by_d + a.eps);
#pragma unroll
  for (int e = 0; e < 8; ++e) t[e] *= r;
}

// A lane's place: its row of the launch's first sweep, the step between rows, its chunk.
template <bool WIDE>
__device__ __forceinline__ void place(const NormArgs& a, int64_t& row, int64_t& step, int& chunk) {
  if constexpr (WIDE) {
    row = blockIdx.x, step = gridDim.x, chunk = threadIdx.x;
  } else {
    const int g = threadIdx.x >> a.ls, groups = (int)blockDim.x >> a.ls;
    row = (int64_t)blockIdx.x * groups + g, step = (int64_t)gridDim.x * groups;
    chunk = threadIdx.x & ((1 << a.ls) - 1);
  }
}

// The vectors of a call: a lane's entries, 1 and 0 where there are none.
struct Vectors {
  float gate[8], w1[8], b1[8], w2[8], b2[8];
};
template <int T, bool FULL, bool BIAS>
__device__ __forceinline__ void load_vectors(const NormArgs& a, bool in, int64_t col, Vectors& w) {
#pragma unroll
  for (int e = 0; e < 8; ++e) w.gate[e] = w.w1[e] = w.w2[e] = 1.f, w.b1[e] = w.b2[e] = 0.f;
  if (!in) return;
  if (FULL && a.gate) load8_or_f32<T>(a.gate, col, a.wf32, w.gate);
  if (FULL && a.post_w) load8_or_f32<T>(a.post_w, col, a.wf32, w.w1);
  if (FULL && BIAS && a.post_b) load8_or_f32<T>(a.post_b, col, a.wf32, w.b1);
  if (a.pre_w) load8_or_f32<T>(a.pre_w, col, a.wf32, w.w2);
  if (BIAS && a.pre_b) load8_or_f32<T>(a.pre_b, col, a.wf32, w.b2);
}

// Rows to be read, or others that are there in the place of rows that are not: every load
// is issued, without a branch, and what should not be there is made zero afterwards.
struct Source {
  const void* p;
  int64_t stride;
  bool there;
  __device__ __forceinline__ Source(const void* q, int64_t s, const void* other) : p(q ? q : other), stride(q ? s : 0), there(q != nullptr) {}
  __device__ __forceinline__ int64_t at(int64_t row, bool in, int64_t col) const { return row * stride + (in ? col : 0); }
};

// WIDE: rows of several waves, up to 1024 lanes; else rows within a wave.  FULL: with a gate, a
// norm of y or a dropout (DROP); without, the registers of their vectors and sums are free
// for more waves.  FAR: rows' outputs are past the caches.
template <int T, bool WIDE, bool FULL, bool DROP, bool FAR>
__global__ void __launch_bounds__(WIDE ? 1024 : 256, WIDE ? 4 : 2) norm_fwd(const NormArgs a) {
  __shared__ float buf[2][16][2];
  int64_t row, step;
  int chunk, turn = 0;
  place<WIDE>(a, row, step, chunk);
  const bool in = chunk < a.c;
  const int64_t col = 8 * (int64_t)chunk;
  Vectors w;
  load_vectors<T, FULL, true>(a, in, col, w);
  if constexpr (WIDE) clear(buf);
  const uint64_t seed = DROP ? a.drop.the_seed() : 0;
  const Source from_x(a.x, a.xs, a.x), from_y(a.y, a.ys, a.x);
  // Where up to four sums over several waves follow one another, the next row is loaded beside
  // them (20001 x 2568 119 us for 128, 8001 x 8192 111 for 125); lean kernels have more
  // waves instead (20001 x 2568 68 us, 71 with it).
  constexpr bool kAhead = WIDE && FULL;
  Raw8<T> next_x, next_y;
  auto load = [&](int64_t r) {
    next_x.load(from_x.p, from_x.at(r, in, col));
    next_y.load(from_y.p, from_y.at(r, in, col));
  };
  if (kAhead && row < a.n) load(row);
  for (; row < a.n; row += step) {
    if (!kAhead) load(row);
    const Raw8<T> rx = next_x, ry = next_y;
    if (kAhead) load(row + step < a.n ? row + step : row);
    float x[8], t[8];
    rx.get(in, x);
    float m1 = 0.f, r1 = 0.f, m2 = 0.f, r2 = 0.f;
    if (a.y) {
      ry.get(in, t);
      if (FULL && a.post_w) {
        norm_row<WIDE>(t, in, a, m1, r1, buf, turn);
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = fmaf(t[e], w.w1[e], w.b1[e]);
      }
      if constexpr (DROP) {
        const Random128 u = philox(a.drop.first + (uint64_t)row * a.c + chunk, a.drop.site, seed);
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = u.bits16(e) >= a.drop.cut ? t[e] * a.drop.unit : 0.f;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = fmaf(a.alpha, x[e], FULL ? w.gate[e] * t[e] : t[e]);
      if (in) store8<T, FAR>(a.h, row * (8 * (int64_t)a.c) + col, x);
    }
    if (a.pre_w) {
      if (!in)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.f;
      norm_row<WIDE>(x, in, a, m2, r2, buf, turn);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = fmaf(x[e], w.w2[e], w.b2[e]);
      if (in) store8<T, FAR>(a.z, row * (8 * (int64_t)a.c) + col, x);
    }
    if (a.stats && chunk == 0) a.stats[row] = make_float4(m1, r1, m2, r2);
  }
}

// The sums of the first norm and the gate are two for each feature, S = sum e D v and
// B = sum e D, whatever of them is asked for:
//   dgate = post_w S,  dpost_w = gate S,  dpost_b = gate B
// and the rows' loop needs the vectors as gate post_w and gate post_b alone.  The gradient of a
// gate behind a norm with a bias (kGate) has a sum of its own, G = sum e D (v post_w + post_b): as
// post_w S + post_b B it would have the roundings of both where they cancel.  Its vectors are
// apart then, those of rows within a wave in LDS; backward and join, with it and from S and B:
// 20001 x 2568 in fp32 260 us and 257, 17408 x 512 in bf16 34 and 33, and where it takes the
// next row's registers 16001 x 4096 in bf16 181 and 169, 50001 x 1160 in fp16 196 and 174.
// BIAS: with sums for biases.  In rows of several waves with everything their sums and gate
// post_b are in LDS, each lane its own 32 bytes of them, so that 16 waves fit a compute unit with
// the next row's loads (116 to 118 registers; 106 without).  With sums for each vector instead of
// S and B: 151 registers, 50001 x 1160 188 us for 173, 20001 x 2568 183 for 164.
enum Bias { kNoBias, kBias, kGateBias };
template <int T, bool WIDE, bool FULL, Bias BIASES, bool DROP, bool FAR>
__global__ void __launch_bounds__(WIDE ? 1024 : 256, 4) norm_bwd(const NormArgs a) {
  __shared__ float buf[2][16][2];
  __shared__ float joined[WIDE ? 1 : 4][WIDE ? 1 : 512];
  constexpr bool BIAS = BIASES != kNoBias, kGate = BIASES == kGateBias;
  // kGate in rows within a wave: all rows' gate, post_w, post_b and pre_w
  constexpr bool kTable = kGate && !WIDE;
  __shared__ __attribute__((aligned(16))) float table[kTable ? 4 : 1][kTable ? 512 : 4];
  int64_t row, step;
  int chunk, turn = 0;
  place<WIDE>(a, row, step, chunk);
  const bool in = chunk < a.c;
  const int64_t col = 8 * (int64_t)chunk;
  extern __shared__ f32x4 own[];  // kOwn: [sb2, B, gate post_b (kGate: post_b, G)][halves][lanes]
  constexpr bool kOwn = WIDE && FULL && BIAS;
  auto get_own = [&](int k, float (&q)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const f32x4 x = own[(2 * k + i) * blockDim.x + threadIdx.x];
#pragma unroll
      for (int e = 0; e < 4; ++e) q[4 * i + e] = x[e];
    }
  };
  auto put_own = [&](int k, const float (&q)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      own[(2 * k + i) * blockDim.x + threadIdx.x] = f32x4{q[4 * i], q[4 * i + 1], q[4 * i + 2], q[4 * i + 3]};
  };
  auto add_own = [&](int k, const float (&q)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      own[(2 * k + i) * blockDim.x + threadIdx.x] += f32x4{q[4 * i], q[4 * i + 1], q[4 * i + 2], q[4 * i + 3]};
  };
  float gw[8], gb[8], w2[8], S[8], B[8], sw2[8], sb2[8];
  float w1[8], b1[8], g1[8], G[8];  // kGate: the vectors apart
  const float unit = DROP ? a.drop.unit : 1.f;
  {
    Vectors w;
    load_vectors<T, FULL, BIAS>(a, in, col, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float g = DROP ? w.gate[e] * unit : w.gate[e];  // dropout's factor is the gate's
      gw[e] = g * w.w1[e], gb[e] = g * w.b1[e], w2[e] = w.w2[e];
      w1[e] = w.w1[e], b1[e] = w.b1[e], g1[e] = g;
      S[e] = B[e] = sw2[e] = sb2[e] = G[e] = 0.f;
    }
  }
  if constexpr (kOwn) put_own(0, sb2), put_own(1, B), put_own(2, kGate ? b1 : gb);
  if constexpr (kOwn && kGate) put_own(3, G);
  if constexpr (kTable) {
    if (threadIdx.x < 1u << a.ls) {
      store8<kF32>(table[0], col, g1), store8<kF32>(table[1], col, w1);
      store8<kF32>(table[2], col, b1), store8<kF32>(table[3], col, w2);
    }
    __syncthreads();
  }
  auto get_vectors = [&] {
    if constexpr (kOwn) get_own(2, kGate ? b1 : gb);
    if constexpr (kTable) load8<kF32>(table[0], col, g1), load8<kF32>(table[1], col, w1), load8<kF32>(table[2], col, b1);
  };
  if constexpr (WIDE) clear(buf);
  const uint64_t seed = DROP ? a.drop.the_seed() : 0;
  const Source from_x(a.x, a.xs, a.x), from_y(a.y, a.ys, a.x), from_dh(a.dh, a.dhs, a.x), from_dz(a.dz, a.dzs, a.x);
  const bool post = FULL && a.post_w;
  // The next row beside the sums, as in the forward (50001 x 1160 154 us for 173, 20001 x 2568 134 for
  // 164; 16001 x 4096 168 for 162, the one size of these that loses, and not worth a rule); fp32 rows
  // with biases' sums, and kGate, leave no registers for it (kGate with 24 to 32 bytes of them spilled:
  // 50001 x 1160 214 for 196, 20001 x 2568 178 for 180).
  constexpr bool kAhead = WIDE && FULL && !(BIAS && T == kF32) && !kGate;
  Raw8<T> next_x, next_y, next_dh, next_dz;
  float4 next_st;
  auto load = [&](int64_t r) {
    next_x.load(from_x.p, from_x.at(r, in, col));
    next_y.load(from_y.p, from_y.at(r, in, col));
    next_dh.load(from_dh.p, from_dh.at(r, in, col));
    next_dz.load(from_dz.p, from_dz.at(r, in, col));
    next_st = a.stats[r];
  };
  if (kAhead && row < a.n) load(row);
  for (; row < a.n; row += step) {
    if (!kAhead) load(row);
    const Raw8<T> rx = next_x, ry = next_y, rh = next_dh, rz = next_dz;
    float4 st = next_st;
    if (kAhead) load(row + step < a.n ? row + step : row);
    if (!post) st.x = 0.f, st.y = 1.f;
    if (!in) st.y = st.w = 0.f;  // (normed rows of lanes past the row are zeros)
    bool keep[8];
    if constexpr (DROP) {
      const Random128 u = philox(a.drop.first + (uint64_t)row * a.c + chunk, a.drop.site, seed);
#pragma unroll
      for (int e = 0; e < 8; ++e) keep[e] = u.bits16(e) >= a.drop.cut;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) keep[e] = true;
    }
    float h[8], v[8], e8[8], g[8];
    rx.get(in, h);
    ry.get(in && from_y.there, v);
    rh.get(in && from_dh.there, e8);
    rz.get(in && from_dz.there, g);
    if (a.y) {
      get_vectors();
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (FULL) v[e] = (v[e] - st.x) * st.y;
        const float t = !FULL ? v[e] : kGate ? g1[e] * fmaf(v[e], w1[e], b1[e]) : BIAS ? fmaf(v[e], gw[e], gb[e]) : v[e] * gw[e];
        h[e] = fmaf(a.alpha, h[e], keep[e] ? t : 0.f);
      }
    }
    if (a.pre_w) {
      if constexpr (kTable) load8<kF32>(table[3], col, w2);
      if (kOwn && a.want_pre_b) add_own(0, g);
      float s[2] = {0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        h[e] = (h[e] - st.z) * st.w;
        sw2[e] = fmaf(g[e], h[e], sw2[e]);
        if (BIAS && !kOwn) sb2[e] += g[e];
        g[e] *= w2[e];
        s[0] += g[e], s[1] = fmaf(g[e], h[e], s[1]);
      }
      row_sums<WIDE, 2>(s, a.ls, buf, turn);
      const float m = a.rms ? 0.f : s[0] * a.by_d, k = s[1] * a.by_d;
#pragma unroll
      for (int e = 0; e < 8; ++e) e8[e] = fmaf(st.w, g[e] - fmaf(h[e], k, m), e8[e]);
    }
    if (a.dx && in) {
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = a.alpha * e8[e];
      store8<T, FAR>(a.dx, row * (8 * (int64_t)a.c) + col, o);
    }
    if (!a.y) continue;
    if constexpr (FULL) {
      float s[2] = {0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        S[e] = fmaf(e8[e], keep[e] ? v[e] : 0.f, S[e]);
        e8[e] = keep[e] ? e8[e] : 0.f;
        if (BIAS && !kOwn) B[e] += e8[e];
      }
      if (kOwn && a.want_post_b) add_own(1, e8);
      if constexpr (kGate) {
        get_vectors();
        if constexpr (kOwn) get_own(3, G);
#pragma unroll
        for (int e = 0; e < 8; ++e) G[e] = fmaf(e8[e], keep[e] ? fmaf(v[e], w1[e], b1[e]) : 0.f, G[e]);
        if constexpr (kOwn) put_own(3, G);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        e8[e] = kGate ? e8[e] * g1[e] * w1[e] : e8[e] * gw[e];
        s[0] += e8[e], s[1] = fmaf(e8[e], v[e], s[1]);
      }
      if (post) {
        row_sums<WIDE, 2>(s, a.ls, buf, turn);
        const float m = a.rms ? 0.f : s[0] * a.by_d, k = s[1] * a.by_d;
#pragma unroll
        for (int e = 0; e < 8; ++e) e8[e] = st.y * (e8[e] - fmaf(v[e], k, m));
      }
    }
    if (a.dy && in) store8<T, FAR>(a.dy, row * (8 * (int64_t)a.c) + col, e8);
  }
  if constexpr (kOwn) get_own(0, sb2), get_own(1, B);
  if constexpr (kOwn && kGate) get_own(3, G);
  float sg[8];
  if constexpr (FULL) {  // the vectors' own sums
    Vectors w;
    load_vectors<T, FULL, BIAS>(a, in, col, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      sg[e] = unit * (kGate ? G[e] : w.w1[e] * S[e]);
      S[e] *= w.gate[e] * unit, B[e] *= w.gate[e] * unit;
    }
  }

  // One row of sums of the workgroup: groups of a wave, then waves, in order.
  const int d = 8 * a.c;
  float* part = a.part;
  int k = 0;
  const int sums = a.want_gate + a.want_post + a.want_post_b + a.want_pre + a.want_pre_b;
  auto put = [&](float (&s)[8]) {
    float* to = part + ((int64_t)blockIdx.x * sums + k++) * d;
    if constexpr (WIDE) {
      if (in) store8<kF32>(to, col, s);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float p, q;
        if (a.ls < 4) s[e] += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(s[e]), 0x128, 0xF, 0xF, true));  // row_ror 8
        if (a.ls < 5) both16(s[e], p, q), s[e] = p + q;
        if (a.ls < 6) both32(s[e], p, q), s[e] = p + q;
      }
      const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
      __syncthreads();
      if (lane < 1 << a.ls)
#pragma unroll
        for (int e = 0; e < 8; ++e) joined[wave][64 * e + lane] = s[e];
      __syncthreads();
      for (int i = threadIdx.x; i < d; i += 256) {
        const int at = 64 * (i & 7) + (i >> 3);
        to[i] = joined[0][at] + joined[1][at] + joined[2][at] + joined[3][at];
      }
    }
  };
  if (FULL && a.want_gate) put(sg);
  if (FULL && a.want_post) put(S);
  if (FULL && BIAS && a.want_post_b) put(B);
  if (a.want_pre) put(sw2);
  if (BIAS && a.want_pre_b) put(sb2);
}

// Sums of parts [parts][sums][d] in a fixed order: 32 columns of one vector for each
// workgroup, 32 slices of the parts, sixteen loads at a time, joined through LDS.
template <int T>
__global__ void __launch_bounds__(1024) norm_join(const float* __restrict__ part, int parts, int sums, int d, int wf32,
                                                 void* o0, void* o1, void* o2, void* o3, void* o4) {
  __shared__ float lds[32][33];
  const int cols = (d + 31) / 32, k = blockIdx.x / cols, col = (blockIdx.x - k * cols) * 32 + (threadIdx.x & 31);
  const int slice = threadIdx.x >> 5;
  float s = 0.f;
  if (col < d) {
    const float* p = part + (int64_t)k * d + col;
    const int64_t row = (int64_t)sums * d;
    int i = slice;
    for (; i < parts; i += 32 * 16) {
      float v[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] = p[(i + 32 * j < parts ? i + 32 * j : i) * row];
#pragma unroll
      for (int j = 0; j < 16; ++j) s += i + 32 * j < parts ? v[j] : 0.f;
    }
  }
  lds[slice][threadIdx.x & 31] = s;
  __syncthreads();
  if (slice == 0 && col < d) {
    float t = 0.f;
#pragma unroll
    for (int j = 0; j < 32; ++j) t += lds[j][threadIdx.x];
    void* const to = k == 0 ? o0 : k == 1 ? o1 : k == 2 ? o2 : k == 3 ? o3 : o4;
    if (T == kF32 || wf32)
      ((float*)to)[col] = t;
    else if constexpr (T == kF16)
      ((_Float16*)to)[col] = (_Float16)t;
    else
      ((__bf16*)to)[col] = (__bf16)t;
  }
}

struct Shape {
  bool wide;
  unsigned threads;
  int ls;
  int64_t groups;  // rows of a workgroup at a time
};
Shape shape_of(int64_t d) {
  Shape s;
  const int c = (int)(d / 8);
  s.wide = c > 64;
  s.threads = s.wide ? (unsigned)((c + 63) / 64 * 64) : 256;
  s.ls = s.wide ? 6 : row_lanes_log2(c, 8);
  s.groups = s.wide ? 1 : 256 >> s.ls;
  return s;
}
// Workgroups: what covers the rows, at most as many as are resident at once with
// `waves` to a compute unit, so that all of them go through as many rows.
unsigned grid_of(const Shape& s, int64_t n, int waves) {
  const int64_t need = (n + s.groups - 1) / s.groups, each = waves / (int)(s.threads / 64), most = 256 * (each < 1 ? 1 : each);
  return (unsigned)(need < most ? need : most);
}
// The forward starts more than that: nothing is left to be joined.  The backward's kernels
// have registers for 16 waves (30001 x 2048 without gate and norm of y: 144 us with 16, 151
// with 20).
constexpr int kFwdWaves = 32, kBwdWaves = 16;

infcl_status check(const infcl_add_norm* a) {
  if (!a || a->n < 0 || a->d < 1 || !type_known(a->dtype) || !type_known(a->wdtype) ||
      (a->norm != INFCL_NORM_LAYER && a->norm != INFCL_NORM_RMS) || !(a->eps >= 0.f) || a->eps > 3e38f ||
      !(a->alpha >= -3e38f && a->alpha <= 3e38f) || !drop_ok(a->drop) || a->x_stride < a->d ||
      (a->post_b && !a->post_w) || (a->pre_b && !a->pre_w))
    return INFCL_ERR_INVALID;
  if (a->d % 8 != 0 || a->d > 8192 || a->x_stride % 8 != 0 || a->n > ((int64_t)1 << 40) / a->d ||
      a->x_stride > ((int64_t)1 << 32) || (a->wdtype != INFCL_F32 && a->wdtype != a->dtype) ||
      a->drop.row0 > ((int64_t)1 << 62) / a->d)
    return INFCL_ERR_UNSUPPORTED;
  return INFCL_OK;
}
// The vectors and y of a call that has rows.
infcl_status check_rows(const infcl_add_norm* a, const void* x, const void* y) {
  const void* w[5] = {a->gate, a->post_w, a->post_b, a->pre_w, a->pre_b};
  for (const void* p : w)
    if (p && ((uintptr_t)p % 16) != 0) return INFCL_ERR_INVALID;
  if (a->n == 0) return INFCL_OK;  // (rows have no addresses then)
  if (!y && (a->gate || a->post_w || a->drop.p > 0.f || a->alpha != 1.f || !a->pre_w)) return INFCL_ERR_INVALID;
  if (y && a->y_stride < a->d) return INFCL_ERR_INVALID;
  if (y && (a->y_stride % 8 != 0 || a->y_stride > ((int64_t)1 << 32))) return INFCL_ERR_UNSUPPORTED;
  if (!block_aligned(x, 16) || ((uintptr_t)y % 16) != 0) return INFCL_ERR_INVALID;
  return INFCL_OK;
}
NormArgs args_of(const infcl_add_norm* a, const Shape& s, const void* x, const void* y) {
  NormArgs r = {};
  r.x = x, r.y = y, r.gate = a->gate, r.post_w = a->post_w, r.post_b = a->post_b, r.pre_w = a->pre_w, r.pre_b = a->pre_b;
  r.n = a->n, r.xs = a->x_stride, r.ys = a->y_stride, r.c = (int)(a->d / 8), r.ls = s.ls;
  r.rms = a->norm == INFCL_NORM_RMS, r.wf32 = a->wdtype == INFCL_F32, r.eps = a->eps, r.alpha = a->alpha;
  r.by_d = 1.f / (float)a->d;
  r.drop = drop_of(a->drop, a->d);
  return r;
}

template <int T, bool FULL, bool DROP, bool FAR>
void fwd_t(const NormArgs& r, const Shape& s, hipStream_t st) {
  const dim3 grid(grid_of(s, r.n, kFwdWaves)), block(s.threads);
  if (s.wide)
    hipLaunchKernelGGL((norm_fwd<T, true, FULL, DROP, FAR>), grid, block, 0, st, r);
  else
    hipLaunchKernelGGL((norm_fwd<T, false, FULL, DROP, FAR>), grid, block, 0, st, r);
}
template <int T, bool FULL, Bias BIAS, bool DROP, bool FAR>
void bwd_t(const NormArgs& r, const Shape& s, unsigned wgs, hipStream_t st) {
  const dim3 grid(wgs), block(s.threads);
  const size_t own = FULL && BIAS != kNoBias ? (BIAS == kGateBias ? 8 : 6) * 16 * (size_t)s.threads : 0;
  if (!s.wide)
    hipLaunchKernelGGL((norm_bwd<T, false, FULL, BIAS, DROP, FAR>), grid, block, 0, st, r);
  else
    hipLaunchKernelGGL((norm_bwd<T, true, FULL, BIAS, DROP, FAR>), grid, block, own, st, r);
}
bool full(const NormArgs& r) { return r.gate || r.post_w || r.drop.cut; }
template <int T, bool FAR>
void fwd_far(const NormArgs& r, const Shape& s, hipStream_t st) {
  if (!full(r))
    fwd_t<T, false, false, FAR>(r, s, st);
  else if (r.drop.cut)
    fwd_t<T, true, true, FAR>(r, s, st);
  else
    fwd_t<T, true, false, FAR>(r, s, st);
}
template <int T, bool FAR, Bias BIAS>
void bwd_full(const NormArgs& r, const Shape& s, unsigned wgs, hipStream_t st) {
  r.drop.cut ? bwd_t<T, true, BIAS, true, FAR>(r, s, wgs, st) : bwd_t<T, true, BIAS, false, FAR>(r, s, wgs, st);
}
template <int T, bool FAR>
void bwd_far(const NormArgs& r, const Shape& s, unsigned wgs, hipStream_t st) {
  if (!full(r))
    bwd_t<T, false, kBias, false, FAR>(r, s, wgs, st);
  else if (r.gate && r.post_b)  // (whether dgate is asked for or not: the other results are the same bits)
    bwd_full<T, FAR, kGateBias>(r, s, wgs, st);
  else
    r.post_b || r.pre_b ? bwd_full<T, FAR, kBias>(r, s, wgs, st) : bwd_full<T, FAR, kNoBias>(r, s, wgs, st);
}
template <int T>
bool far(const NormArgs& r) {
  return r.n * r.c * 8 * (T == kF32 ? 4 : 2) > kL2Bytes;
}
template <int T>
void fwd_any(const NormArgs& r, const Shape& s, hipStream_t st) {
  far<T>(r) ? fwd_far<T, true>(r, s, st) : fwd_far<T, false>(r, s, st);
}
template <int T>
void bwd_any(const NormArgs& r, const Shape& s, unsigned wgs, hipStream_t st) {
  far<T>(r) ? bwd_far<T, true>(r, s, wgs, st) : bwd_far<T, false>(r, s, wgs, st);
}
template <int T>
void join_t(const NormArgs& r, unsigned wgs, int sums, void* const* o, hipStream_t st) {
  const int d = 8 * r.c;
  hipLaunchKernelGGL((norm_join<T>), dim3((unsigned)(sums * ((d + 31) / 32))), dim3(1024), 0, st, r.part, (int)wgs, sums, d,
                     r.wf32, o[0], o[1], o[2], o[3], o[4]);
}

}  // namespace
}  // namespace infcl

using namespace infcl;

extern "C" infcl_status infcl_add_norm_fwd(const infcl_add_norm* a, const void* x, const void* y, void* h, void* z,
                                           float* stats, void* stream) {
  infcl_status s = check(a);
  if (s == INFCL_OK) s = check_rows(a, x, y);
  if (s != INFCL_OK || a->n == 0) return s;
  if ((y && !block_aligned(h, 16)) || (a->pre_w && !block_aligned(z, 16)) || ((uintptr_t)stats % 16) != 0)
    return INFCL_ERR_INVALID;
  const Shape sh = shape_of(a->d);
  NormArgs r = args_of(a, sh, x, y);
  r.h = h, r.z = z, r.stats = (float4*)stats;
  hipStream_t st = (hipStream_t)stream;
  if (a->dtype == INFCL_BF16)
    fwd_any<kBF16>(r, sh, st);
  else if (a->dtype == INFCL_F16)
    fwd_any<kF16>(r, sh, st);
  else
    fwd_any<kF32>(r, sh, st);
  return launch_status();
}

extern "C" infcl_status infcl_add_norm_bwd_workspace(const infcl_add_norm* a, size_t* bytes) {
  const infcl_status s = check(a);
  if (s != INFCL_OK) return s;
  if (!bytes) return INFCL_ERR_INVALID;
  const Shape sh = shape_of(a->d);
  const size_t n = (size_t)grid_of(sh, a->n, kBwdWaves) * 5 * (size_t)a->d * 4;
  *bytes = n < 256 ? 256 : (n + 255) & ~(size_t)255;
  return INFCL_OK;
}

extern "C" infcl_status infcl_add_norm_bwd(const infcl_add_norm* a, const void* x, const void* y, const float* stats,
                                           const infcl_add_norm_grads* g, void* workspace, size_t ws_bytes,
                                           void* stream) {
  infcl_status s = check(a);
  if (s == INFCL_OK) s = check_rows(a, x, y);
  if (s != INFCL_OK) return s;
  if (!g || (g->dh && g->dh_stride < a->d) || (g->dz && (g->dz_stride < a->d || !a->pre_w)) || (g->dy && !y && a->n > 0) ||
      (g->dgate && !a->gate) || (g->dpost_w && !a->post_w) || (g->dpost_b && !a->post_b) || (g->dpre_w && !a->pre_w) ||
      (g->dpre_b && !a->pre_b))
    return INFCL_ERR_INVALID;
  if ((g->dh && (g->dh_stride % 8 != 0 || g->dh_stride > ((int64_t)1 << 32))) ||
      (g->dz && (g->dz_stride % 8 != 0 || g->dz_stride > ((int64_t)1 << 32))))
    return INFCL_ERR_UNSUPPORTED;
  const void* p[9] = {g->dh, g->dz, g->dx, g->dy, g->dgate, g->dpost_w, g->dpost_b, g->dpre_w, g->dpre_b};
  for (const void* q : p)
    if (((uintptr_t)q % 16) != 0) return INFCL_ERR_INVALID;
  if (!block_aligned(workspace, 256) || (a->n > 0 && !block_aligned(stats, 16))) return INFCL_ERR_INVALID;
  size_t need = 0;
  s = infcl_add_norm_bwd_workspace(a, &need);
  if (s != INFCL_OK) return s;
  if (ws_bytes < need) return INFCL_ERR_WORKSPACE;
  const Shape sh = shape_of(a->d);
  NormArgs r = args_of(a, sh, x, y);
  r.stats = (float4*)stats, r.part = (float*)workspace;
  r.dh = g->dh, r.dz = g->dz, r.dhs = g->dh_stride, r.dzs = g->dz_stride, r.dx = g->dx, r.dy = g->dy;
  r.want_gate = g->dgate != nullptr, r.want_post = g->dpost_w != nullptr, r.want_post_b = g->dpost_b != nullptr;
  r.want_pre = g->dpre_w != nullptr, r.want_pre_b = g->dpre_b != nullptr;
  void* outs[5] = {nullptr, nullptr, nullptr, nullptr, nullptr};
  int sums = 0;
  for (void* o : {g->dgate, g->dpost_w, g->dpost_b, g->dpre_w, g->dpre_b})
    if (o) outs[sums++] = o;
  hipStream_t st = (hipStream_t)stream;
  const unsigned wgs = grid_of(sh, a->n, kBwdWaves);
  if (wgs > 0) {
    if (a->dtype == INFCL_BF16)
      bwd_any<kBF16>(r, sh, wgs, st);
    else if (a->dtype == INFCL_F16)
      bwd_any<kF16>(r, sh, wgs, st);
    else
      bwd_any<kF32>(r, sh, wgs, st);
    s = launch_status();
    if (s != INFCL_OK) return s;
  }
  if (sums > 0) {  // (no rows: zeros)
    if (a->dtype == INFCL_BF16)
      join_t<kBF16>(r, wgs, sums, outs, st);
    else if (a->dtype == INFCL_F16)
      join_t<kF16>(r, wgs, sums, outs, st);
    else
      join_t<kF32>(r, wgs, sums, outs, st);
    return launch_status();
  }
  return INFCL_OK;
}

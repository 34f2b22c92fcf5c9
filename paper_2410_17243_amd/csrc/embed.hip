// Token embedding with scaling, and the table's gradient by sorted tokens.
//
//   out_t    = scale W[tok_t]
//   dW_v     = scale sum_{t: tok_t = v} dout_t
//
// Both are bound by memory.  The forward is one copy of rows.  The gradient
// has to read dout once and write the table once; a token's rows are spread
// over dout, so the positions are first sorted by token (a stable radix sort:
// 12 bytes per token, against 2 d bytes of its row) and each table row is then
// one group of lanes that adds its rows in order of t: no atomics on floats,
// one write per table row, and the order of every sum is fixed.  Tokens with
// many rows (those that open and close every caption) are summed in parts of 32
// or 64 sorted positions, joined in order.
//
// 524288 tokens, 512 features of bf16, vocabulary 50000: forward 147 us (4.0 TB/s of
// the 588 MB), sort 54 us in five launches, sums 140 us (638 MB at 4.6 TB/s), joins 15
// us (the parts of the two tokens that every caption has are a chain each).  2001
// tokens, 512 features of fp32, vocabulary 8192: 4 + 11 + 8 + 4 us, launches and the
// latency of dependent reads.
#include "infcl_tower.h"
#include "rows.hpp"

namespace infcl {
namespace {

// ------------------------------------------------------------------- forward

// A group of 1 << ls lanes copies a row; each group takes kFwdRows rows at a
// time so that as many loads are in flight.
constexpr int kFwdRows = 4;

template <int T, typename Tok>
__global__ void __launch_bounds__(256) embed_fwd_kernel(const Tok* __restrict__ tok, int64_t n,
                                                        const u32x4* __restrict__ table, int64_t vocab, int c, int ls,
                                                        float scale, u32x4* __restrict__ out) {
  const int gl = threadIdx.x & ((1 << ls) - 1);
  const int64_t g = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> ls, ng = (int64_t)gridDim.x * 256 >> ls;
  for (int64_t t0 = g * kFwdRows; t0 < n; t0 += ng * kFwdRows) {
    int64_t v[kFwdRows];
#pragma unroll
    for (int k = 0; k < kFwdRows; ++k) {
      v[k] = t0 + k < n ? (int64_t)tok[t0 + k] : -1;
      if (v[k] >= vocab) v[k] = -1;
    }
    for (int i = gl; i < c; i += 1 << ls) {
      u32x4 r[kFwdRows];
#pragma unroll
      for (int k = 0; k < kFwdRows; ++k) {
        r[k] = u32x4{0, 0, 0, 0};
        if (v[k] >= 0) r[k] = table[v[k] * c + i];
      }
#pragma unroll
      for (int k = 0; k < kFwdRows; ++k) {
        if (v[k] >= 0) {
          float x[Chunk<T>::N];
          Chunk<T>::load(r[k], x);
#pragma unroll
          for (int e = 0; e < Chunk<T>::N; ++e) x[e] *= scale;
          r[k] = Chunk<T>::store(x);
        }
        if (t0 + k < n) __builtin_nontemporal_store(r[k], &out[(t0 + k) * c + i]);
      }
    }
  }
}

// ---------------------------------------------------------------------- sort

template <typename Tok>
__device__ __forceinline__ uint32_t token_key(Tok t, uint32_t vocab) {
  return t >= 0 && (uint64_t)t < vocab ? (uint32_t)t : vocab;  // (invalid ones last)
}

// Where the rows of one token begin and end in sorted order: by table row
// (start, of many tokens) or by sorted position (few tokens).
struct Runs {
  const uint2* sorted;    // (token, position), n of them
  const uint32_t* start;  // by row: first sorted position whose token is >= v, v = 0 .. vocab
  const uint2* run;       // by position: [begin, end) of its run; null: by row
  int lg;                 // log2 of the positions of a part
};

__device__ __forceinline__ void run_of(const Runs& r, int64_t at, uint32_t v, uint32_t& a, uint32_t& b) {
  if (r.run) {
    const uint2 x = r.run[at];
    a = x.x, b = x.y;
  } else {
    a = r.start[v], b = r.start[v + 1];
  }
}

__device__ __forceinline__ void zero_rows(u32x4* p, int64_t n, int64_t i, int64_t step) {
  for (; i < n; i += step) p[i] = u32x4{0, 0, 0, 0};
}

// Few tokens (up to kFew): a token's place is the number of smaller ones, plus
// that of its equals before it, and the former and the number of its equals are
// its run.  n^2 comparisons, which the whole chip shares: 16 tokens to a
// workgroup, each counted by 16 groups of lanes (n = 2001: 11 us; a bitonic network
// in one workgroup 24, the radix sort below 32 in five launches).  The other workgroups clear the table meanwhile,
// whose absent rows no one else writes.
constexpr int kFew = 4096, kRankTokens = 16;

template <typename Tok>
__global__ void __launch_bounds__(256) sort_few(const Tok* __restrict__ tok, int n, uint32_t vocab, unsigned rank_blocks,
                                                uint2* __restrict__ sorted, uint2* __restrict__ run,
                                                u32x4* __restrict__ table, int64_t chunks) {
  if (blockIdx.x >= rank_blocks) {
    zero_rows(table, chunks, ((int64_t)blockIdx.x - rank_blocks) * 256 + threadIdx.x,
              ((int64_t)gridDim.x - rank_blocks) * 256);
    return;
  }
  __shared__ __attribute__((aligned(16))) uint32_t key[kFew];
  __shared__ uint32_t red[4][kRankTokens][3];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n4 = (n + 3) & ~3;
#pragma unroll 4
  for (int i = tid; i < n4; i += 256) key[i] = i < n ? token_key(tok[i], vocab) : 0xFFFFFFFFu;  // (no token's key)
  __syncthreads();
  const int i0 = (int)blockIdx.x * kRankTokens, i = i0 + (lane & 15), sub = wave * 4 + (lane >> 4);
  const uint32_t mine = i < n ? key[i] : 0xFFFFFFFEu;
  uint32_t less = 0, same = 0, ahead = 0;
#pragma unroll 4
  for (int j = 4 * sub; j < n4; j += 64) {
    const u32x4 k = *(const u32x4*)&key[j];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      less += k[e] < mine;
      same += k[e] == mine;
      ahead += k[e] == mine && j + e < i;
    }
  }
#pragma unroll
  for (int s = 16; s <= 32; s <<= 1) {
    less += __shfl_xor(less, s);
    same += __shfl_xor(same, s);
    ahead += __shfl_xor(ahead, s);
  }
  if (lane < 16) red[wave][lane][0] = less, red[wave][lane][1] = same, red[wave][lane][2] = ahead;
  __syncthreads();
  if (tid >= kRankTokens || i0 + tid >= n) return;
  uint32_t t[3] = {0, 0, 0};
  for (int w = 0; w < 4; ++w)
    for (int e = 0; e < 3; ++e) t[e] += red[w][tid][e];
  sorted[t[0] + t[2]] = make_uint2(mine, (uint32_t)i);
  run[t[0] + t[2]] = make_uint2(t[0], t[0] + t[1]);
}

// More tokens: a radix sort, least significant digit first, `bits` bits a pass
// (at most kMaxBits).  A block of 4 waves owns kTile consecutive elements, a
// wave a quarter of them, 64 at a time in order.
constexpr int kTile = 4096, kMaxBits = 10;

// Counts of a tile's digits.
template <typename Tok, bool FIRST>
__global__ void __launch_bounds__(256) sort_count(const Tok* __restrict__ tok, const uint2* __restrict__ in, int64_t n,
                                                  uint32_t vocab, int shift, int bits, uint32_t* __restrict__ hist) {
  __shared__ uint32_t cnt[1 << kMaxBits];
  const int bins = 1 << bits;
  for (int i = threadIdx.x; i < bins; i += 256) cnt[i] = 0;
  __syncthreads();
  const int64_t t0 = (int64_t)blockIdx.x * kTile;
#pragma unroll 8
  for (int i = threadIdx.x; i < kTile; i += 256)
    if (t0 + i < n) {
      const uint32_t k = FIRST ? token_key(tok[t0 + i], vocab) : in[t0 + i].x;
      atomicAdd(&cnt[(k >> shift) & (bins - 1)], 1u);
    }
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += 256) hist[(int64_t)blockIdx.x * bins + i] = cnt[i];
}

// One pass: every element to its place.  The place is the number of elements
// with smaller digits (all tiles), plus those of its digit in earlier tiles,
// plus those earlier in this tile.
template <typename Tok, bool FIRST>
__global__ void __launch_bounds__(256) sort_scatter(const Tok* __restrict__ tok, const uint2* __restrict__ in,
                                                    int64_t n, uint32_t vocab, int shift, int bits,
                                                    const uint32_t* __restrict__ hist, uint2* __restrict__ out) {
  __shared__ uint32_t base[1 << kMaxBits], wcnt[4][1 << kMaxBits], wsum[4];
  const int bins = 1 << bits, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int tiles = gridDim.x;
  constexpr int kWave = kTile / 4;
  const int64_t w0 = (int64_t)blockIdx.x * kTile + wave * kWave;
  uint2 el[kWave / 64];
#pragma unroll
  for (int i = 0; i < kWave / 64; ++i) {
    const int64_t t = w0 + 64 * i + lane;
    el[i] = make_uint2(0, 0);
    if (t < n) el[i] = FIRST ? make_uint2(token_key(tok[t], vocab), (uint32_t)t) : in[t];
  }
  for (int i = threadIdx.x; i < 4 * bins; i += 256) wcnt[i >> bits][i & (bins - 1)] = 0;
  // a thread's share of the bins: 1 to 4 consecutive ones
  const int per = bins > 256 ? bins >> 8 : 1;
  uint32_t all[4] = {0, 0, 0, 0}, mine = 0;
  if ((int)threadIdx.x * per < bins) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (k >= per) break;
      const uint32_t* h = hist + threadIdx.x * per + k;
      uint32_t before = 0, sum = 0;
#pragma unroll 16
      for (int t = 0; t < tiles; ++t) {
        const uint32_t x = h[(int64_t)t << bits];
        sum += x;
        before += t < (int)blockIdx.x ? x : 0;
      }
      all[k] = sum;
      base[threadIdx.x * per + k] = before;
      mine += sum;
    }
  }
  // exclusive scan over the threads
  uint32_t inc = mine;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const uint32_t o = __shfl_up(inc, s);
    if (lane >= s) inc += o;
  }
  if (lane == 63) wsum[wave] = inc;
  __syncthreads();
  uint32_t off = inc - mine;
  for (int w = 0; w < wave; ++w) off += wsum[w];
  if ((int)threadIdx.x * per < bins) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < per) {
        base[threadIdx.x * per + k] += off;
        off += all[k];
      }
  }
  // counts of this wave's quarter, then places
#pragma unroll
  for (int i = 0; i < kWave / 64; ++i)
    if (w0 + 64 * i + lane < n) atomicAdd(&wcnt[wave][(el[i].x >> shift) & (bins - 1)], 1u);
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += 256) {
    uint32_t o = base[i];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t h = wcnt[w][i];
      wcnt[w][i] = o;
      o += h;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWave / 64; ++i) {
    const bool live = w0 + 64 * i + lane < n;
    const uint32_t dg = (el[i].x >> shift) & (bins - 1);
    uint64_t same = __ballot(live);
    for (int k = 0; k < bits; ++k) {  // lanes with this lane's digit
      const bool bit = (dg >> k) & 1;
      const uint64_t m = __ballot(bit);
      same &= bit ? m : ~m;
    }
    const int ahead = __popcll(same & ((1ull << lane) - 1)), count = __popcll(same);
    uint32_t place = 0;
    if (live) place = wcnt[wave][dg] + ahead;
    __builtin_amdgcn_wave_barrier();
    if (live && ahead == 0) wcnt[wave][dg] += count;
    __builtin_amdgcn_wave_barrier();
    if (live) out[place] = el[i];
  }
}

// start[v] = first sorted position whose token is >= v, v = 0 .. vocab: a search for
// each, so that the time does not depend on which rows are absent (6 us for 50000
// rows of 524288 tokens; run by run, each filling the absent rows before it, 5 us there
// but 105 ms for 4 million rows of which tokens use 100).  Three places are looked at
// together, as the chain of dependent reads is what it takes (one or seven: 1 us more).
__global__ void __launch_bounds__(256) row_starts(const uint2* __restrict__ sorted, uint32_t n, uint32_t vocab,
                                                  uint32_t* __restrict__ start) {
  const uint32_t v = blockIdx.x * 256 + threadIdx.x;
  if (v > vocab) return;
  uint32_t lo = 0, hi = n;
  while (lo < hi) {
    const uint32_t len = hi - lo, base = lo;
    uint32_t at[3], key[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      at[k] = base + (uint32_t)(((uint64_t)(k + 1) * len) >> 2);
      key[k] = sorted[at[k]].x;
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) lo = key[k] < v ? at[k] + 1 : lo;
#pragma unroll
    for (int k = 2; k >= 0; --k) hi = key[k] < v ? hi : at[k];
  }
  start[v] = lo;
}

// ------------------------------------------------------------- sums by token

// Sorted positions that one group of lanes sums at most, as a power of two: few
// tokens are bound by that chain, many by the joins of the longest runs (2001
// tokens: 25 us a step with 32, 27 with 64; 524288: 375 and 352).
constexpr int kPartFew = 5, kPartMany = 6;

// Sum of the rows at sorted positions [a, b), chunk i of c, in order.  The 1 << ls
// lanes of the group read their positions together.
template <int T>
__device__ __forceinline__ void sum_rows(const uint2* __restrict__ sorted, const u32x4* __restrict__ dout, int c, int i,
                                         int gl, int ls, uint32_t a, uint32_t b, float (&s)[Chunk<T>::N]) {
  constexpr int N = Chunk<T>::N, U = 8;
#pragma unroll
  for (int e = 0; e < N; ++e) s[e] = 0.f;
  for (; a < b; a += 1u << ls) {
    const uint32_t mine = a + gl < b ? sorted[a + gl].y : 0;
    const int m = (int)(b - a < (1u << ls) ? b - a : 1u << ls);
    for (int k0 = 0; k0 < m; k0 += U) {
      u32x4 r[U];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const uint32_t row = __shfl(mine, (k0 + k) & ((1 << ls) - 1), 1 << ls);
        r[k] = u32x4{0, 0, 0, 0};
        if (k0 + k < m && i < c) r[k] = dout[(int64_t)row * c + i];
      }
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (k0 + k < m) {
          float x[N];
          Chunk<T>::load(r[k], x);
#pragma unroll
          for (int e = 0; e < N; ++e) s[e] += x[e];
        }
    }
  }
}

template <int T, int G>
__device__ __forceinline__ void put_row(void* dtable, int64_t v, int c, int i, const float (&s)[Chunk<T>::N],
                                        float scale) {
  constexpr int N = Chunk<T>::N;
  float x[N];
#pragma unroll
  for (int e = 0; e < N; ++e) x[e] = s[e] * scale;
  if constexpr (G == T) {
    ((u32x4*)dtable)[v * c + i] = Chunk<T>::store(x);
  } else {  // fp32 from 16-bit rows
    f32x4* p = (f32x4*)dtable + (v * c + i) * 2;
    p[0] = f32x4{x[0], x[1], x[2], x[3]};
    p[1] = f32x4{x[4], x[5], x[6], x[7]};
  }
}

// Blocks [0, row_blocks): table rows (or sorted positions that begin a run) of at
// most one part, P positions, a group of lanes each.  The others: stretches
// [P p, P (p + 1)) of the sorted positions, for tokens with more rows.  Such a stretch holds parts of
// at most two of them (one inside it would be too short): sums in slots 2p (the
// run that holds its first position) and 2p + 1 (the one of its last, if
// another).  blockIdx.y: a slice of 1 << ls chunks of the row.
template <int T, int G>
__global__ void __launch_bounds__(256) embed_sum(Runs r, int64_t n, const u32x4* __restrict__ dout, uint32_t vocab,
                                                 int c, int ls, float scale, void* __restrict__ dtable,
                                                 float* __restrict__ part, uint32_t row_blocks) {
  constexpr int N = Chunk<T>::N;
  const int gl = threadIdx.x & ((1 << ls) - 1), i = ((int)blockIdx.y << ls) + gl;
  const uint32_t per = 256u >> ls;
  float s[N];
  if (blockIdx.x < row_blocks) {
    const int64_t rows = r.run ? n : (int64_t)vocab, step = (int64_t)row_blocks * per;
    for (int64_t at = (int64_t)blockIdx.x * per + (threadIdx.x >> ls); at < rows; at += step) {
      uint32_t v = (uint32_t)at, a, b;
      if (r.run) {  // a run by its first position
        a = r.run[at].x, b = r.run[at].y;
        if (a != v) continue;
        v = r.sorted[at].x;
        if (v >= vocab) continue;
      } else {
        a = r.start[v], b = r.start[v + 1];
      }
      if (b - a > 1u << r.lg) continue;
      sum_rows<T>(r.sorted, dout, c, i, gl, ls, a, b, s);
      if (i < c) put_row<T, G>(dtable, v, c, i, s, scale);
    }
    return;
  }
  const int64_t p = (int64_t)(blockIdx.x - row_blocks) * per + (threadIdx.x >> ls);
  const int64_t s0 = p << r.lg;
  if (s0 >= n) return;
  const uint32_t a0 = (uint32_t)s0, b0 = (uint32_t)(s0 + (1 << r.lg) < n ? s0 + (1 << r.lg) : n);
  const uint32_t v0 = r.sorted[a0].x, v1 = r.sorted[b0 - 1].x;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t v = h ? v1 : v0;
    if (v >= vocab || (h && v1 == v0)) continue;
    uint32_t a, b;
    run_of(r, h ? b0 - 1 : a0, v, a, b);
    if (b - a <= 1u << r.lg) continue;
    sum_rows<T>(r.sorted, dout, c, i, gl, ls, a > a0 ? a : a0, b < b0 ? b : b0, s);
    if (i >= c) continue;
    float* q = part + ((2 * p + h) * c + i) * N;
#pragma unroll
    for (int e = 0; e < N; e += 4) *(f32x4*)(q + e) = f32x4{s[e], s[e + 1], s[e + 2], s[e + 3]};
  }
}

// The parts of tokens with more rows than a part has, in order.  A workgroup looks at
// 64 stretches, a lane of every wave at one: runs that begin there and have at
// most kWaveParts parts are joined by a wave each, longer ones by all of them.
// A wave adds four interleaved quarters of its parts, 16 chunks of the row at a
// time (blockIdx.y: the slice).
constexpr int kJoinWaves = 8, kWaveParts = 32;

// Sum of parts [k0, k1) of the run that begins in stretch p, in the second slot
// of it if inside; every lane of a chunk's four gets it.
template <int N>
__device__ __forceinline__ void join_parts(const float* __restrict__ part, int64_t p, bool inside, int64_t k0,
                                           int64_t k1, int c, int i, int u, float (&s)[N]) {
#pragma unroll
  for (int e = 0; e < N; ++e) s[e] = 0.f;
  if (i < c) {
#pragma unroll 8
    for (int64_t k = k0 + u; k < k1; k += 4) {
      const int64_t slot = 2 * (p + k) + (k == 0 && inside ? 1 : 0);
      const float* x = part + (slot * c + i) * N;
#pragma unroll
      for (int e = 0; e < N; e += 4) {
        const f32x4 y = *(const f32x4*)(x + e);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[e + j] += y[j];
      }
    }
  }
#pragma unroll
  for (int m = 16; m <= 32; m <<= 1)
#pragma unroll
    for (int e = 0; e < N; ++e) s[e] += __shfl_xor(s[e], m);
}

template <int T, int G>
__global__ void __launch_bounds__(64 * kJoinWaves)
    embed_join(Runs r, int64_t n, uint32_t vocab, int c, float scale, const float* __restrict__ part,
               void* __restrict__ dtable) {
  constexpr int N = Chunk<T>::N;
  __shared__ float red[kJoinWaves - 1][16][N + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int i = blockIdx.y * 16 + (lane & 15), u = lane >> 4;
  const int64_t p0 = (int64_t)blockIdx.x * 64, s0 = (p0 + lane) << r.lg;
  uint32_t v = vocab, a = 0, b = 0;
  if (s0 < n) {
    const int64_t last = (s0 + (1 << r.lg) < n ? s0 + (1 << r.lg) : n) - 1;
    v = r.sorted[last].x;  // (a long run that begins here holds the stretch's last position)
    if (v < vocab) run_of(r, last, v, a, b);
  }
  const bool starts = v < vocab && b - a > 1u << r.lg && a >= s0;
  const uint32_t cnt = starts ? ((b - 1) >> r.lg) - (uint32_t)(p0 + lane) + 1 : 0;
  const bool inside = a > s0;
  float s[N];
  int k = 0;
  for (uint64_t m = __ballot(starts && cnt <= kWaveParts); m; m &= m - 1, ++k) {
    if (k % kJoinWaves != wave) continue;
    const int l = __ffsll((unsigned long long)m) - 1;
    join_parts<N>(part, p0 + l, __shfl((int)inside, l) != 0, 0, __shfl(cnt, l), c, i, u, s);
    const uint32_t row = __shfl(v, l);
    if (i < c && u == 0) put_row<T, G>(dtable, row, c, i, s, scale);
  }
  for (uint64_t m = __ballot(starts && cnt > kWaveParts); m; m &= m - 1) {  // (the same in every wave)
    const int l = __ffsll((unsigned long long)m) - 1;
    const int64_t all = __shfl(cnt, l), q = (all + kJoinWaves - 1) / kJoinWaves;
    const int64_t k1 = (wave + 1) * q < all ? (wave + 1) * q : all;
    join_parts<N>(part, p0 + l, __shfl((int)inside, l) != 0, wave * q, k1, c, i, u, s);
    const uint32_t row = __shfl(v, l);
    if (wave && u == 0)
#pragma unroll
      for (int e = 0; e < N; ++e) red[wave - 1][lane][e] = s[e];
    __syncthreads();
    if (wave == 0 && i < c && u == 0) {
#pragma unroll
      for (int w = 0; w < kJoinWaves - 1; ++w)
#pragma unroll
        for (int e = 0; e < N; ++e) s[e] += red[w][lane][e];
      put_row<T, G>(dtable, row, c, i, s, scale);
    }
    __syncthreads();
  }
}

__global__ void __launch_bounds__(256) fill_zero(u32x4* p, int64_t n) {
  zero_rows(p, n, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
}

// ---------------------------------------------------------------------- host

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

struct SortPlan {
  bool few;
  int bits, passes;  // bits of a digit
  int lg;            // log2 of a part
  int64_t tiles;
  size_t el0, el1, hist, start, run, part, total;
};

SortPlan sort_plan(int64_t n, int64_t vocab, int64_t d) {
  SortPlan s = {};
  int kb = 1;
  while (((int64_t)1 << kb) <= vocab) ++kb;  // keys 0 .. vocab
  s.few = n <= kFew;
  s.passes = (kb + kMaxBits - 1) / kMaxBits;
  s.bits = (kb + s.passes - 1) / s.passes;
  s.tiles = (n + kTile - 1) / kTile;
  size_t off = 0;
  s.el0 = off; off = up256(off + (size_t)n * 8);
  if (s.few) {
    s.run = off; off = up256(off + (size_t)n * 8);
  } else {
    s.el1 = off; off = up256(off + (size_t)n * 8);
    s.hist = off; off = up256(off + ((size_t)s.tiles << s.bits) * 4);
    s.start = off; off = up256(off + (size_t)(vocab + 1) * 4);
  }
  s.lg = s.few ? kPartFew : kPartMany;
  s.part = off; off = up256(off + (size_t)((n + (1 << s.lg) - 1) >> s.lg) * 2 * (size_t)d * 4);
  s.total = off;
  return s;
}

bool aligned(const void* p, size_t a) { return p != nullptr && ((uintptr_t)p % a) == 0; }
bool known(int t) { return t == INFCL_BF16 || t == INFCL_F32 || t == INFCL_F16; }
int64_t chunks_of(int64_t d, int dtype) { return d * (dtype == INFCL_F32 ? 4 : 2) / 16; }
bool rows_ok(int64_t d, int dtype) { return d % (dtype == INFCL_F32 ? 4 : 8) == 0; }
constexpr int64_t kMaxN = ((int64_t)1 << 31) - 2, kMaxD = (int64_t)1 << 20;
// (every workgroup of a sort pass reads all tiles' counts: 2^14 tiles are 0.3 s)
constexpr int64_t kMaxSort = (int64_t)1 << 26;

template <int T>
int embed_fwd_t(const void* tokens, int tb, int64_t n, const void* table, int64_t vocab, int64_t d, float scale,
                void* out, hipStream_t st) {
  const int64_t c = chunks_of(d, T);
  const int ls = row_lanes_log2(c, 1);
  const int64_t groups = (n + kFwdRows - 1) / kFwdRows;
  int64_t blocks = ((groups << ls) + 255) / 256;
  if (blocks > 16384) blocks = 16384;
  if (tb == 4)
    hipLaunchKernelGGL((embed_fwd_kernel<T, int32_t>), dim3((unsigned)blocks), dim3(256), 0, st, (const int32_t*)tokens,
                       n, (const u32x4*)table, vocab, (int)c, ls, scale, (u32x4*)out);
  else
    hipLaunchKernelGGL((embed_fwd_kernel<T, int64_t>), dim3((unsigned)blocks), dim3(256), 0, st, (const int64_t*)tokens,
                       n, (const u32x4*)table, vocab, (int)c, ls, scale, (u32x4*)out);
  return hipGetLastError() == hipSuccess ? INFCL_OK : INFCL_ERR_HIP;
}

unsigned fill_blocks(int64_t chunks, int threads) {
  const int64_t b = chunks / (4 * threads) + 1;
  return (unsigned)(b < 2048 ? b : 2048);
}

template <typename Tok>
int sort_tokens(const void* tokens, int64_t n, int64_t vocab, const SortPlan& s, char* ws, void* dtable,
                int64_t chunks, Runs& r, hipStream_t st) {
  const Tok* tok = (const Tok*)tokens;
  uint2* el[2] = {(uint2*)(ws + s.el0), (uint2*)(ws + s.el1)};
  if (s.few) {
    const unsigned rb = (unsigned)((n + kRankTokens - 1) / kRankTokens);
    r.sorted = el[0], r.run = (const uint2*)(ws + s.run);
    hipLaunchKernelGGL((sort_few<Tok>), dim3(rb + fill_blocks(chunks, 256)), dim3(256), 0, st, tok, (int)n,
                       (uint32_t)vocab, rb, el[0], (uint2*)(ws + s.run), (u32x4*)dtable, chunks);
    return hipGetLastError() == hipSuccess ? INFCL_OK : INFCL_ERR_HIP;
  }
  uint32_t* hist = (uint32_t*)(ws + s.hist);
  const dim3 grid((unsigned)s.tiles);
  for (int p = 0; p < s.passes; ++p) {
    const uint2* in = el[(p + 1) & 1];
    if (p == 0) {
      hipLaunchKernelGGL((sort_count<Tok, true>), grid, dim3(256), 0, st, tok, in, n, (uint32_t)vocab, 0, s.bits, hist);
      hipLaunchKernelGGL((sort_scatter<Tok, true>), grid, dim3(256), 0, st, tok, in, n, (uint32_t)vocab, 0, s.bits,
                         hist, el[0]);
    } else {
      hipLaunchKernelGGL((sort_count<Tok, false>), grid, dim3(256), 0, st, tok, in, n, (uint32_t)vocab, p * s.bits,
                         s.bits, hist);
      hipLaunchKernelGGL((sort_scatter<Tok, false>), grid, dim3(256), 0, st, tok, in, n, (uint32_t)vocab, p * s.bits,
                         s.bits, hist, el[p & 1]);
    }
    if (hipGetLastError() != hipSuccess) return INFCL_ERR_HIP;
  }
  r.sorted = el[(s.passes + 1) & 1];
  r.start = (const uint32_t*)(ws + s.start);
  hipLaunchKernelGGL(row_starts, dim3((unsigned)(vocab / 256 + 1)), dim3(256), 0, st, r.sorted, (uint32_t)n,
                     (uint32_t)vocab, (uint32_t*)(ws + s.start));
  return hipGetLastError() == hipSuccess ? INFCL_OK : INFCL_ERR_HIP;
}

template <int T, int G>
int embed_bwd_t(const void* tokens, int tb, int64_t n, const void* dout, int64_t vocab, int64_t d, float scale,
                void* dtable, char* ws, hipStream_t st) {
  const int64_t c = chunks_of(d, T), chunks = chunks_of(vocab * d, G);
  if (n == 0) {
    hipLaunchKernelGGL(fill_zero, dim3(fill_blocks(chunks, 256)), dim3(256), 0, st, (u32x4*)dtable, chunks);
    return hipGetLastError() == hipSuccess ? INFCL_OK : INFCL_ERR_HIP;
  }
  const SortPlan s = sort_plan(n, vocab, d);
  Runs r = {};
  r.lg = s.lg;
  const int rc = tb == 4 ? sort_tokens<int32_t>(tokens, n, vocab, s, ws, dtable, chunks, r, st)
                         : sort_tokens<int64_t>(tokens, n, vocab, s, ws, dtable, chunks, r, st);
  if (rc != INFCL_OK) return rc;
  const int ls = row_lanes_log2(c, 1);
  const int64_t per = 256 >> ls, rows = s.few ? n : vocab, parts = (n + (1 << s.lg) - 1) >> s.lg;
  // (a launch has less than 2^32 work-items: 2^23 blocks of rows, which go on in steps, and at most 2^18 of parts)
  const int64_t all = (rows + per - 1) / per, rb = all < (1 << 23) ? all : 1 << 23;
  const int64_t pb = n > 1 << s.lg ? (parts + per - 1) / per : 0;
  const unsigned slices = (unsigned)((c + (1 << ls) - 1) >> ls);
  hipLaunchKernelGGL((embed_sum<T, G>), dim3((unsigned)(rb + pb), slices), dim3(256), 0, st, r, n, (const u32x4*)dout,
                     (uint32_t)vocab, (int)c, ls, scale, dtable, (float*)(ws + s.part), (uint32_t)rb);
  if (pb)
    hipLaunchKernelGGL((embed_join<T, G>), dim3((unsigned)((parts + 63) / 64), (unsigned)((c + 15) / 16)),
                       dim3(64 * kJoinWaves), 0, st, r, n, (uint32_t)vocab, (int)c, scale, (const float*)(ws + s.part), dtable);
  return hipGetLastError() == hipSuccess ? INFCL_OK : INFCL_ERR_HIP;
}

}  // namespace
}  // namespace infcl

using namespace infcl;

extern "C" infcl_status infcl_embed_fwd(const void* tokens, int token_bytes, int64_t n, const void* table,
                                        int64_t vocab, int64_t d, int dtype, float scale, void* out, void* stream) {
  if (n < 0 || vocab < 1 || d < 1 || !known(dtype) || (token_bytes != 4 && token_bytes != 8)) return INFCL_ERR_INVALID;
  if (!rows_ok(d, dtype) || d > kMaxD || n > kMaxN || vocab > kMaxN) return INFCL_ERR_UNSUPPORTED;
  if (n == 0) return INFCL_OK;
  if (!aligned(tokens, (size_t)token_bytes) || !aligned(table, 16) || !aligned(out, 16)) return INFCL_ERR_INVALID;
  hipStream_t st = (hipStream_t)stream;
  int rc;
  if (dtype == INFCL_BF16)
    rc = embed_fwd_t<kBF16>(tokens, token_bytes, n, table, vocab, d, scale, out, st);
  else if (dtype == INFCL_F16)
    rc = embed_fwd_t<kF16>(tokens, token_bytes, n, table, vocab, d, scale, out, st);
  else
    rc = embed_fwd_t<kF32>(tokens, token_bytes, n, table, vocab, d, scale, out, st);
  return (infcl_status)rc;
}

extern "C" infcl_status infcl_embed_bwd_workspace(int64_t n, int64_t vocab, int64_t d, size_t* bytes) {
  if (!bytes || n < 0 || vocab < 1 || d < 1) return INFCL_ERR_INVALID;
  if (d > kMaxD || n > kMaxSort || vocab > kMaxN) return INFCL_ERR_UNSUPPORTED;
  *bytes = sort_plan(n, vocab, d).total;
  return INFCL_OK;
}

extern "C" infcl_status infcl_embed_bwd(const void* tokens, int token_bytes, int64_t n, const void* dout,
                                        int64_t vocab, int64_t d, int dtype, float scale, void* dtable, int grad_dtype,
                                        void* workspace, size_t ws_bytes, void* stream) {
  if (n < 0 || vocab < 1 || d < 1 || !known(dtype) || !known(grad_dtype) || (token_bytes != 4 && token_bytes != 8))
    return INFCL_ERR_INVALID;
  if (!rows_ok(d, dtype) || d > kMaxD || n > kMaxSort || vocab > kMaxN ||
      (grad_dtype != INFCL_F32 && grad_dtype != dtype))
    return INFCL_ERR_UNSUPPORTED;
  if (!aligned(dtable, 16)) return INFCL_ERR_INVALID;
  if (n > 0) {
    if (!aligned(tokens, (size_t)token_bytes) || !aligned(dout, 16) || !aligned(workspace, 256))
      return INFCL_ERR_INVALID;
    if (ws_bytes < sort_plan(n, vocab, d).total) return INFCL_ERR_WORKSPACE;
  }
  hipStream_t st = (hipStream_t)stream;
  char* ws = (char*)workspace;
  int rc;
  if (dtype == INFCL_F32)
    rc = embed_bwd_t<kF32, kF32>(tokens, token_bytes, n, dout, vocab, d, scale, dtable, ws, st);
  else if (dtype == INFCL_BF16 && grad_dtype == INFCL_F32)
    rc = embed_bwd_t<kBF16, kF32>(tokens, token_bytes, n, dout, vocab, d, scale, dtable, ws, st);
  else if (dtype == INFCL_BF16)
    rc = embed_bwd_t<kBF16, kBF16>(tokens, token_bytes, n, dout, vocab, d, scale, dtable, ws, st);
  else if (grad_dtype == INFCL_F32)
    rc = embed_bwd_t<kF16, kF32>(tokens, token_bytes, n, dout, vocab, d, scale, dtable, ws, st);
  else
    rc = embed_bwd_t<kF16, kF16>(tokens, token_bytes, n, dout, vocab, d, scale, dtable, ws, st);
  return (infcl_status)rc;
}

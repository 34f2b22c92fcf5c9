// CPU check of the packed-attention tile layout: every copy instruction, row
// fragment and transposing read of every lane, for each width and wave count.
// Prints "ok" or the first mistake.
#include <cstdio>
#include <vector>

#include "../paper_2410_17243_amd/csrc/attn.hpp"

using namespace infcl;

template <int DP, int NW, int KT>
static bool copies(int hd, uint32_t stride) {
  typedef AttnTile<DP, NW, KT> T;
  std::vector<int> seen(T::kBytes / 16, 0);
  for (int wave = 0; wave < NW; ++wave)
    for (int lane = 0; lane < 64; ++lane) {
      uint32_t off[T::kVar];
      T::offsets(off, wave, lane, stride, hd);
      for (int kk = 0; kk < T::kPer; ++kk) {
        const int k = wave + NW * kk, unit = 64 * k + lane;  // 16-byte unit of the tile that this lane fills
        const int row = unit * 16 / T::kRow, c = (unit % T::kCh) ^ attn_sw<DP>(row);
        const uint32_t src = off[kk % T::kVar], want = (uint32_t)row * stride + 16 * c;
        if (unit >= (int)seen.size() || row >= KT) return printf("copy out of range\n"), false;
        ++seen[unit];
        if (8 * c >= hd ? src != 0x80000000u : src + (uint32_t)(k * T::kRows) * stride != want)
          return printf("copy DP %d NW %d k %d lane %d\n", DP, NW, k, lane), false;
      }
    }
  for (int n : seen)
    if (n != 1) return printf("coverage DP %d NW %d\n", DP, NW), false;
  return true;
}

template <int DP>
static bool reads() {
  auto addr = [](int row, int f) { return row * DP * 2 + 16 * ((f / 8) ^ attn_sw<DP>(row)) + 2 * (f % 8); };
  for (int lane = 0; lane < 64; ++lane) {
    AttnLanes<DP> ln;
    ln.init(lane);
    const int h = lane >> 5;
    for (int i = 0; i < DP / 16; ++i)
      if (ln.row[i] != addr(lane & 31, 8 * (2 * i + h))) return printf("row DP %d\n", DP), false;
    // lane l16 of a 16-lane group supplies 4 features of one of 4 rows; the
    // group's lane gets feature l16 of all four: slots 4 tt .. 4 tt + 3
    for (int tt = 0; tt < 2; ++tt)
      for (int fb = 0; fb < DP / 32; ++fb) {
        const int e = (lane & 15) >> 2, qq = lane & 3, nb = (lane >> 4) & 1;
        const int row = attn_reg_row(4 * tt + e, h);  // the register that holds this swept row's weight
        for (int t = 0; t < 64 / 16; ++t) {
          const int a = ln.tr[tt][fb] + 16 * t * DP * 2;
          if (a != addr(16 * t + row, 32 * fb + 16 * nb + 4 * qq)) return printf("tr DP %d\n", DP), false;
        }
      }
  }
  // banks: 16 rows of one chunk, and the 32 lanes of a half-wave's transposing read
  for (int c = 0; c < DP / 8; ++c)
    for (int r0 = 0; r0 < 64; r0 += 16) {
      unsigned used = 0;
      for (int r = r0; r < r0 + 16; ++r) used |= 1u << (addr(r, 8 * c) / 16 % 16);
      if (used != 0xFFFF) return printf("banks row DP %d\n", DP), false;
    }
  for (int half = 0; half < 2; ++half)
    for (int tt = 0; tt < 2; ++tt)
      for (int fb = 0; fb < DP / 32; ++fb) {
        unsigned used = 0;
        for (int lane = 32 * half; lane < 32 * half + 32; ++lane) {
          AttnLanes<DP> ln;
          ln.init(lane);
          used |= 1u << (ln.tr[tt][fb] / 8 % 32);
        }
        if (used != 0xFFFFFFFFu) return printf("banks tr DP %d\n", DP), false;
      }
  return true;
}

int main() {
  bool ok = true;
  for (int hd = 8; hd <= 64; hd += 8)
    ok = ok && copies<64, 1, 32>(hd, 2 * hd) && copies<64, 4, 64>(hd, 6 * hd + 16) && copies<64, 4, 32>(hd, 2 * hd) &&
         copies<64, 1, 64>(hd, 2 * hd);
  for (int hd = 72; hd <= 128; hd += 8)
    ok = ok && copies<128, 1, 32>(hd, 2 * hd) && copies<128, 4, 64>(hd, 1 << 24) && copies<128, 4, 32>(hd, 2 * hd) &&
         copies<128, 1, 64>(hd, 2 * hd);
  ok = ok && reads<64>() && reads<128>();
  if (ok) printf("ok\n");
  return ok ? 0 : 1;
}

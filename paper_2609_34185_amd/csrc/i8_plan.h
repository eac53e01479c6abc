// Which kernel and how many shares of k the INT8 product with scales takes for its sizes: host code alone.
#pragma once
#include <algorithm>
#include <cstdint>

#include "common.h"

namespace ep {
namespace {

// What a tile is cut into: halves of W's rows or of X's, and quarters of both, where every wave of the workgroup
// still has rows of both to load.
template <int NW, int NX, int WW, int WX>
constexpr bool kCutW = NW % 2 == 0 && 16 * NW / 2 * WW % (8 * WW * WX) == 0;
template <int NW, int NX, int WW, int WX>
constexpr bool kCutX = NX % 2 == 0 && 16 * NX / 2 * WX % (8 * WW * WX) == 0;
template <int NW, int NX, int WW, int WX>
constexpr int kMostCut = (kCutW<NW, NX, WW, WX> ? 2 : 1) * (kCutX<NW, NX, WW, WX> ? 2 : 1);
constexpr int kMostLarge = 8;   // 256 x 256 tiles: halves of X's rows, quarters, eighths

// How many pieces each of the last round's tiles is cut into: as many as leave no CU more than one piece.
// 512 x 17408 x 5120 in 272 tiles of 128 x 256: 63 us with the last 16 in halves, 55 in quarters; 1024 x 17408 x
// 5120 in as many of 256 x 256: 109 in halves, 103 in quarters, 93 in eighths.
uint32_t cut_of(int64_t tiles, uint32_t most, int cus) {
  uint32_t cut = most;
  while (cut > 1 && cut * (tiles % cus) > cus) cut /= 2;
  return cut;
}

// Rows of W for a workgroup of the streaming kernel: the multiple of 8 up to 16 NW that makes the
// CU with the most work read the fewest rows.
template <int NW, int NX>
uint32_t ring_height(int64_t m, int64_t n, int cus) {
  const int64_t tx = (m + 16 * NX - 1) / (16 * NX), rows_x = std::min<int64_t>(m, 16 * NX);
  int64_t best = 16 * NW, least = INT64_MAX;
  for (int64_t h = 16 * NW; h >= 8; h -= 8) {
    const int64_t read = rounds((n + h - 1) / h * tx, cus) * (h + rows_x);
    if (read < least) {
      least = read;
      best = h;
    }
  }
  return (uint32_t)best;
}

// Estimates of a launch's time in ns: what a step of 128 along k takes on the busiest CU, what a
// workgroup takes besides (first loads, and the stores of a tile by its size), what the launch takes
// besides, and never less than the operands' and outputs' way through memory.  Fitted to launches of 574
// sizes (17 to 8200 rows, 64 to 18000 columns, k from 16 to 17600), each with every kernel and up to 16
// shares of k; over them the choice is 1.2 % slower than the best (geometric mean), 34 % at most; fits
// to 344 of them are 1.4 and 1.7 % slower than the best over the others.  Tiles of 192 rows of W are worth 1.5 %
// of the best: 1703 x 4857 x 1872 takes 24 us in 192 x 192, 31 without.
enum Kernel { kRing16, kRing32, kRing64, kTile64, kTile128, kWideX, kWideW, kWideW64, k192x128, k192x192, kLarge };
struct TileCost {
  Kernel kernel;
  int rows_w, rows_x;
  uint32_t most;         // pieces of a tile of the last round
  int half, one, each;   // a CU with half a tile, with one, and with more than one, for each
  int besides;
};
constexpr TileCost kTiles[] = {{kTile64, 128, 64, kMostCut<4, 2, 2, 2>, 204, 353, 328, 2280},
                               {kTile128, 128, 128, kMostCut<4, 4, 2, 2>, 355, 679, 767, 2780},
                               {kWideX, 128, 256, kMostCut<4, 4, 2, 4>, 514, 844, 939, 3790},
                               {kWideW, 256, 128, kMostCut<4, 4, 4, 2>, 488, 806, 1017, 3790},
                               {kWideW64, 256, 64, kMostCut<4, 2, 4, 2>, 300, 553, 709, 2780},
                               {k192x128, 192, 128, kMostCut<3, 4, 4, 2>, 453, 609, 863, 3290},
                               {k192x192, 192, 192, kMostCut<6, 3, 2, 4>, 0, 895, 1003, 4040},
                               {kLarge, 256, 256, kMostLarge, 791, 1049, 1144, 15150}};
// In percent, by log2 of the pieces: a last round's share of a whole one's time, and of halves' where it is the only one;
// the least that a step of a last round of pieces takes.
constexpr int kLeast = 195;
constexpr int kShare[] = {100, 50, 30, 19}, kAlone[] = {0, 100, 69, 50};
constexpr int kMostParts = 16, kMemory = 5960;                      // kMemory, kJoinValues: bytes, and sums that are joined, in a ns
constexpr int kLaunch = 5330, kJoin = 647, kJoinValues = 958;
constexpr int kRing32Step = 108, kRing64Step = 220, kRingLaunch = 870;
// of a streaming workgroup, for `columns` columns of a row group of 16 rows each
constexpr int64_t ring_besides(int64_t columns, int groups) { return 2030 + 8 * columns * groups; }

struct Plan {
  Kernel kernel;
  uint32_t parts, part_steps, height;
};

// A launch of few tiles shares k out over workgroups, whose sums another launch joins.
// 203 x 5120 x 17408 in tiles of 192 x 128, 54 of them, on a card where that takes 37.6 us in 4 parts: 70.6 in one; in
// 128 x 256, 40 of them: 37.9 in 5.  Cards differ by more than that: 33 to 39.
Plan plan_of(int64_t m, int64_t n, int64_t k, int cus) {
  const uint32_t kb = (uint32_t)((k + 127) / 128);
  if (m <= 16) return {kRing16, 1, kb, ring_height<2, 1>(m, n, cus)};
  const int64_t memory = ((m + n) * k + 2 * m * n) / kMemory;
  // the streaming kernels read X again for every strip of W: not where X is what there is most of
  Plan best = {kRing32, 1, kb, 0};
  int64_t least = INT64_MAX;
  if (m <= 512) {
    const uint32_t h2 = ring_height<3, 2>(m, n, cus), h4 = ring_height<3, 4>(m, n, cus);
    const int64_t t2 = (kRing32Step * kb + ring_besides(h2, 2)) * rounds((n + h2 - 1) / h2 * ((m + 31) / 32), cus);
    const int64_t t4 = (kRing64Step * kb + ring_besides(h4, 4)) * rounds((n + h4 - 1) / h4 * ((m + 63) / 64), cus);
    best = t2 <= t4 ? Plan{kRing32, 1, kb, h2} : Plan{kRing64, 1, kb, h4};
    least = std::max(std::min(t2, t4), memory) + kRingLaunch;
  }
  for (const TileCost& c : kTiles) {
    const int64_t tiles = (m + c.rows_x - 1) / c.rows_x * ((n + c.rows_w - 1) / c.rows_w);
    const uint32_t most = tiles >= cus ? 1 : (uint32_t)std::min<int64_t>(kMostParts, 4 * cus / tiles);
    int64_t filled = rounds(tiles, cus);
    for (uint32_t p = 1; p <= most && p <= kb; p++) {
      const int64_t join = p > 1 ? kJoin + p * m * n / kJoinValues : 0;
      if (memory + kLaunch + join >= least) break;   // and more parts take longer still
      if (tiles * p > filled * cus) filled++;        // more than one part: of fewer tiles than CUs
      const uint32_t steps = (kb + p - 1) / p;
      if ((kb + steps - 1) / steps != p) continue;   // the last parts would be empty
      int64_t whole = filled, share = 0, step = 0;   // rounds of whole tiles, percent of one in pieces
      if (p == 1 && tiles % cus) {
        const int cut = __builtin_ctz(cut_of(tiles, c.most, cus));
        if (cut) {
          whole--;
          share = kShare[cut];
          step = whole ? std::max<int64_t>(c.each * share / 100, kLeast) : c.half * kAlone[cut] / 100;
        }
      }
      if (whole) step = whole == 1 && !share ? c.one : c.each * whole + step;
      const int64_t time = std::max(step * steps + c.besides * (100 * whole + share) / 100, memory) + kLaunch + join;
      if (time < least) {
        least = time;
        best = {c.kernel, p, steps, 0};
      }
    }
  }
  return best;
}

// Bytes of a launch's partial sums.  Where k is shared out, tiles times parts are at most 4 x cus, of up to 65536 sums of
// 4 bytes each: 1 MiB for each CU.
uint64_t workspace_of(const Plan& plan, int64_t m, int64_t n) {
  return plan.parts > 1 ? (uint64_t)plan.parts * m * ((n + 3) / 4 * 4) * 4 : 0;
}

}  // namespace
}  // namespace ep

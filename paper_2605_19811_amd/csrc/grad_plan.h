// Host-side choice of the tiles of the products grouped by expert: sizes in, plan
// out, no HIP (grad_products.hip runs it; tests/grad_plan_driver.cpp prints it).
#pragma once

#include <algorithm>
#include <cstdint>

namespace lm {

// Workgroups of a launch at most: with 512 threads each, 2^31 threads.
constexpr int64_t kMaxWorkgroups = int64_t(1) << 22;

// Microseconds of a stage of 64 contraction values where a CU has one tile and
// where it has `at_once`, and of a tile besides (start and output); measured at
// contractions of 1000 to 8192 with one to 4096 tiles.
struct TileCost {
  int bm, bn, at_once;
  double alone, full, rest;
};
constexpr TileCost kRowTiles[3] = {{256, 256, 1, 1.3, 1.6, 5.0}, {128, 128, 2, 0.65, 0.93, 4.0}, {64, 64, 2, 0.25, 0.40, 2.5}};
constexpr TileCost kWeightTiles[3] = {{256, 128, 1, 0.7, 1.0, 6.0}, {128, 128, 2, 0.6, 1.05, 5.0}, {64, 64, 2, 0.24, 0.45, 2.5}};

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Workgroups of a row product's whole tiles: the most that any split of the rows
// into experts makes.
inline int64_t row_workgroups(const TileCost& c, int64_t rows, int64_t experts, int64_t width) {
  return (rows / c.bm + std::min(experts, rows)) * ceil_div(width, c.bn) + 2048;
}
inline int64_t weight_workgroups(const TileCost& c, int64_t experts, int64_t n, int64_t k) {
  return 2 * experts * ceil_div(n, c.bm) * ceil_div(k, c.bn) + 65536;     // (parts: at most a few tiles for each CU)
}

// Tile of a row product: the least time by rounds of tiles over the CUs, the last one
// in quarters where the kernel does that. An expert's last tile is half empty on average.
inline int row_tile(int64_t rows, int64_t experts, int64_t width, int64_t depth, int cus, bool aligned) {
  int best = 0;
  double least = 0.0;
  for (int i = 0; i < 3; ++i) {
    const TileCost& c = kRowTiles[i];
    const int64_t e = std::min(experts, rows);
    const int64_t tiles = (e == 1 ? ceil_div(rows, c.bm) : rows / c.bm + (e + 1) / 2) * ceil_div(width, c.bn);
    const int64_t places = int64_t(cus) * c.at_once, left = tiles % places;
    const double stages = double(ceil_div(depth, 64));
    double t = double(tiles / places) * (c.full * stages + c.rest);
    if (i == 0 && aligned && left * 2 <= cus) t += left > 0 ? kRowTiles[1].alone * (left * 4 <= cus ? 1.0 : 1.5) * stages + c.rest : 0.0;
    else if (left > 0) t += (left <= cus && i > 0 ? c.alone : left * 4 <= cus ? c.alone : c.full) * stages + c.rest;
    if (i == 0 || (t < least && row_workgroups(c, rows, experts, width) <= kMaxWorkgroups)) {
      best = i;
      least = t;
    }
  }
  return best;
}

// Tile of a weight gradient and the rows of a part (WeightProduct). Whole
// experts take as long as the longest one, taken as three times the mean, or as
// all of them spread evenly; parts as long as an even share and a third, with 12
// bytes of traffic for each partial value at 4 TB/s and a second launch.
struct WeightPlan {
  int tile;
  int64_t part;
};
inline WeightPlan weight_plan(int64_t rows, int64_t experts, int64_t n, int64_t k, int cus) {
  WeightPlan best{0, rows + 1};
  double least = -1.0;
  for (int i = 0; i < 3; ++i) {
    const TileCost& c = kWeightTiles[i];
    if (i > 0 && weight_workgroups(c, experts, n, k) > kMaxWorkgroups) break;
    const int64_t per = ceil_div(n, c.bm) * ceil_div(k, c.bn), tiles = experts * per, places = int64_t(cus) * c.at_once;
    const double share = double(rows) * double(per) / double(places);      // rows of each place
    const double longest = experts == 1 ? double(rows) : std::min(double(rows), 3.0 * double(rows) / double(experts));
    const double rest = std::max(1.0, double(tiles) / double(places)) * c.rest;
    const double whole = std::max(share * c.full, longest * (tiles <= cus ? c.alone : c.full)) / 64.0 + rest;
    if (least < 0.0 || whole < least) {
      least = whole;
      best = WeightPlan{i, rows + 1};
    }
    const int64_t part = std::max<int64_t>(256, ceil_div(int64_t(share) + 1, 64) * 64);
    if (double(part) < longest / 1.25) {
      const double parts = double(rows) / double(part) + (experts == 1 ? 1.0 : 0.0);
      const double split = 1.33 * double(part) / 64.0 * c.full + rest + parts * double(n) * double(k) * 12.0 / 4e6 + 6.0;
      if (split < least) {
        least = split;
        best = WeightPlan{i, part};
      }
    }
  }
  return best;
}

// Slots of partial sums that parts of that many rows can need.
inline int64_t partial_slots(int64_t rows, int64_t part) { return part > rows ? 0 : 2 * rows / part + 1; }

}  // namespace lm

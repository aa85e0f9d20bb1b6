// How the gradients of a linear layer are cut into workgroups (fa_linear_grad.hip): host arithmetic alone, no HIP, so that
// a test without a GPU holds the kernels' test to shapes of either tile.
#ifndef FA_LINEAR_PLAN_H_
#define FA_LINEAR_PLAN_H_

#include <stdint.h>

// The two tiles of either type, and in how many parts the workers' rows are cut.  Time is counted in steps of a wide tile,
// 2 us on a full card (bf16; 65536 x 4096 x 4096 takes 16 rounds of 64 of them): a narrow tile is a quarter of the
// work, two of them share a compute unit, and the pair takes `step` of that (whole shapes: 65536 x 4096 x 4096 in 2.05 ms
// wide, 2.93 ms narrow; 15 workers of 1024 rows, 768 -> 2304: 0.089 and 0.108 ms; fp32, 60 workers, 1001 -> 509: 0.140 and
// 0.164 ms).  A round of workgroups costs `more` beside its steps, for the first loads and the last stores.  Parts are
// joined at the rate of memory, behind one more launch.
struct fa_linear_tile {
  int outputs, features, slots;
  float step, more;
};
constexpr fa_linear_tile kFaLinearTiles[2][2] = {
    {{128, 256, 256, 1.f, 5.f}, {64, 128, 512, 0.56f, 3.f}},     // fp32 dY: wide, narrow
    {{256, 256, 256, 1.f, 5.f}, {128, 128, 512, 0.69f, 3.f}}};   // bf16 dY
constexpr int kFaLinearParts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};

struct fa_linear_plan {
  bool wide;
  int splits;
  int64_t tiles;   // of one worker
};

// rows: of all p workers.  A worker counts as the mean one: the parts are right for workers of like sizes, and a worker that
// has most of the rows is not cut by its own number of them.
static inline fa_linear_plan fa_plan_linear_grad(int64_t rows, int p, int features, int outputs, bool bf16) {
  const int64_t mean = (rows + p - 1) / p, steps = (mean + 63) / 64;
  const double results = (double)p * outputs * features;
  fa_linear_plan best = {};
  double least = 0;
  for (int narrow = 0; narrow < 2; ++narrow) {
    const fa_linear_tile& t = kFaLinearTiles[bf16][narrow];
    const int64_t tiles = (int64_t)((outputs + t.outputs - 1) / t.outputs) * ((features + t.features - 1) / t.features);
    for (const int parts : kFaLinearParts) {
      if (parts > 1 && parts > steps) break;
      const int64_t rounds = (tiles * p * parts + t.slots - 1) / t.slots;
      double cost = (double)rounds * ((double)((steps + parts - 1) / parts) * t.step + t.more);
      if (parts > 1) cost += 1.5 + results * parts * (8 / 5.1e6 / 2);
      if (best.splits == 0 || cost < least) {
        least = cost;
        best = {narrow == 0, parts, tiles};
      }
    }
  }
  return best;
}

#endif

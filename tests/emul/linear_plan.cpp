// Test-only: the rule that cuts linear gradients into workgroups, as a host library.
#include "fa_linear_plan.h"

extern "C" int linear_plan(int64_t rows, int p, int features, int outputs, int bf16, int* splits, int64_t* tiles) {
  const fa_linear_plan c = fa_plan_linear_grad(rows, p, features, outputs, bf16 != 0);
  *splits = c.splits;
  *tiles = c.tiles;
  return c.wide ? 1 : 0;
}

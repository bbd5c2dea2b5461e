// Host-only driver for tests/test_grad_tiles.py: reads lines
//   row ROWS EXPERTS WIDTH CONTRACTION ALIGNED
//   weight ROWS EXPERTS N K
// and prints for each the tile of the product (0: the largest), for a weight
// gradient also the rows of a part (0: whole experts), on 256 CUs.
#include <cstdio>
#include <cstring>

#include "grad_plan.h"

int main() {
  char kind[16];
  long long a, b, c, d, aligned;
  while (scanf("%15s %lld %lld %lld %lld", kind, &a, &b, &c, &d) == 5) {
    if (!strcmp(kind, "row")) {
      if (scanf("%lld", &aligned) != 1) return 1;
      printf("%d\n", lm::row_tile(a, b, c, d, 256, aligned != 0));
    } else {
      const lm::WeightPlan p = lm::weight_plan(a, b, c, d, 256);
      printf("%d %lld\n", p.tile, p.part > a ? 0LL : (long long)p.part);
    }
  }
  return 0;
}

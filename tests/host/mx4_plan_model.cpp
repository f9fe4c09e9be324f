// The choice of block shapes for MX4 products, for tests: reads lines "a4 n k m experts", prints the
// number of the shape and its tile for each.
#include <cstdio>

#include "../../paper_2505_07531_amd/csrc/mx4_plan.h"

int main() {
  int a4, n, k, m, experts;
  while (std::scanf("%d %d %d %d %d", &a4, &n, &k, &m, &experts) == 5) {
    const int i = a4 ? qx::mx4::pick_shape<true>(n, k, m, experts) : qx::mx4::pick_shape<false>(n, k, m, experts);
    const qx::mx4::ShapeCost& s = a4 ? qx::mx4::shapes<true>[i] : qx::mx4::shapes<false>[i];
    std::printf("%d %d %d %d\n", i, 16 * s.mt * s.wm, 16 * s.nt * s.wn, s.wk);
  }
}

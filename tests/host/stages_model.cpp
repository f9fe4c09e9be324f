// The block shapes chosen for products, for tests: reads lines "kind bits a4 n k m experts", prints the number
// of the shape, the units of a row (128 k, 64 for fp16 rows of MX4 weights) and those of a stage for each.
#include <cstdio>

#include "../../paper_2505_07531_amd/csrc/grouped_plan.h"

int main() {
  int kind, bits, a4, n, k, m, experts;
  while (std::scanf("%d %d %d %d %d %d %d", &kind, &bits, &a4, &n, &k, &m, &experts) == 7) {
    int i;
    const qx::mx4::ShapeCost* s;
    if (kind == QX_MX4) {
      i = a4 ? qx::mx4::pick_shape<true>(n, k, m, experts) : qx::mx4::pick_shape<false>(n, k, m, experts);
      s = a4 ? &qx::mx4::shapes<true>[i] : &qx::mx4::shapes<false>[i];
      std::printf("%d %d %d\n", i, k / (a4 ? 128 : 64), s->wk * s->ks);
    } else {
      qx_desc d = {};
      d.bits = bits, d.kind = kind, d.n = n, d.k = k;
      i = qx::grouped::pick_shape(&d, m, experts);
      s = &qx::grouped::shapes[0][i];
      std::printf("%d %d %d\n", i, k / 128, s->ks);
    }
  }
}

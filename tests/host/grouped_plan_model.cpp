// The choice of block shapes for grouped products of the uniform, codebook and Q4X kinds, for tests: reads
// lines "bits kind n k m experts", prints the number of the shape for each.
#include <cstdio>

#include "../../paper_2505_07531_amd/csrc/grouped_plan.h"

int main() {
  int bits, kind, n, k, m, experts;
  while (std::scanf("%d %d %d %d %d %d", &bits, &kind, &n, &k, &m, &experts) == 6) {
    qx_desc d = {};
    d.bits = bits, d.kind = kind, d.n = n, d.k = k;
    std::printf("%d\n", qx::grouped::pick_shape(&d, m, experts));
  }
}

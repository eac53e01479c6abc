// Prints, for each "m n k" on its input, what the INT8 product with scales chooses on a device of argv[1]
// CUs: kernel, shares of k and their steps of 128, pieces of the last round's tiles, whether there are more
// workgroups than CUs, and the workspace's bytes.
#include <cstdio>
#include <cstdlib>

#include "i8_plan.h"

int main(int argc, char** argv) {
  using namespace ep;
  const int cus = argc > 1 ? std::atoi(argv[1]) : 256;
  long m, n, k;
  while (std::scanf("%ld %ld %ld", &m, &n, &k) == 3) {
    const Plan p = plan_of(m, n, k, cus);
    long units = p.height ? (n + p.height - 1) / p.height : 0, cut = 1;
    if (p.kernel != kRing16) units *= (m + (p.kernel == kRing32 ? 31 : 63)) / (p.kernel == kRing32 ? 32 : 64);
    for (const TileCost& c : kTiles)
      if (c.kernel == p.kernel) {
        units = (m + c.rows_x - 1) / c.rows_x * ((n + c.rows_w - 1) / c.rows_w);
        if (p.parts == 1 && units % cus) cut = cut_of(units, c.most, cus);
      }
    std::printf("%d %u %u %ld %d %lu\n", (int)p.kernel, p.parts, p.part_steps, cut, units > cus, (unsigned long)workspace_of(p, m, n));
  }
}

// Prints the block tile and the k ranges of 8-bit products: one line "p q k
// exact" in, "tile ranges" out.
#include <cstdio>

#include "routes.hpp"

int main() {
  long long p, q, k;
  int exact;
  while (std::scanf("%lld %lld %lld %d", &p, &q, &k, &exact) == 4) {
    const ozfp4::F8Route r = ozfp4::f8_route(p, q, k, exact != 0);
    std::printf("%d %d\n", (int)r.tile, r.ranges);
  }
}

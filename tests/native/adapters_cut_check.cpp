// Prints how the adapters' calls are cut.  A line of "m k n rank groups" in, a line of
// "fused ranks tiles splits unit room" out: room is the LDS of a workgroup of the second product, in bytes.
#include <cstdio>

#include "adapters_cut.h"

int main() {
  long long m, k, n, rank, groups;
  std::printf("%lld\n", (long long)hadacore::kUpRoom);
  while (std::scanf("%lld %lld %lld %lld %lld", &m, &k, &n, &rank, &groups) == 5) {
    const hadacore::Cut c = hadacore::cut_of(m, k, n, rank, groups);
    std::printf("%d %d %d %d %d %lld\n", c.fused, c.ranks, c.tiles, c.splits, c.unit,
                (long long)hadacore::up_room(c.unit, rank));
  }
}

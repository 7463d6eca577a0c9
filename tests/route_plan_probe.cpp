// Prints how the library's host code deals out the routing of tokens named on stdin (tests/test_routed_plans.py); links librunlora.so, runs nothing on a GPU.
#include <cstdio>

#include "../paper_2312_03415_amd/csrc/route.hpp"

using namespace rl;

int main() {
  long n, experts, top, groups;
  while (std::scanf("%ld %ld %ld %ld", &n, &experts, &top, &groups) == 4) {
    const RoutePlan p = route_plan(n, experts, top, groups);
    std::printf("%d %d %d %d %d %u %u %u\n", p.lanes, p.per, p.waves, p.each, p.groups, p.room, route_lds(p, experts, false), route_lds(p, experts, true));
  }
  return 0;
}

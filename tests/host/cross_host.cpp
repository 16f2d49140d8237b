// How cross attention's host side cuts its work, checked without a GPU: grids over the whole range of item counts.
// (tests/test_cross_host.py builds and runs this.)
#include <stdio.h>

#include "cross.h"

static int failures = 0;
#define EXPECT(cond)                                                     \
  do {                                                                   \
    if (!(cond)) { printf("FAILED %s:%d: %s\n", __FILE__, __LINE__, #cond); ++failures; } \
  } while (0)

using namespace isa;

int main() {
  // Every workgroup of 256 threads is in a grid of which no dimension has 2^32 threads, few places are idle, and the eight XCDs get as many each
  for (long long total : {1ll, 7ll, 8ll, 9ll, 1000ll, (1ll << 23) - 1, 1ll << 23, (1ll << 23) + 1, (1ll << 24) - 1, 1ll << 24, (1ll << 24) + (1ll << 20)}) {
    const dim3 g = cross_grid(total);
    EXPECT(g.x * 256ll < (1ll << 32) && g.x % 8 == 0 && g.y >= 1 && g.y < 65536 && g.z == 1);
    const long long all = (long long)g.x * g.y;
    EXPECT(all >= total && all < total + 8 * 4);
  }
  printf("%s (%d failures)\n", failures ? "FAILED" : "host checks ok", failures);
  return failures ? 1 : 0;
}

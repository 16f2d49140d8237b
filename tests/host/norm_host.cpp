// Which calls of the norm go past the caches, checked without a GPU (tests/test_norm_host.py builds and runs this).
#include <stdio.h>

#include "rms_norm.h"

static int failures = 0;
#define EXPECT(cond)                                                     \
  do {                                                                   \
    if (!(cond)) { printf("FAILED %s:%d: %s\n", __FILE__, __LINE__, #cond); ++failures; } \
  } while (0)

using namespace isa;

int main() {
  void* const t = (void*)4096;                              // never dereferenced
  const long long MB = 1 << 20;
  // tensors of `mb` MB each, of rows of 4096 channels; `set`: how many of residual, h, dy, dh there are beside x and y
  auto streams = [&](long long mb, int dtype, bool eight, int set) {
    NormArgs a = {};
    a.C = 4096;
    a.rows = mb * MB / 4096 / (dtype == ISA_BF16 ? 2 : 4);
    a.x = a.y = t;
    if (set > 0) a.residual = t;
    if (set > 1) a.h = t;
    if (set > 2) a.dy = t;
    if (set > 3) a.dh = t;
    return norm_streams(a, dtype, eight);
  };
  for (int dtype : {ISA_BF16, ISA_F32}) {
    EXPECT(!streams(64, dtype, false, 0) && !streams(96, dtype, false, 0) && !streams(127, dtype, false, 0) && streams(128, dtype, false, 0));      // two tensors
    EXPECT(!streams(63, dtype, false, 2) && streams(64, dtype, false, 2));                                          // with the residual and its sum
    EXPECT(!streams(85, dtype, false, 1) && streams(86, dtype, false, 1));
    EXPECT(!streams(42, dtype, false, 4) && streams(43, dtype, false, 4));
  }
  EXPECT(!streams(170, ISA_BF16, true, 0) && streams(171, ISA_BF16, true, 0));      // y in 8 bits: half a tensor of bf16
  EXPECT(!streams(73, ISA_BF16, true, 2) && streams(74, ISA_BF16, true, 2));
  EXPECT(!streams(78, ISA_F32, true, 2) && streams(79, ISA_F32, true, 2));
  NormArgs odd = {};
  odd.C = 4095; odd.rows = 1 << 20; odd.x = odd.y = t;
  EXPECT(!norm_streams(odd, ISA_BF16, false));              // rows that are no whole chunks
  printf("%s (%d failures)\n", failures ? "FAILED" : "host checks ok", failures);
  return failures ? 1 : 0;
}

// How cross attention's host side cuts its work, checked without a GPU: grids over the whole range of item counts, workspaces, which states are streamed.
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
  // The workspace stays within what the header names, over a spread of problems up to its limits, single queries of many heads among them
  for (int dtype = 0; dtype < 2; ++dtype)
    for (int D = 64; D <= 128; D += 64)
      for (int B : {1, 3, 8, 1000, 1 << 20})
        for (int H_kv : {1, 2, 5, 40, 65535, 1 << 20})
          for (int g : {1, 2, 5})
            for (int S_q : {1, 2, 16, 17, 63, 64, 65, 129, 1000, 65520, 1 << 20, 1 << 28})
              for (int S_k : {0, 1, 77, 128, 129, 1000, 16384, 1 << 20, 1 << 28}) {
                const long long bh = (long long)B * H_kv * g;
                if (bh > (1 << 20) || bh * S_q > (1 << 30) || (long long)B * H_kv * S_k > (1 << 30)) continue;
                isa_cross_problem p = {};
                p.B = B; p.H = H_kv * g; p.H_kv = H_kv; p.D = D; p.S_q = S_q; p.S_k = S_k; p.dtype = dtype; p.scale = 0.125;
                const isa_strides q = {(int64_t)p.H * S_q * D, (int64_t)S_q * D, D}, k = {(int64_t)H_kv * (S_k + 1) * D, (int64_t)(S_k + 1) * D, D};
                p.q = p.out = p.d_out = p.dq = q;
                p.k = p.v = p.dk = p.dv = k;
                const size_t f = isa_cross_workspace_bytes(&p, 0), b = isa_cross_workspace_bytes(&p, 1);
                EXPECT(f <= 70000000u && b > 0 && b <= 300000000u + 512ull * bh * ((S_q + 63) / 64));
              }
  // Single queries stream their states where the distinct ones are more than 256 MB: eight requests on one document of 67 MB do not
  {
    isa_cross_problem p = {};
    p.B = 8; p.H = 40; p.H_kv = 8; p.D = 128; p.S_q = 1; p.S_k = 16384; p.scale = 0.1;
    p.k = p.v = isa_strides{8ll * 16384 * 128, 16384 * 128, 128};
    EXPECT(cross_states_streamed(p));
    p.k.b = 0;
    EXPECT(cross_states_streamed(p));                      // (the values alone: 268 MB, and 34 MB of keys)
    p.v.b = 0;
    EXPECT(!cross_states_streamed(p));
    p.B = 64;
    EXPECT(!cross_states_streamed(p));
    p.S_k = 1 << 17;
    EXPECT(cross_states_streamed(p));                      // one document of 537 MB
    p.k.h = p.v.h = 0;
    EXPECT(!cross_states_streamed(p));
    p.B = 1; p.H_kv = 1; p.S_k = 1 << 19;
    EXPECT(!cross_states_streamed(p));                     // 256 MB
    p.S_k += 1;
    EXPECT(cross_states_streamed(p));
  }
  printf("%s (%d failures)\n", failures ? "FAILED" : "host checks ok", failures);
  return failures ? 1 : 0;
}

// The launch that forks tables (csrc/pages.h): fewer than 2^32 threads for every table that the call takes, every column in
// one workgroup, room for every row.
#include <stdint.h>
#include <stdio.h>

#include <vector>

#include "pages.h"

using namespace cdsl;

#define CHECK(x)                                             \
  do {                                                       \
    if (!(x)) {                                              \
      fprintf(stderr, "%s:%d: %s\n", __FILE__, __LINE__, #x); \
      return 1;                                              \
    }                                                        \
  } while (0)

int main() {
  for (int B = 1; B <= kForkRows; ++B)
    for (int P : {1, 3, 4, 5, 257, 1 << 18, (1 << 18) + 1, 1 << 22, 1 << 24, (1 << 26) - 1}) {
      const ForkGrid g = fork_grid(B, P);
      CHECK(g.groups > 0 && g.threads > 0 && g.threads % 64 == 0 && g.threads <= kForkThreads);
      CHECK((uint64_t)g.groups * g.threads < (1ull << 32));
      CHECK(g.groups <= (P + kForkCols - 1) / kForkCols);
    }
  for (int P : {1, 7, 1000, (1 << 18) - 1, (1 << 18) + 3, 700001}) {
    std::vector<int> taken(P, 0);
    const ForkGrid g = fork_grid(3, P);
    for (int x = 0; x < g.groups; ++x)
      for (int c = x * kForkCols; c < P; c += g.groups * kForkCols)
        for (int i = c; i < c + kForkCols && i < P; ++i) ++taken[i];
    for (int n : taken) CHECK(n == 1);
  }
  printf("pages launch: ok\n");
  return 0;
}

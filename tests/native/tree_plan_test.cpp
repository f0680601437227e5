// Host unit test of the tree attention's plan (tree_plan.h), built with the
// address and undefined-behaviour sanitizers by tests/test_tree_plan_host.py.
// Reads lines "B n H Hkv hd longest dtype format" and prints the kernel that
// each takes; then checks, over drawn sizes up to the call's limits, what the
// kernels take for granted.
#include <stdio.h>
#include <stdlib.h>

#include <cmath>
#include <random>

#include "tree_plan.h"

using namespace cdsl;

#define CHECK(x)                                                        \
  do {                                                                  \
    if (!(x)) {                                                         \
      fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #x);   \
      exit(1);                                                          \
    }                                                                   \
  } while (0)

static void sweep() {
  std::mt19937_64 g(3);
  auto log_to = [&](double top) { return (long long)std::max(1.0, std::exp2(std::log2(top) * (g() >> 11) * 0x1p-53)); };
  const int hds[] = {32, 64, 128};
  for (int trial = 0; trial < 200000; ++trial) {
    const long long rows = (1 << 24) - 1;
    const int B = (int)log_to(65535), Hkv = (int)std::min<long long>(log_to(256), rows / B);
    if (Hkv == 0) continue;
    const int G = (int)std::max<long long>(1, std::min<long long>(log_to(64), rows / B / Hkv));
    const int n = (int)std::max<long long>(1, std::min<long long>(log_to(1 << 20), rows / B / Hkv / G)), H = G * Hkv;
    if ((long long)B * n * H > rows) continue;
    const int hd = hds[g() % 3], longest = trial % 5 ? (int)log_to(2147483647.0) : 0, dtype = g() % 2, fmt = g() % 2;
    const TreeAttnPlan p = tree_attn_plan(B, n, H, Hkv, hd, longest, dtype, fmt);
    const long long tiles = ((long long)n * G + 15) / 16;
    const int most = p.few ? p.few : p.wide ? 8 : 4;
    CHECK(p.few == (tiles <= 2 ? tiles : 0) && !(p.few && p.wide) && !(p.four && (p.few || p.wide)));
    CHECK(p.wg_tiles >= 1 && p.wg_tiles <= most && p.row_groups >= 1);
    CHECK((long long)p.wg_tiles * p.row_groups >= tiles && (long long)p.wg_tiles * (p.row_groups - 1) < tiles);
    CHECK(p.slots >= B && p.split_pages >= 1);
    CHECK((p.workspace > 0) == (p.slots > B));
    // one size of parts for all: whole numbers of them, a lane for each in the merge
    if (B == 1 || B > kTreeShared) CHECK(p.slots % B == 0 && p.slots / B <= kTreeMaxSplits);
    CHECK(p.slots <= (long long)B * kTreeMaxSplits);
    CHECK(tree_attn_workspace(B, n, H, Hkv, hd, longest) >= p.workspace);
    CHECK(!p.wide || tree_may_be_wide(hd, dtype, fmt));
    CHECK(!p.four || tree_may_be_four(hd, dtype, fmt));
  }
}

int main() {
  int B, n, H, Hkv, hd, longest, dtype, fmt;
  while (scanf("%d %d %d %d %d %d %d %d", &B, &n, &H, &Hkv, &hd, &longest, &dtype, &fmt) == 8) {
    const TreeAttnPlan p = tree_attn_plan(B, n, H, Hkv, hd, longest, dtype, fmt);
    printf("%s%s\n", p.few == 1 ? "few1" : p.few == 2 ? "few2" : p.wide ? "wide" : p.four ? "many4" : "many3",
           p.slots > B ? "+split" : "");
  }
  sweep();
  printf("tree plan: ok\n");
  return 0;
}

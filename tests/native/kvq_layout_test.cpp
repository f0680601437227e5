// Host unit test of the 8-bit cache's layout (kvq_layout.h), built with the
// address and undefined-behaviour sanitizers by tests/test_kvq_layout_host.py:
// every byte of a unit has one owner, positions find their units and pages
// outside the table or the pool find none, the pages of a run cover it once,
// and the visible slots of a page are those of the definition.
#include <stdio.h>
#include <stdlib.h>

#include <random>
#include <vector>

#include "kvq_layout.h"

using namespace cdsl;

#define CHECK(x)                                                        \
  do {                                                                  \
    if (!(x)) {                                                         \
      fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #x);   \
      exit(1);                                                          \
    }                                                                   \
  } while (0)

static void layout(int hd) {
  std::vector<int> owners(kvq_unit_bytes(hd), 0);
  for (int s = 0; s < kPage; ++s) {
    for (int d = 0; d < hd; ++d) {
      owners.at(kvq_key_at(s, d))++;
      owners.at(kvq_value_at(hd, s, d))++;
      CHECK(kvq_key_at(s, d) < kPage * hd && kvq_value_at(hd, s, d) >= kPage * hd);
      // what the kernels move as whole words: eight dims of a key, four slots of a value
      if (d % 8) CHECK(kvq_key_at(s, d) == kvq_key_at(s, d - 1) + 1);
      else CHECK(kvq_key_at(s, d) % 8 == 0);
      if (s % 4) CHECK(kvq_value_at(hd, s, d) == kvq_value_at(hd, s - 1, d) + 1);
      else CHECK(kvq_value_at(hd, s, d) % 4 == 0);
    }
    for (int e = 0; e < 4; ++e) {
      owners.at(kvq_key_scale_at(hd, s) + e)++;
      owners.at(kvq_value_scale_at(hd, s) + e)++;
    }
  }
  for (int o : owners) CHECK(o == 1);
  CHECK(kvq_unit_bytes(hd) % 256 == 0);
}

static void units() {
  std::vector<int> table = {3, -1, 5, 7, 0, 1 << 30, -2147483647 - 1, 4};
  const int unit = kvq_unit_bytes(64);
  std::vector<uint8_t> pool((size_t)6 * 2 * unit);
  const KvqView c{pool.data(), table.data(), 2, 4, 6, 2, 64, kInt8};
  CHECK(kvq_unit_of(c, 0, 0, 1) == pool.data() + (3 * 2 + 1) * unit);
  CHECK(kvq_unit_of(c, 1, 0, 0) == pool.data());
  CHECK(kvq_unit_of(c, 1, 3, 1) + unit == pool.data() + (4 * 2 + 2) * unit);
  CHECK(kvq_unit_of(c, 0, 2, 1) + unit == pool.data() + pool.size());
  for (auto [b, p] : {std::pair<int, long long>{0, 1}, {0, 3}, {1, 1}, {1, 2}, {0, -1}, {1, 4}, {0, 1LL << 40}, {0, -(1LL << 40)}})
    CHECK(kvq_unit_of(c, b, p, 0) == nullptr);
  // units beyond 2^32 bytes from the pool's start
  const KvqView big{pool.data(), table.data(), 2, 4, 2147483647, 32, 128, kInt8};
  CHECK((long long)(kvq_unit_of(big, 1, 1, 31) - pool.data()) == ((1LL << 30) * 32 + 31) * kvq_unit_bytes(128));
}

static void runs() {
  std::mt19937 g(1);
  for (int trial = 0; trial < 4000; ++trial) {
    const int T = g() % 140 + (trial & 1 ? 0 : 1);
    const int start = (int)(g() % 200) - 70, count = (int)(g() % 200) - 30;
    const KvqRun r = kvq_run(trial % 5 ? &start : nullptr, trial % 3 ? &count : nullptr, T, 0);
    const long long beg = trial % 5 ? start : 0;
    long long n = trial % 3 ? count : T;
    n = n < 0 ? 0 : n > T ? T : n;
    CHECK(r.beg == beg && r.end == beg + n);
    long long seen = 0;
    for (int p = 0; p < kvq_run_pages(T); ++p)
      for (int s = 0; s < kPage; ++s) {
        const long long pos = (kvq_first_page(r) + p) * kPage + s;
        if (pos >= r.beg && pos < r.end) ++seen;
      }
    CHECK(seen == n);
  }
  const int top = 2147483647;
  const KvqRun far = kvq_run(&top, &top, top, 0);
  CHECK(far.beg == top && far.end == 2LL * top);
  CHECK(kvq_run_pages(top) == top / kPage + 2);
}

static void visibility() {
  std::mt19937 g(2);
  for (int trial = 0; trial < 3000; ++trial) {
    const int L = g() % 100, n = trial % 7 ? g() % kTreeMax + 1 : kTreeMax, node = g() % n;
    uint32_t mask[kTreeWords] = {};
    for (int m = 0; m <= node; ++m)
      if (m == node || g() % 3 == 0) mask[m >> 5] |= 1u << (m & 31);
    for (int page = 0; page <= (L + n - 1) / kPage; ++page) {
      const int i0 = page * kPage - L;
      const uint32_t chain = slots_of_chain(i0, node), tree = slots_of_tree(i0, mask);
      for (int s = 0; s < kPage; ++s) {
        const int m = i0 + s;
        CHECK((chain >> s & 1) == (m <= node));
        CHECK((tree >> s & 1) == (m < 0 || (m <= node && (mask[m >> 5] >> (m & 31) & 1))));
      }
    }
  }
}

int main() {
  for (int hd : {32, 64, 128}) layout(hd);
  units();
  runs();
  visibility();
  printf("kvq layout: ok\n");
  return 0;
}

// Host unit test of the 4-bit cache's layout (kvq_layout.h), built with the
// address and undefined-behaviour sanitizers by tests/test_fp4_host.py: every
// byte of a unit has one owner, what the kernels move as whole words stands
// together, and a lane's pieces are where the kernels look for them.
#include <stdio.h>
#include <stdlib.h>

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
  std::vector<int> owners(fp4_unit_bytes(hd), 0);
  const int W = fp4_pair(hd);
  for (int s = 0; s < kPage; ++s) {
    for (int d = 0; d < hd; d += 2) {
      owners.at(fp4_key_at(hd, s, d))++;
      owners.at(fp4_value_at(hd, s, d))++;
      CHECK(fp4_key_at(hd, s, d) < 16 * hd && fp4_value_at(hd, s, d) < 32 * hd);
      // whole words: eight dims of a key, four slots of a value's dims
      if (d % 8) CHECK(fp4_key_at(hd, s, d) == fp4_key_at(hd, s, d - 2) + 1);
      else CHECK(fp4_key_at(hd, s, d) % 4 == 0);
      if (s % 4) CHECK(fp4_value_at(hd, s, d) == fp4_value_at(hd, s - 1, d) + 1);
      else CHECK(fp4_value_at(hd, s, d) % 4 == 0);
      // a lane's chunk: [block of the pair][half of the page]
      const int lane = d % 32 / 8 * 16 + s % 16;
      CHECK((fp4_key_at(hd, s, d) - d / 64 * 1024 - lane * 8 * W) == d / 32 % 2 * 8 + s / 16 * 4 + d % 8 / 2);
      CHECK(fp4_value_at(hd, s, d) == fp4_value_at(hd, s % 16, d) + s / 16 * 4);
    }
    for (int d = 0; d < hd; d += 32) {
      owners.at(fp4_key_scale_at(hd, s, d))++;
      owners.at(fp4_value_scale_at(hd, s, d))++;
      // the same dims and slots as the codes' chunks, a byte for their rows of lanes
      CHECK(fp4_key_scale_at(hd, s, d) - 32 * hd == d / 64 * 64 + s % 16 * 2 * W + d / 32 % 2 * 2 + s / 16);
      if (s % 4) CHECK(fp4_value_scale_at(hd, s, d) == fp4_value_scale_at(hd, s - 1, d) + 1);
      else CHECK(fp4_value_scale_at(hd, s, d) % 4 == 0);
      if (d + 1 < hd) CHECK(fp4_key_scale_at(hd, s, d) == fp4_key_scale_at(hd, s, d / 32 * 32));
    }
  }
  for (int o : owners) CHECK(o == 1);
  CHECK(fp4_unit_bytes(hd) % 16 == 0 && kvq_unit_bytes(hd, kMxfp4) == fp4_unit_bytes(hd));
  CHECK(kvq_unit_bytes(hd, kInt8) == kvq_unit_bytes(hd) && kvq_unit_bytes(hd, kE4M3) == kvq_unit_bytes(hd));
}

static void units() {
  std::vector<int> table = {3, -1, 5, 6};
  const int unit = fp4_unit_bytes(64);
  std::vector<uint8_t> pool((size_t)6 * 2 * unit);
  const KvqView c{pool.data(), table.data(), 1, 4, 6, 2, 64, kMxfp4};
  CHECK(kvq_unit_of(c, 0, 0, 1) == pool.data() + (3 * 2 + 1) * unit);
  CHECK(kvq_unit_of(c, 0, 2, 1) + unit == pool.data() + pool.size());
  CHECK(kvq_unit_of(c, 0, 1, 0) == nullptr && kvq_unit_of(c, 0, 3, 0) == nullptr && kvq_unit_of(c, 0, 4, 0) == nullptr);
}

int main() {
  for (int hd : {32, 64, 128}) layout(hd);
  units();
  printf("fp4 layout: ok\n");
  return 0;
}

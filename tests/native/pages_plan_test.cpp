// Host unit test of the pages' plans (pages.h), built with the address and
// undefined-behaviour sanitizers by tests/test_pages_host.py: the pages that a run
// of tokens reaches, workspaces whose parts do not meet, and pieces that cover
// a page once.
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>
#include <vector>

#include "pages.h"

using namespace cdsl;

#define CHECK(x)                                                        \
  do {                                                                  \
    if (!(x)) {                                                         \
      fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #x);   \
      exit(1);                                                          \
    }                                                                   \
  } while (0)

static void runs() {
  const int big = 2147483647, ends[] = {-big - 1, -1, 0, 1, 2, 31, 32, 33, 63, 64, 95, 96, 97, big - 1, big};
  for (int P : {1, 2, 3, (1 << 26) - 1})
    for (int len : ends)
      for (int count : ends)
        for (int T : {0, 1, 31, 32, 33, 100, big}) {
          const PagesRun r = pages_run(len, count, T, P);
          const long long l = std::max(len, 0);
          const long long want = std::max(0ll, std::min({(long long)count, (long long)T, 32ll * P - l}));
          CHECK(r.fit == want && r.first == l / 32);
          CHECK(r.end == (want ? (l + want + 31) / 32 : l / 32));
          CHECK(r.end <= P || want == 0);
          CHECK(r.end - r.first <= kvq_run_pages(T));
        }
}

static void spaces() {
  for (int B : {0, 1, 7, 65535})
    for (int pages : {1, 2, 9000, 1 << 30})
      for (int T : {0, 1, 32, 5000}) {
        const ReserveSpace s = reserve_space(B, pages, T);
        CHECK(s.entries == (long long)B * kvq_run_pages(T));
        const long long at[] = {s.leave, s.first, s.last, s.need, s.free_ids, s.src, s.dst, s.jobs, s.starts, s.ints};
        const long long n[] = {pages, pages, pages, s.entries, std::min<long long>(s.entries, pages), B, B, 1, B + 1};
        for (int i = 0; i < 9; ++i) CHECK(at[i] + n[i] == at[i + 1]);
      }
  for (int pages : {1, 2, 3, 1001, 1 << 30}) {
    const CompactSpace s = compact_space(pages);
    CHECK(s.move == 0 && s.src == pages && s.dst - s.src >= (pages + 1) / 2 && s.moves - s.dst >= (pages + 1) / 2 && s.ints == s.moves + 1);
  }
}

static void pieces() {
  for (long long bytes : {1088ll, 2304ll, 16384ll, 16400ll, 34816ll, 270336ll, (1ll << 34) - 16}) {
    const Pieces p = page_pieces(bytes);
    CHECK(p.words == bytes / 16 && p.size <= kPieceWords && p.size > 0);
    CHECK((long long)p.count * p.size >= p.words && (long long)(p.count - 1) * p.size < p.words);
  }
}

int main() {
  runs();
  spaces();
  pieces();
  printf("pages plan: ok\n");
  return 0;
}

// Internal interface of the calls that give and take a cache's pages (pages.hip),
// and the arithmetic of their plans.  The latter is plain C++ without HIP
// headers, so that it is tested on the host.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "kvq_layout.h"

namespace cdsl {

constexpr int kForkRows = 512;      // prompts whose tables one launch forks
constexpr int kForkThreads = 1024, kForkCols = 4;   // of a workgroup of that launch, at most; columns of the table at a time
constexpr int kForkGroups = 1 << 16;                // its workgroups, at most: a launch has fewer than 2^32 threads
constexpr int kPieceWords = 512;    // 16-byte words that a workgroup copies at a time, at most

// Pages that a run of count tokens behind len others reaches: [first, end), cut
// at the table's end; and how many of the tokens fit in the table.
struct PagesRun {
  int first, end, fit;
};
CDSL_KVQ_HD PagesRun pages_run(int len, int count, int T, int P) {
  const long long l = len < 0 ? 0 : len, room = (long long)P * kPage - l;
  long long c = count < 0 ? 0 : count < T ? count : T;
  c = c < room ? c : room < 0 ? 0 : room;
  PagesRun r;
  r.fit = (int)c;
  r.first = (int)(l / kPage);
  r.end = c > 0 ? (int)((l + c + kPage - 1) / kPage) : r.first;
  return r;
}

// Workspace of a reserve in ints: [pages] reservers, first reserver and last need
// of each shared page, a state per entry of the runs, the free pages that are
// handed out, the copies, and where each prompt's entries start.
struct ReserveSpace {
  long long entries;        // B * pages of a run: at most
  long long leave, first, last, need, free_ids, src, dst, jobs, starts, ints;
};
CDSL_KVQ_HD ReserveSpace reserve_space(int B, int pages, int T) {
  ReserveSpace s;
  s.entries = (long long)B * kvq_run_pages(T);
  const long long handed = s.entries < pages ? s.entries : pages;
  s.leave = 0;
  s.first = s.leave + pages;
  s.last = s.first + pages;
  s.need = s.last + pages;
  s.free_ids = s.need + s.entries;
  s.src = s.free_ids + handed;
  s.dst = s.src + B;
  s.jobs = s.dst + B;
  s.starts = s.jobs + 1;
  s.ints = s.starts + B + 1;
  return s;
}

// Of a compaction: [pages] the move that takes a page, the moves, their number.
struct CompactSpace {
  long long move, src, dst, moves, ints;
};
CDSL_KVQ_HD CompactSpace compact_space(int pages) {
  CompactSpace s;
  const long long most = pages / 2 + 1;
  s.move = 0;
  s.src = pages;
  s.dst = s.src + most;
  s.moves = s.dst + most;
  s.ints = s.moves + 1;
  return s;
}

// The launch that forks up to kForkRows prompts: workgroup g takes the columns
// kForkCols * (g + k * groups), k = 0, 1, ... and those behind.
struct ForkGrid {
  int groups, threads;
};
CDSL_KVQ_HD ForkGrid fork_grid(int B, int P) {
  const int threads = (B * kForkCols + 63) / 64 * 64, groups = (P + kForkCols - 1) / kForkCols;
  return {groups < kForkGroups ? groups : kForkGroups, threads < kForkThreads ? threads : kForkThreads};
}

// How a page of a layer is cut into pieces of nearly one size.
struct Pieces {
  int words, count, size;   // of a page; pieces; words a piece
};
CDSL_KVQ_HD Pieces page_pieces(long long page_bytes) {
  Pieces p;
  p.words = (int)(page_bytes / 16);
  p.count = (p.words + kPieceWords - 1) / kPieceWords;
  p.size = (p.words + p.count - 1) / p.count;
  return p;
}

#if defined(__HIPCC__)
struct PagesArgs {
  int* table;               // [B][P]
  int* refs;                // [pages]
  int B, P, pages;
  uint8_t* pool;
  int n_layers;
  long long layer_bytes, page_bytes;
};

hipError_t pages_fork_launch(const PagesArgs& a, const int* parents, int* workspace, hipStream_t st);
hipError_t pages_reserve_launch(const PagesArgs& a, const int* lens, const int* count, int T, int* got, int* workspace,
                                hipStream_t st);
hipError_t pages_free_launch(const PagesArgs& a, const int* lens, hipStream_t st);
hipError_t pages_compact_launch(const PagesArgs& a, int* used, int* workspace, hipStream_t st);
// from a's pool to another of the same page
hipError_t pages_copy_launch(const PagesArgs& a, const int* src, uint8_t* to, int to_pages, long long to_layer_bytes,
                             const int* dst, int n, hipStream_t st);
#endif

}  // namespace cdsl

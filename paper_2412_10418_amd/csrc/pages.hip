// Pages of a cache that prompts share: forking, reserving with copy on write,
// freeing, compacting and copying (include/cdsl_ops.h has the definitions).
//
// refs[p] counts the table entries that hold page p, so a page is free at 0 and
// shared above 1.  All results are whole numbers that do not depend on the order
// in which workgroups run: counts change by atomic additions, and which page goes
// where follows from prefix sums over the pages and over the entries.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "pages.h"

namespace cdsl {

namespace {

__device__ __forceinline__ bool is_page(int id, int pages) { return id >= 0 && id < pages; }

// An entry changes from page `old` to page `now` (neither need be one).
__device__ __forceinline__ void hold(int* refs, int pages, int old, int now) {
  if (old == now) return;
  if (is_page(old, pages)) atomicSub(&refs[old], 1);
  if (is_page(now, pages)) atomicAdd(&refs[now], 1);
}

__device__ __forceinline__ int parent_entry(const PagesArgs& a, int parent, int i) {
  return parent >= 0 && parent < a.B ? a.table[(long long)parent * a.P + i] : -1;
}

// Workgroup = four columns of the table at a time, which it holds in LDS, all rows of
// them, before it writes any: one launch, where a copy of the table takes two.  A thread an
// entry, as far as they go: loads and atomics that wait for each other bound it (with 16
// columns and 256 threads: 64 prompts of 17 pages 5.8 -> 3.3 us, 256 of 65 24 -> 7,
// 512 of 257 49 -> 16, 512 of 1025 58 -> 48, where the atomics do).
__global__ __launch_bounds__(kForkThreads) void fork_kernel(PagesArgs a, const int* parents) {
  constexpr int COLS = kForkCols;
  __shared__ int old[kForkRows * COLS];
  const int col = threadIdx.x % COLS, rows = blockDim.x / COLS;
  for (int c = blockIdx.x * COLS; c < a.P; c += gridDim.x * COLS) {
    const int i = c + col;
    if (i < a.P)
      for (int b = threadIdx.x / COLS; b < a.B; b += rows) old[b * COLS + col] = a.table[(long long)b * a.P + i];
    __syncthreads();
    if (i < a.P)
      for (int b = threadIdx.x / COLS; b < a.B; b += rows) {
        const int p = parents[b];
        if (p == b) continue;
        const int now = p >= 0 && p < a.B ? old[p * COLS + col] : -1;
        hold(a.refs, a.pages, old[b * COLS + col], now);
        a.table[(long long)b * a.P + i] = now;
      }
    __syncthreads();   // before the next columns take their place
  }
}

// More prompts: the new rows into a workspace, then into the table.
__global__ __launch_bounds__(256) void fork_rows_kernel(PagesArgs a, const int* parents, int* rows) {
  const int b = blockIdx.y, p = parents[b];
  if (p == b) return;
  for (int i = blockIdx.x * 256 + threadIdx.x; i < a.P; i += gridDim.x * 256) {
    const long long at = (long long)b * a.P + i;
    const int now = parent_entry(a, p, i);
    hold(a.refs, a.pages, a.table[at], now);
    rows[at] = now;
  }
}
__global__ __launch_bounds__(256) void fork_write_kernel(PagesArgs a, const int* parents, const int* rows) {
  const int b = blockIdx.y;
  if (parents[b] == b) return;
  for (int i = blockIdx.x * 256 + threadIdx.x; i < a.P; i += gridDim.x * 256) {
    const long long at = (long long)b * a.P + i;
    a.table[at] = rows[at];
  }
}

__global__ __launch_bounds__(256) void free_kernel(PagesArgs a, const int* lens) {
  const int b = blockIdx.y, kept = (int)(((long long)max(lens[b], 0) + kPage - 1) / kPage);
  for (int i = kept + blockIdx.x * 256 + threadIdx.x; i < a.P; i += gridDim.x * 256) {
    const long long at = (long long)b * a.P + i;
    const int id = a.table[at];
    if (id != -1) {
      hold(a.refs, a.pages, id, -1);
      a.table[at] = -1;
    }
  }
}

// The sum over the lanes before this one.
__device__ __forceinline__ int wave_before(int v) {
  int s = v;
  s += __builtin_amdgcn_update_dpp(0, s, 0x111, 0xF, 0xF, false);   // row_shr 1, 2, 4, 8 ...
  s += __builtin_amdgcn_update_dpp(0, s, 0x112, 0xF, 0xF, false);
  s += __builtin_amdgcn_update_dpp(0, s, 0x114, 0xF, 0xF, false);
  s += __builtin_amdgcn_update_dpp(0, s, 0x118, 0xF, 0xF, false);
  s += __builtin_amdgcn_update_dpp(0, s, 0x142, 0xA, 0xF, false);   // ... and the sums of the rows before
  s += __builtin_amdgcn_update_dpp(0, s, 0x143, 0xC, 0xF, false);
  return s - v;
}

constexpr int kPlanThreads = 1024;

// The sums over the threads before this one, and over all; sums: in LDS, of which
// two take turns, so that one barrier is enough.
struct Sums {
  int v[2][2][16];
};
template <int N>
__device__ __forceinline__ void block_before(const int (&v)[N], Sums& sums, int& turn, int (&before)[N], int (&total)[N]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    before[n] = wave_before(v[n]);
    if (lane == 63) sums.v[turn][n][wave] = before[n] + v[n];
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < N; ++n) {
    total[n] = 0;
#pragma unroll
    for (int w = 0; w < kPlanThreads / 64; ++w) {
      const int s = sums.v[turn][n][w];
      before[n] += w < wave ? s : 0;
      total[n] += s;
    }
  }
  turn ^= 1;
}

// Atomics and loads among the threads of one workgroup, which is all that works on
// these arrays: no fence of the whole chip (four of them took 12 of 22 us).
__device__ __forceinline__ int here_load(const int* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}
__device__ __forceinline__ void here_store(int* p, int v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}
__device__ __forceinline__ void here_add(int* p, int v) {
  __hip_atomic_fetch_add(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}
__device__ __forceinline__ void here_min(int* p, int v) {
  __hip_atomic_fetch_min(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}
__device__ __forceinline__ void here_max(int* p, int v) {
  __hip_atomic_fetch_max(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}

// Which of eight pages from p on are free (USED: used).
template <bool USED>
__device__ __forceinline__ unsigned page_mask(const PagesArgs& a, int p) {
  unsigned mask = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int r = p + k < a.pages ? a.refs[p + k] : USED ? 0 : 1;
    mask |= (USED ? r > 0 : r == 0) ? 1u << k : 0u;
  }
  return mask;
}

// States of an entry that needs no page (one that does: its number).
constexpr int kFine = -1, kKeeps = -2;
constexpr int kFewEntries = 256;   // entries that are looked up in each other
constexpr int kPlanPer = 8, kPlanChunk = kPlanThreads * kPlanPer;   // entries of a thread, of the workgroup at a time

// The plan of a reserve, by one workgroup: pages and entries are few (4 bytes for
// a page's megabyte), and every step waits for all of the one before, so that what
// bounds it is a chain of loads and barriers: 8 us for 64 prompts.  Entries are
// those that the runs reach, in the order of the prompts, eight a thread; up to
// kPlanChunk of them stay in registers, more are loaded again for every step (256
// prompts of up to 65 pages each, of which they reach 3,000 entries: 12 us; with
// all 16,640 taken as entries 55).
__global__ __launch_bounds__(kPlanThreads) void reserve_kernel(PagesArgs a, const int* lens, const int* count, int T, int* got,
                                                               int* ws) {
  constexpr int PER = kPlanPer, CH = kPlanChunk, NEAR = 2048;
  __shared__ Sums sums;
  __shared__ int n_jobs;
  __shared__ int near_ids[CH];              // the first free pages
  __shared__ int near_starts[NEAR + 1], near_lens[NEAR];
  __shared__ int few_id[kFewEntries], few_number[kFewEntries];
  int turn = 0;
  const ReserveSpace at = reserve_space(a.B, a.pages, T);
  const int tid = threadIdx.x;
  int *leave = ws + at.leave, *first = ws + at.first, *last = ws + at.last, *need = ws + at.need;
  int *free_ids = ws + at.free_ids, *src = ws + at.src, *dst = ws + at.dst;
  const unsigned near = page_mask<false>(a, tid * PER);

  // where each prompt's entries start
  const bool few = a.B <= NEAR;
  int* starts = few ? near_starts : ws + at.starts;
  int E = 0;
  for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
    const int b = b0 + tid;
    int v[1] = {0}, before[1], total[1];
    if (b < a.B) {
      const int len = max(lens[b], 0);
      const PagesRun r = pages_run(len, count[b], T, a.P);
      got[b] = r.fit;
      v[0] = r.end - r.first;
      if (few) near_lens[b] = len;
    }
    block_before<1>(v, sums, turn, before, total);
    if (b < a.B) starts[b] = E + before[0];
    E += total[0];
  }
  if (tid == 0) {
    starts[a.B] = E;
    n_jobs = 0;
  }
  __syncthreads();

  struct Entry {
    int b, i, id, refs;                      // refs: -1 past the last entry
    bool tokens;                             // the prompt has tokens on it
  };
  // N entries of this thread, from e on
  auto load = [&](int e, auto& x) __attribute__((always_inline)) {
    constexpr int N = sizeof(x) / sizeof(x[0]);
    int low = 0, high = a.B;                 // the last prompt that starts at or before e
    if (e < E)
      while (high - low > 1) {
        const int mid = (low + high) / 2;
        if (starts[mid] <= e) low = mid;
        else high = mid;
      }
#pragma unroll
    for (int k = 0; k < N; ++k) {
      x[k] = {0, 0, -1, -1, false};
      if (e + k >= E) continue;
      while (starts[low + 1] <= e + k) ++low;
      const int len = few ? near_lens[low] : max(lens[low], 0);
      x[k].b = low;
      x[k].i = len / kPage + (e + k - starts[low]);
      x[k].tokens = (long long)x[k].i * kPage < len;
      x[k].id = a.table[(long long)low * a.P + x[k].i];
      if (!is_page(x[k].id, a.pages)) x[k].id = -1;
    }
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (e + k < E) x[k].refs = x[k].id >= 0 ? a.refs[x[k].id] : 0;
  };
  auto classify = [&](const Entry& x, int e, int& n) __attribute__((always_inline)) {
    if (x.refs < 0 || x.refs == 1 || (x.refs == 0 && x.id >= 0)) return kFine;
    if (x.refs > 1 && here_load(&leave[x.id]) == x.refs && here_load(&first[x.id]) == e) return kKeeps;
    return n++;
  };

  // free pages of a mask, `before` of them below; those past what is needed are not kept
  auto search = [&](int needed, int before, unsigned mask, int p) __attribute__((always_inline)) {
    for (; mask; mask &= mask - 1, ++before) {
      const int id = p + __builtin_ctz(mask);
      if (before < CH) near_ids[before] = id;
      else if (before < needed) free_ids[before] = id;
    }
  };
  // an entry for which no page is left, and one that takes the s-th
  auto fails = [&](const Entry& x) __attribute__((always_inline)) {
    const long long len = few ? near_lens[x.b] : max(lens[x.b], 0);
    here_min(&got[x.b], (int)max((long long)x.i * kPage - len, 0ll));
  };
  auto takes = [&](const Entry& x, int s) __attribute__((always_inline)) {
    const int now = s < CH ? near_ids[s] : free_ids[s];
    a.table[(long long)x.b * a.P + x.i] = now;
    a.refs[now] = 1;
    if (x.id < 0) return;
    here_add(&a.refs[x.id], -1);
    if (x.tokens) {
      const int j = atomicAdd(&n_jobs, 1);
      src[j] = x.id;
      dst[j] = now;
    }
  };

  auto plan = [&](auto registers) __attribute__((always_inline)) {
    constexpr bool ONE = decltype(registers)::value;
    Entry x[PER];
    int state[PER];
    if constexpr (ONE) load(tid * PER, x);
    // f(its first number) for this thread's entries, x
    auto each = [&](auto f) __attribute__((always_inline)) {
      if constexpr (ONE) f(tid * PER);
      else
        for (int e0 = 0; e0 < E; e0 += CH) {
          load(e0 + tid * PER, x);
          f(e0 + tid * PER);
        }
    };

    // which prompts leave a shared page in this call
    int any = 0;
    each([&](int) __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        if (x[k].refs <= 1) continue;
        any = 1;
        here_store(&leave[x[k].id], 0);
        here_store(&first[x[k].id], 0x7fffffff);
        here_store(&last[x[k].id], -1);
      }
    });
    if (__syncthreads_or(any)) {
      each([&](int e) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
          if (x[k].refs <= 1) continue;
          here_add(&leave[x[k].id], 1);
          here_min(&first[x[k].id], e + k);
        }
      });
      __syncthreads();
    }

    // the entries that need a page, numbered, and the lowest pages that are free
    int needed = 0, found = 0;
    each([&](int e) __attribute__((always_inline)) {
      int v[2] = {0, ONE ? (int)__popc(near) : 0}, before[2], total[2];
#pragma unroll
      for (int k = 0; k < PER; ++k) state[k] = classify(x[k], e + k, v[0]);
      block_before<2>(v, sums, turn, before, total);
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        if (state[k] >= 0) {
          state[k] += needed + before[0];
          if (x[k].refs > 1) here_max(&last[x[k].id], state[k]);
        }
        if (!ONE && e + k < E) need[e + k] = state[k];
      }
      needed += total[0];
      if constexpr (ONE) {
        found = total[1];
        if (needed) search(needed, before[1], near, tid * PER);
      }
    });
    for (int p0 = ONE ? CH : 0; p0 < a.pages && found < needed; p0 += CH) {
      const unsigned mask = p0 == 0 ? near : page_mask<false>(a, p0 + tid * PER);
      int v[1] = {(int)__popc(mask)}, before[1], total[1];
      block_before<1>(v, sums, turn, before, total);
      search(needed, found + before[0], mask, p0 + tid * PER);
      found += total[0];
    }
    __syncthreads();

    // each gets its page
    each([&](int e) __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        if (x[k].refs < 0) continue;
        const int s = ONE ? state[k] : need[e + k];   // written by this thread
        if (s == kFine) continue;
        const bool ok = s == kKeeps ? here_load(&last[x[k].id]) < found : s < found;
        if (!ok) fails(x[k]);
        else if (s >= 0) takes(x[k], s);
      }
    });
  };
  // Few entries, one a thread: who else leaves an entry's page is looked up in LDS,
  // two passes through memory less (64 beams: 10.6 -> 7.9 us).
  auto plan_few = [&]() __attribute__((always_inline)) {
    Entry x[1];
    load(tid, x);
    const bool shared = x[0].refs > 1;
    if (tid < E) few_id[tid] = shared ? x[0].id : -1;
    __syncthreads();
    int leave_it = 0;
    bool is_first = true;
    if (shared)
      for (int j = 0; j < E; ++j) {
        const bool same = few_id[j] == x[0].id;
        leave_it += same ? 1 : 0;
        is_first = is_first && !(same && j < tid);
      }
    const bool keeps = shared && leave_it == x[0].refs && is_first;
    const bool needs = x[0].refs >= 0 && !keeps && (shared || x[0].id < 0);
    int v[2] = {needs ? 1 : 0, (int)__popc(near)}, before[2], total[2];
    block_before<2>(v, sums, turn, before, total);
    const int needed = total[0];
    int found = total[1];
    if (tid < E) few_number[tid] = needs ? before[0] : -1;
    if (needed) search(needed, before[1], near, tid * PER);
    for (int p0 = CH; p0 < a.pages && found < needed; p0 += CH) {
      const unsigned mask = page_mask<false>(a, p0 + tid * PER);
      int w[1] = {(int)__popc(mask)}, b[1], t[1];
      block_before<1>(w, sums, turn, b, t);
      search(needed, found + b[0], mask, p0 + tid * PER);
      found += t[0];
    }
    __syncthreads();
    bool ok = needs ? before[0] < found : true;
    if (keeps && found < needed)
      for (int j = 0; j < E; ++j) ok = ok && !(few_id[j] == x[0].id && few_number[j] >= found);
    if (x[0].refs < 0) return;
    if (!ok) fails(x[0]);
    else if (needs) takes(x[0], before[0]);
  };

  if (E <= kFewEntries) plan_few();
  else if (E <= CH) plan(std::true_type{});
  else plan(std::false_type{});
  __syncthreads();
  if (tid == 0) ws[at.jobs] = n_jobs;
}

// The plan of a compaction, by one workgroup: U used pages; the k-th page from
// below that is free and below U takes what the k-th from above that is used and not
// below U holds.
__global__ __launch_bounds__(kPlanThreads) void compact_kernel(PagesArgs a, int* used, int* ws) {
  constexpr int PER = kPlanPer, CH = kPlanChunk;
  __shared__ Sums sums;
  int turn = 0;
  const CompactSpace at = compact_space(a.pages);
  const int tid = threadIdx.x;
  const unsigned near = page_mask<true>(a, tid * PER);
  int v[1] = {(int)__popc(near)}, below[1], total[1];
  for (int p0 = CH; p0 < a.pages; p0 += CH) v[0] += __popc(page_mask<true>(a, p0 + tid * PER));
  block_before<1>(v, sums, turn, below, total);
  const int U = total[0];
  if (tid == 0) {
    *used = U;
    if (U == a.pages) ws[at.moves] = 0;
  }
  int before = 0;   // used pages below
  for (int p0 = 0; p0 < a.pages; p0 += CH) {
    const unsigned mask = p0 == 0 ? near : page_mask<true>(a, p0 + tid * PER);
    v[0] = __popc(mask);
    block_before<1>(v, sums, turn, below, total);
    int u = before + below[0];
    before += total[0];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int p = p0 + tid * PER + k;
      if (p >= a.pages) break;
      if (p == U) ws[at.moves] = U - u;
      const bool is = mask >> k & 1u;
      if (is && p >= U) {
        ws[at.src + (U - 1 - u)] = p;
        ws[at.move + p] = U - 1 - u;
      } else if (!is && p < U) {
        ws[at.dst + (p - u)] = p;
      }
      u += is ? 1 : 0;
    }
  }
}

struct CopyArgs {
  const uint8_t* from;
  uint8_t* to;
  long long from_layer, to_layer, page_bytes;
  int from_pages, to_pages, n_layers;
  Pieces pieces;
  const int* src;
  const int* dst;
  const int* n_dev;      // null: n
  int n;
};

// Pages src[k] of every layer to dst[k]: a workgroup takes a piece of a page at a
// time, two 16-byte words a thread in flight.  The bytes bound it: 130 pages of 1.1 MB
// 59 us, 4.9 TB/s.  What is written goes past the caches, where it would take the
// place of what is read (64 beams that copy 8 pages: 31 -> 27 us with the plan, half of a
// pool's 512 pages 41 -> 36); pieces of 16 KB take 1 to 3 us more than of 8.
__device__ __forceinline__ void copy_pages(const CopyArgs& c) {
  const long long items = (long long)(c.n_dev ? *c.n_dev : c.n) * c.n_layers * c.pieces.count;
  for (long long it = blockIdx.x; it < items; it += gridDim.x) {
    const int piece = (int)(it % c.pieces.count);
    const long long t = it / c.pieces.count;
    const int layer = (int)(t % c.n_layers), k = (int)(t / c.n_layers);
    const int s = c.src[k], d = c.dst[k];
    if (!is_page(s, c.from_pages) || !is_page(d, c.to_pages)) continue;
    const u32x4* in = (const u32x4*)(c.from + layer * c.from_layer + s * c.page_bytes);
    u32x4* out = (u32x4*)(c.to + layer * c.to_layer + d * c.page_bytes);
    if (in == out) continue;
    const int w0 = piece * c.pieces.size, w1 = min(w0 + c.pieces.size, c.pieces.words);
    u32x4 x[kPieceWords / 256];
#pragma unroll
    for (int u = 0; u < kPieceWords / 256; ++u) {
      const int w = w0 + threadIdx.x + 256 * u;
      if (w < w1) x[u] = in[w];
    }
#pragma unroll
    for (int u = 0; u < kPieceWords / 256; ++u) {
      const int w = w0 + threadIdx.x + 256 * u;
      if (w < w1) __builtin_nontemporal_store(x[u], out + w);
    }
  }
}

__global__ __launch_bounds__(256) void copy_kernel(CopyArgs c) { copy_pages(c); }

// The moves of a compaction: table entries, counts, contents.
__global__ __launch_bounds__(256) void move_kernel(PagesArgs a, CopyArgs c, const int* move, const int* used) {
  const int n = *c.n_dev, U = *used;
  if (n == 0) return;
  const long long T = (long long)a.B * a.P, step = (long long)gridDim.x * 256;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < T; i += step) {
    const int id = a.table[i];
    if (id < U || id >= a.pages) continue;
    const int k = move[id];   // (of an entry that refs does not count: anything)
    if (k >= 0 && k < n && c.src[k] == id) a.table[i] = c.dst[k];
  }
  for (int k = blockIdx.x * 256 + threadIdx.x; k < n; k += gridDim.x * 256) {
    a.refs[c.dst[k]] = a.refs[c.src[k]];
    a.refs[c.src[k]] = 0;
  }
  copy_pages(c);
}

constexpr int kCopyGroups = 4096;

CopyArgs copy_within(const PagesArgs& a, const int* src, const int* dst, const int* n) {
  return {a.pool, a.pool, a.layer_bytes, a.layer_bytes, a.page_bytes, a.pages, a.pages, a.n_layers,
          page_pieces(a.page_bytes), src, dst, n, 0};
}

}  // namespace

hipError_t pages_fork_launch(const PagesArgs& a, const int* parents, int* workspace, hipStream_t st) {
  if (a.B == 0) return hipSuccess;
  if (a.B <= kForkRows) {
    const ForkGrid g = fork_grid(a.B, a.P);
    fork_kernel<<<(unsigned)g.groups, g.threads, 0, st>>>(a, parents);
    return hipGetLastError();
  }
  const dim3 grid((unsigned)std::min((a.P + 255) / 256, 64), (unsigned)a.B);
  fork_rows_kernel<<<grid, 256, 0, st>>>(a, parents, workspace);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  fork_write_kernel<<<grid, 256, 0, st>>>(a, parents, workspace);
  return hipGetLastError();
}

hipError_t pages_free_launch(const PagesArgs& a, const int* lens, hipStream_t st) {
  if (a.B == 0) return hipSuccess;
  const dim3 grid((unsigned)std::min((a.P + 255) / 256, 64), (unsigned)a.B);
  free_kernel<<<grid, 256, 0, st>>>(a, lens);
  return hipGetLastError();
}

hipError_t pages_reserve_launch(const PagesArgs& a, const int* lens, const int* count, int T, int* got, int* workspace,
                                hipStream_t st) {
  if (a.B == 0) return hipSuccess;
  const ReserveSpace at = reserve_space(a.B, a.pages, T);
  reserve_kernel<<<1, kPlanThreads, 0, st>>>(a, lens, count, T, got, workspace);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || T == 0) return e;
  // a prompt copies one page at most: the one that its tokens end in
  const CopyArgs c = copy_within(a, workspace + at.src, workspace + at.dst, workspace + at.jobs);
  const long long items = (long long)a.B * a.n_layers * c.pieces.count;
  copy_kernel<<<(unsigned)std::min<long long>(items, kCopyGroups), 256, 0, st>>>(c);
  return hipGetLastError();
}

hipError_t pages_compact_launch(const PagesArgs& a, int* used, int* workspace, hipStream_t st) {
  compact_kernel<<<1, kPlanThreads, 0, st>>>(a, used, workspace);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const CompactSpace at = compact_space(a.pages);
  const CopyArgs c = copy_within(a, workspace + at.src, workspace + at.dst, workspace + at.moves);
  const long long items = std::max((long long)(a.pages / 2) * a.n_layers * c.pieces.count, ((long long)a.B * a.P + 255) / 256);
  move_kernel<<<(unsigned)std::max(1ll, std::min<long long>(items, kCopyGroups)), 256, 0, st>>>(a, c, workspace + at.move, used);
  return hipGetLastError();
}

hipError_t pages_copy_launch(const PagesArgs& a, const int* src, uint8_t* to, int to_pages, long long to_layer_bytes,
                             const int* dst, int n, hipStream_t st) {
  if (n == 0) return hipSuccess;
  CopyArgs c = copy_within(a, src, dst, nullptr);
  c.to = to;
  c.to_pages = to_pages;
  c.to_layer = to_layer_bytes;
  c.n = n;
  const long long items = (long long)n * a.n_layers * c.pieces.count;
  copy_kernel<<<(unsigned)std::min<long long>(items, kCopyGroups), 256, 0, st>>>(c);
  return hipGetLastError();
}

}  // namespace cdsl

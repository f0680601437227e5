// Pages of a cache that prompts share: forking, reserving with copy on write,
// freeing, compacting and copying (include/cdsl_ops.h has the definitions).
//
// refs[p] counts the table entries that hold page p, so a page is free at 0 and
// shared above 1.  All results are whole numbers that do not depend on the order
// in which workgroups run: counts change by atomic additions, and which page goes
// where follows from prefix sums over the pages and over the entries.
#include <algorithm>

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

// Workgroup = 16 columns of the table, which it holds in LDS, all rows of them,
// before it writes any: one launch, where a copy of the table takes two.
__global__ __launch_bounds__(256) void fork_kernel(PagesArgs a, const int* parents) {
  __shared__ int old[kForkRows * 16];
  const int col = threadIdx.x & 15, i = blockIdx.x * 16 + col;
  if (i < a.P)
    for (int b = threadIdx.x >> 4; b < a.B; b += 16) old[b * 16 + col] = a.table[(long long)b * a.P + i];
  __syncthreads();
  if (i >= a.P) return;
  for (int b = threadIdx.x >> 4; b < a.B; b += 16) {
    const int p = parents[b];
    if (p == b) continue;
    const int now = p >= 0 && p < a.B ? old[p * 16 + col] : -1;
    hold(a.refs, a.pages, old[b * 16 + col], now);
    a.table[(long long)b * a.P + i] = now;
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

// The sum over the threads before this one; total: over all.  sums: [16] in LDS,
// of which two take turns, so that one barrier is enough.
__device__ __forceinline__ int block_before(int v, int (*sums)[16], int& turn, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int before = wave_before(v);
  if (lane == 63) sums[turn][wave] = before + v;
  __syncthreads();
  int at = before;
  total = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    const int s = sums[turn][w];
    at += w < wave ? s : 0;
    total += s;
  }
  turn ^= 1;
  return at;
}

// What other threads of the workgroup wrote is there after this.
__device__ __forceinline__ void block_fence() {
  __threadfence();
  __syncthreads();
}
__device__ __forceinline__ int read_now(const int* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// States of an entry that needs no page (one that does: its number).
constexpr int kFine = -1, kKeeps = -2;

// The plan of a reserve, by one workgroup: pages and entries are few (4 bytes for
// a page's megabyte), and every step waits for all of the one before.
__global__ __launch_bounds__(kPlanThreads) void reserve_kernel(PagesArgs a, const int* lens, const int* count, int T, int* got,
                                                               int* ws) {
  constexpr int PER = 8;                    // entries of a thread at a time
  constexpr int CH = kPlanThreads * PER;
  __shared__ int sums[2][16];
  __shared__ int n_jobs;
  int turn = 0;
  const ReserveSpace at = reserve_space(a.B, a.pages, T);
  const int M = kvq_run_pages(T), E = (int)at.entries, tid = threadIdx.x;
  int *leave = ws + at.leave, *first = ws + at.first, *last = ws + at.last, *need = ws + at.need;
  int *free_ids = ws + at.free_ids, *src = ws + at.src, *dst = ws + at.dst;

  struct Entry {
    int b, i, id, refs, len;
    bool in, held, shared;
  };
  auto entry = [&](int e) __attribute__((always_inline)) {
    Entry x{};
    if (e >= E) return x;
    x.b = e / M;
    x.len = max(lens[x.b], 0);
    const PagesRun r = pages_run(x.len, count[x.b], T, a.P);
    x.i = r.first + e % M;
    x.in = x.i < r.end;
    if (!x.in) return x;
    x.id = a.table[(long long)x.b * a.P + x.i];
    x.held = is_page(x.id, a.pages);
    x.refs = x.held ? a.refs[x.id] : 0;
    x.shared = x.refs > 1;
    return x;
  };

  // which prompts leave a shared page in this call
  if (tid == 0) n_jobs = 0;
  for (int b = tid; b < a.B; b += kPlanThreads) got[b] = pages_run(lens[b], count[b], T, a.P).fit;
  bool any = false;
  for (int e = tid; e < E; e += kPlanThreads) {
    const Entry x = entry(e);
    if (x.shared) {
      leave[x.id] = 0;
      first[x.id] = 0x7fffffff;
      last[x.id] = -1;
      any = true;
    }
  }
  any = __syncthreads_or(any);
  if (any) {
    block_fence();
    for (int e = tid; e < E; e += kPlanThreads) {
      const Entry x = entry(e);
      if (x.shared) {
        atomicAdd(&leave[x.id], 1);
        atomicMin(&first[x.id], e);
      }
    }
    block_fence();
  }

  // the entries that need a page, numbered
  int needed = 0;
  for (int e0 = 0; e0 < E; e0 += CH) {
    int state[PER], n = 0;
    Entry x[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int e = e0 + tid * PER + k;
      x[k] = entry(e);
      state[k] = kFine;
      if (x[k].shared && read_now(&leave[x[k].id]) == x[k].refs && read_now(&first[x[k].id]) == e) state[k] = kKeeps;
      else if (x[k].in && (!x[k].held || x[k].shared)) state[k] = n++;
    }
    int total;
    const int base = needed + block_before(n, sums, turn, total);
    needed += total;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int e = e0 + tid * PER + k;
      if (e >= E) break;
      if (state[k] >= 0) {
        state[k] += base;
        if (x[k].shared) atomicMax(&last[x[k].id], state[k]);
      }
      need[e] = state[k];
    }
  }

  // the lowest free pages, as many as are needed
  int found = 0;
  for (int p0 = 0; p0 < a.pages && found < needed; p0 += CH) {
    unsigned mask = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int p = p0 + tid * PER + k;
      if (p < a.pages && a.refs[p] == 0) mask |= 1u << k;
    }
    int total;
    int n = found + block_before(__popc(mask), sums, turn, total);
    found += total;
    for (; mask && n < needed; mask &= mask - 1) free_ids[n++] = p0 + tid * PER + __builtin_ctz(mask);
  }
  block_fence();

  // each gets its page
  for (int e0 = 0; e0 < E; e0 += CH)
    for (int k = 0; k < PER; ++k) {
      const int e = e0 + tid * PER + k;
      if (e >= E) break;
      const int s = need[e];   // written by this thread
      if (s == kFine) continue;
      const int b = e / M, len = max(lens[b], 0), i = len / kPage + e % M;
      int* slot = &a.table[(long long)b * a.P + i];
      const int old = *slot;
      const bool ok = s == kKeeps ? read_now(&last[old]) < found : s < found;
      if (!ok) {
        atomicMin(&got[b], max(0, (int)max((long long)i * kPage - len, 0ll)));
      } else if (s >= 0) {
        const int now = free_ids[s];
        *slot = now;
        a.refs[now] = 1;
        if (is_page(old, a.pages)) {
          atomicSub(&a.refs[old], 1);
          if ((long long)i * kPage < len) {   // it holds tokens of the prompt
            const int j = atomicAdd(&n_jobs, 1);
            src[j] = old;
            dst[j] = now;
          }
        }
      }
    }
  __syncthreads();
  if (tid == 0) ws[at.jobs] = n_jobs;
}

// The plan of a compaction, by one workgroup: U used pages; the k-th page from
// below that is free and below U takes what the k-th from above that is used and not
// below U holds.
__global__ __launch_bounds__(kPlanThreads) void compact_kernel(PagesArgs a, int* used, int* ws) {
  constexpr int PER = 8, CH = kPlanThreads * PER;
  __shared__ int sums[2][16];
  int turn = 0;
  const CompactSpace at = compact_space(a.pages);
  const int tid = threadIdx.x;
  int n = 0, U;
  for (int p = tid; p < a.pages; p += kPlanThreads) n += a.refs[p] > 0 ? 1 : 0;
  block_before(n, sums, turn, U);
  if (tid == 0) {
    *used = U;
    if (U == a.pages) ws[at.moves] = 0;
  }
  int before = 0;   // used pages below
  for (int p0 = 0; p0 < a.pages; p0 += CH) {
    unsigned mask = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int p = p0 + tid * PER + k;
      if (p < a.pages && a.refs[p] > 0) mask |= 1u << k;
    }
    int total;
    int u = before + block_before(__popc(mask), sums, turn, total);
    before += total;
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
// time, four 16-byte words a thread in flight.
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
      if (w < w1) out[w] = x[u];
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

constexpr int kCopyGroups = 2048;   // eight a CU

CopyArgs copy_within(const PagesArgs& a, const int* src, const int* dst, const int* n) {
  return {a.pool, a.pool, a.layer_bytes, a.layer_bytes, a.page_bytes, a.pages, a.pages, a.n_layers,
          page_pieces(a.page_bytes), src, dst, n, 0};
}

}  // namespace

hipError_t pages_fork_launch(const PagesArgs& a, const int* parents, int* workspace, hipStream_t st) {
  if (a.B == 0) return hipSuccess;
  if (a.B <= kForkRows) {
    fork_kernel<<<(unsigned)((a.P + 15) / 16), 256, 0, st>>>(a, parents);
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
  reserve_kernel<<<1, kPlanThreads, 0, st>>>(a, lens, count, T, got, workspace);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || T == 0) return e;
  const ReserveSpace at = reserve_space(a.B, a.pages, T);
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
  move_kernel<<<kCopyGroups, 256, 0, st>>>(a, c, workspace + at.move, used);
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

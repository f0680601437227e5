// Which kernel a tree attention takes, and how its rows and keys are split over
// the chip.  Plain C++ without HIP headers, so that the choices are tested on
// the host.
#pragma once

#include <stddef.h>

#include <algorithm>

#include "kvq_layout.h"

namespace cdsl {

constexpr int kTreeMaxSplits = 64;
constexpr int kTreeShared = 64;   // prompts that share the key splits by their lengths

struct TreeAttnPlan {
  int few;                 // 1, 2: tree_few_kernel with so many row tiles
  bool wide;               // tree_wide_kernel; else tree_many_kernel
  bool four;               // tree_many_kernel at four waves a SIMD; else three
  int wg_tiles;            // row tiles (of 16) per workgroup
  int row_groups, slots, split_pages;
  size_t workspace;
};

// dtype: 0 fp32, 1 bf16.  fp32 over e4m3 (heads of 128) is as fast in tiles of 16
// rows (188 us) as of 32 (190).
constexpr bool tree_may_be_wide(int hd, int dtype, int format) { return !(hd == 128 && dtype == 0 && format == kE4M3); }

// Four workgroups a CU where there are as many; fewer are faster in three (64
// trees of 65 at 2048 in bf16: 152 -> 146 us; 16 of them: 56 -> 61).  Heads of 64
// gain nothing by it, fp32 over int8 loses 5% (231 -> 243).
constexpr bool tree_may_be_four(int hd, int dtype, int format) { return hd == 128 && (dtype == 1 || format == kE4M3); }

inline TreeAttnPlan tree_attn_plan(int B, int n, int H, int Hkv, int hd, int max_len, int dtype, int format) {
  TreeAttnPlan p{};
  const int tiles = (int)(((long long)n * (H / Hkv) + 15) / 16);
  p.few = tiles <= 2 ? tiles : 0;
  // Tiles of 32 rows, of which two workgroups fit a CU:
  //  - where they fill their workgroups to 15 of 16, and those the chip one and a
  //    half times or more (64 prompts x 8 KV heads of 16 tiles of 16 at up to 2048
  //    tokens: 119 against 127 us in bf16, 194 against 201 in fp32 over int8; of
  //    14 tiles 75.0 against 74.7, of 17 134 against 125; chunks of 500 x 4 at 1000,
  //    12 prompts: 191 against 207), or in bf16 just once (32 prompts at 4096: 188
  //    against 215; up to 4096: 128 against 124);
  //  - where the keys are split anyway, are many, and half the workgroups take
  //    the rows (8 prompts of 17 x 4 rows at 8192: 62 against 68 us in bf16, 85
  //    against 90 in fp32; 32: 184 against 240 and 281 against 331; but 8 of 32 x
  //    4 at 2048: 36.5 against 35.1; one of 61 x 4 at 4096: 27.1 against 24.6; two
  //    chunks of 509 x 4 at 4000: 121 against 145 in bf16, at 2000: 82 against 79).
  const long long pairs = (long long)B * Hkv;
  const long long one = (tiles + 3) / 4, two = (tiles + 7) / 8, full = pairs * two;
  const long long pages = ((long long)max_len + n + kPage - 1) / kPage;
  const bool filled = 16 * (8 * two - tiles) <= 8 * two && (full >= 768 || (dtype == 1 && full >= 448 && full <= 512));
  const bool split = one == 2 * two && full * 3 <= 512 * 2 && pages >= 128 && full * pages >= 8192;
  p.wide = !p.few && (filled || split) && tree_may_be_wide(hd, dtype, format);
  const int most_tiles = p.few ? p.few : p.wide ? 8 : 4;
  p.row_groups = (tiles + most_tiles - 1) / most_tiles;
  p.wg_tiles = (tiles + p.row_groups - 1) / p.row_groups;
  // Keys are split until there are two workgroups a CU (few rows, tiles of 32) or
  // three.  More parts start more often than they balance (at 512, 768 and 1024
  // workgroups: 32 prompts of one token at 4096: 38, 38, 42 us; 8 trees of 65 at
  // 8192: 248, 151, 153; 4 of 40 at 4000: 34.6, 32.7, 38.8).  Less than two
  // parts a prompt only where prompts are long and 1.5 are to be had (12 trees
  // of 65: at 8192 198 us instead of 252, at 2048 72 either way).
  //
  // A part has 16 pages or more (few rows: four a wave), or 4 and one more for
  // every 1024 rows of 128, since those are written, read and merged per part (at
  // 256 and 1024 tokens, 8 trees of 51 x 32 heads take 20 and 42 us whole, 32
  // and 46 in parts of 4; one tree 16.7 and 20 in parts of 4, 28 at 1024 in parts of
  // 16).  Few rows: not below 48 pages (one token at 512: 11 us whole, 16.5 in
  // parts of 8; at 1024 13.6 and 14.8 in two; at 2048 21 and 14.8 in four), nor
  // below 128 where a workgroup a CU starts anyway (8 prompts x 32 KV heads at
  // 2048: 27 whole, 31.5).  Few rows over a long cache are split in two whatever
  // their number: one prompt of 16384 among 63 short ones takes 37 us instead of
  // 116, 64 of up to 8192 115 instead of 119.
  p.split_pages = p.few ? 16 : (int)(4 + ((long long)B * n * H * hd >> 17));
  long long most = std::min<long long>(std::max<long long>(1, pages / p.split_pages), kTreeMaxSplits);
  if (p.few && pages < (pairs >= 256 ? 128 : 48)) most = 1;
  const bool shared = B > 1 && B <= kTreeShared;
  long long slots = p.few ? 512 / Hkv : p.wide ? 512 / (Hkv * two) : 768 / (Hkv * one);
  if (p.few && shared && pages >= 256) slots = std::max(slots, 2ll * B);
  if (!shared || slots < 2 * B && (pages < 128 || 2 * slots < 3 * B)) slots -= slots % B;
  p.slots = (int)std::max<long long>(B, std::min(slots, B * most));
  p.four = !p.few && !p.wide && tree_may_be_four(hd, dtype, format) &&
           (long long)p.row_groups * p.slots * Hkv >= 1024;
  p.workspace = p.slots > B ? (size_t)p.slots * n * H * (hd + 2) * sizeof(float) : 0;
  return p;
}

// Enough for every type and format.
inline size_t tree_attn_workspace(int B, int n, int H, int Hkv, int hd, int max_len) {
  // the types decide on the tiles alone: one pair that may have them of 32, one not
  return std::max(tree_attn_plan(B, n, H, Hkv, hd, max_len, 1, kInt8).workspace,
                  tree_attn_plan(B, n, H, Hkv, hd, max_len, 0, kE4M3).workspace);
}

}  // namespace cdsl

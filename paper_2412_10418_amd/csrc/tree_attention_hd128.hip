// Tree attention over the 8-bit cache: head dimension 128, the plan and the
// dispatch over head dimensions.
#include <algorithm>

#include "tree_attention.h"

namespace cdsl {

hipError_t tree_attn_hd128(const TreeAttnArgs& a, const TreeAttnPlan& p, int dtype, hipStream_t st) {
  return tree_attn_hd<128>(a, p, dtype, st);
}

TreeAttnPlan tree_attn_plan(int B, int n, int H, int Hkv, int hd, int max_len) {
  TreeAttnPlan p{};
  const int tiles = (int)(((long long)n * (H / Hkv) + 15) / 16);
  p.rpw = tiles == 1 ? 1 : 2;
  p.kw = tiles <= 2 ? 4 : tiles <= 4 ? 2 : 1;
  const int per_wg = p.rpw * (4 / p.kw);
  p.row_groups = (tiles + per_wg - 1) / per_wg;
  const long long wgs = (long long)B * Hkv * p.row_groups;
  // two workgroups a CU at a time; a wave of a split takes two pages at least
  const long long pages = ((long long)max_len + n + kPage - 1) / kPage;
  const long long most = std::max<long long>(1, pages / (2 * p.kw));
  p.nsplit = (int)std::min<long long>({std::max<long long>(1, 512 / std::max<long long>(wgs, 1)), most, kTreeMaxSplits});
  p.workspace = p.nsplit > 1 ? (size_t)p.nsplit * B * n * H * (hd + 2) * sizeof(float) : 0;
  return p;
}

hipError_t tree_attn_launch(TreeAttnArgs a, const TreeAttnPlan& p, int dtype, void* workspace, hipStream_t st) {
  if (a.c.B == 0 || a.n == 0) return hipSuccess;
  a.nsplit = p.nsplit;
  a.row_groups = p.row_groups;
  a.part_o = (float*)workspace;
  a.part_ml = a.part_o + (size_t)p.nsplit * a.c.B * a.n * a.H * a.c.hd;
  switch (a.c.hd) {
    case 32: return tree_attn_hd32(a, p, dtype, st);
    case 64: return tree_attn_hd64(a, p, dtype, st);
    case 128: return tree_attn_hd128(a, p, dtype, st);
  }
  return hipErrorInvalidValue;
}

}  // namespace cdsl

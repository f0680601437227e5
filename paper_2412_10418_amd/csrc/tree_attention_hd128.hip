// Tree attention over the 8-bit cache: head dimension 128, the plan and the
// dispatch over head dimensions.
#include <algorithm>

#include "tree_attention.h"

namespace cdsl {

hipError_t tree_attn_hd128(const TreeAttnArgs& a, const TreeAttnPlan& p, int dtype, hipStream_t st) {
  return tree_attn_hd<128>(a, p, dtype, st);
}

TreeAttnPlan tree_attn_plan(int B, int n, int H, int Hkv, int hd, int max_len, int dtype) {
  TreeAttnPlan p{};
  const int tiles = (int)(((long long)n * (H / Hkv) + 15) / 16);
  p.few = tiles <= 2 ? tiles : 0;
  // Two row tiles a wave read every fragment of a page once for both: better
  // where the LDS and the vector units bound it (bf16, 16 prompt x KV head
  // pairs of 128 tiles: 78 against 95 us).  In fp32 the matrix units have
  // twice the work and more waves hide more (512 pairs of 17 tiles: 279
  // against 310 us).
  p.rpw = dtype == 1 && tiles > 4 ? 2 : 1;
  const int most_tiles = p.few ? p.few : 4 * p.rpw;
  p.row_groups = (tiles + most_tiles - 1) / most_tiles;
  p.wg_tiles = (tiles + p.row_groups - 1) / p.row_groups;
  // Keys are split until there are two workgroups a CU, counted in groups of
  // four tiles whatever the type; a split has four pages (few rows: eight, two
  // a wave) at least.
  const long long wgs = (long long)B * Hkv * (p.few ? 1 : (tiles + 3) / 4);
  const long long pages = ((long long)max_len + n + kPage - 1) / kPage;
  const long long most = std::max<long long>(1, pages / (p.few ? 8 : 4));
  p.nsplit = (int)std::min<long long>({std::max<long long>(1, 512 / std::max<long long>(wgs, 1)), most, kTreeMaxSplits});
  p.workspace = p.nsplit > 1 ? (size_t)p.nsplit * B * n * H * (hd + 2) * sizeof(float) : 0;
  return p;
}

hipError_t tree_attn_launch(TreeAttnArgs a, const TreeAttnPlan& p, int dtype, void* workspace, hipStream_t st) {
  if (a.c.B == 0 || a.n == 0) return hipSuccess;
  a.nsplit = p.nsplit;
  a.row_groups = p.row_groups;
  a.wg_tiles = p.wg_tiles;
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

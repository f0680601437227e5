// Tree attention over the 8-bit cache: head dimension 128, and the dispatch over
// formats and head dimensions.
#include "tree_attention.h"

namespace cdsl {

hipError_t tree_attn_hd128(const TreeAttnArgs& a, const TreeAttnPlan& p, int dtype, hipStream_t st) {
  return tree_attn_hd<128>(a, p, dtype, st);
}

hipError_t tree_attn_launch(TreeAttnArgs a, const TreeAttnPlan& p, int dtype, void* workspace, hipStream_t st) {
  if (a.c.B == 0 || a.n == 0) return hipSuccess;
  a.slots = p.slots;
  a.row_groups = p.row_groups;
  a.split_pages = p.split_pages;
  a.wg_tiles = p.wg_tiles;
  a.part_o = (float*)workspace;
  a.part_ml = a.part_o + (size_t)p.slots * a.n * a.H * a.c.hd;
  if (a.c.format == kMxfp4) {
    switch (a.c.hd) {
      case 32: return fp4_attn_hd32(a, p, dtype, st);
      case 64: return fp4_attn_hd64(a, p, dtype, st);
      case 128: return fp4_attn_hd128(a, p, dtype, st);
    }
    return hipErrorInvalidValue;
  }
  switch (a.c.hd) {
    case 32: return tree_attn_hd32(a, p, dtype, st);
    case 64: return tree_attn_hd64(a, p, dtype, st);
    case 128: return tree_attn_hd128(a, p, dtype, st);
  }
  return hipErrorInvalidValue;
}

}  // namespace cdsl

// Tree attention over the 8-bit cache, head dimension 32.
#include "tree_attention.h"

namespace cdsl {

hipError_t tree_attn_hd32(const TreeAttnArgs& a, const TreeAttnPlan& p, int dtype, hipStream_t st) {
  return tree_attn_hd<32>(a, p, dtype, st);
}

}  // namespace cdsl

// Tree attention over the 4-bit cache, head dimension 128.
#include "tree_attention_fp4.h"

namespace cdsl {

hipError_t fp4_attn_hd128(const TreeAttnArgs& a, const TreeAttnPlan& p, int dtype, hipStream_t st) {
  return dtype == 1 ? fp4_attn_rows<128, bf16>(a, p, st) : fp4_attn_rows<128, float>(a, p, st);
}

}  // namespace cdsl

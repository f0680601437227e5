// What the kernels of the 8-bit cache (kvq.hip) and of the 4-bit one (kvq_fp4.hip)
// share: lane moves, and the order of a unit's words in LDS.
#pragma once
#include "common.h"

namespace cdsl {

namespace {

// Bytes (t, e) -> (e, t) of four words.
__device__ __forceinline__ void transpose4(const unsigned (&w)[4], unsigned (&o)[4]) {
  const unsigned a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400), b = __builtin_amdgcn_perm(w[3], w[2], 0x05010400);
  const unsigned c = __builtin_amdgcn_perm(w[1], w[0], 0x07030602), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602);
  o[0] = __builtin_amdgcn_perm(b, a, 0x05040100);
  o[1] = __builtin_amdgcn_perm(b, a, 0x07060302);
  o[2] = __builtin_amdgcn_perm(d, c, 0x05040100);
  o[3] = __builtin_amdgcn_perm(d, c, 0x07060302);
}

// The larger of a lane's value and that of the lane that CTRL moves to it.
template <int CTRL>
__device__ __forceinline__ unsigned max_moved(unsigned a) {
  return max(a, (unsigned)__builtin_amdgcn_update_dpp(0, (int)a, CTRL, 0xf, 0xf, false));
}
// Where word w of a unit's codes stands in LDS: the sixteen 16-byte chunks of a
// row of 64 words are permuted by the row, so that neither the order of the
// rows (dims along the lanes) nor that of the unit meets one bank often.
__device__ __forceinline__ int banked(int w) { return w ^ ((w >> 6 & 15) << 2); }

// The pointer that another lane holds.
template <typename P>
__device__ __forceinline__ P* ptr_of_lane(P* p, int lane) {
  return (P*)__shfl((long long)p, lane, 64);
}

}  // namespace

}  // namespace cdsl

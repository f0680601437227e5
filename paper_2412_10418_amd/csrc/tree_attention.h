// Attention of a token tree over the 8-bit paged cache: the kernels, one
// instance file per head dimension (tree_attention_*.hip).
//
//   o_i = sum_j softmax_j(scale q_i . k_j) v_j
//
// over the prompt's L cached tokens and the node's ancestors and itself.
// With k = s_k c_k and v = s_v c_v (codes c, one scale per token and KV head)
// the scales leave the sums over dims: s_k multiplies a score, s_v a
// probability, and the matrix products run on the codes, which are exact in
// f16 and in bf16.  One pass over the keys with a running maximum and sum
// (fp32).  The rows of a (prompt, KV head) are its nodes x the G query heads
// of that KV head, in tiles of 16.  Scores are computed transposed,
//   S^T[16 keys, 16 rows] = K[16, hd] . Q^T[hd, 16]       (MFMA 16x16x32)
// so that a lane's scores are its operand of the second product,
//   O^T[16 dims, 16 rows] += V^T[16 dims, 32 keys] . P^T[32 keys, 16 rows].
//
// Precision.  A row of q is scaled by a power of two to a largest entry in
// [2^14, 2^15), the top of f16, and taken as f16 planes: two for fp32 activations
// (each entry to 2^-24 of itself or 2^-39 of the largest, whichever is more), one
// for bf16 (exact down to 2^-31 of the largest).  The key codes are taken times
// 2^-14 in turn, exact in f16, whose subnormals the products keep.
// Probabilities times s_v can be of any size, so they stay bf16: three planes
// (their 24 bits) for fp32, where two would lose 2^-16 of each: 2.5e-6 of the
// result, where fp32 products give 0.8e-6.  For bf16 two (2^-16 of each; 0.0017 of
// the result in the mean square, its own rounding) with one tile of rows, where
// the keys' bytes bound the time, and one (2^-8; 0.0023) with more rows, where the
// second takes 6 to 24% longer (8 prompts of 8 nodes x 4 at 4096: 22.2 -> 23.6 us, 64
// trees of 65 at 2048: 140 -> 155, two chunks of 512 over 32768: 685 -> 852).
//
// Three kernels.  Few rows (one or two tiles): the codes go from memory
// straight to the registers of the wave that uses them, and the waves of a
// workgroup take different pages (tree_few_kernel).  More rows: the
// workgroup's waves take different rows, and the pages are converted once for
// all of them through LDS (tree_many_kernel; tree_wide_kernel with tiles of 32
// rows where they fill the chip).
#pragma once
#include <type_traits>

#include "tree.h"

namespace cdsl {

namespace {

typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;
typedef __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16 f16x2;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;

constexpr float kLazy = 8.f;   // log2 units that the running maximum may lag behind

// Eight codes (two words) as bf16, exact.
template <int FMT>
__device__ __forceinline__ bf16x8 codes_bf16(unsigned a, unsigned b) {
  union {
    unsigned u[4];
    bf16x2v p[4];
    bf16x8 v;
  } o;
  if constexpr (FMT == kE4M3) {
    o.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false);
    o.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true);
    o.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false);
    o.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true);
  } else {
    // an 8-bit integer has at most 7 significant bits: the upper half of
    // its fp32 form is its bf16 form
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const unsigned w = i ? b : a;
      const unsigned f0 = __float_as_uint((float)(int8_t)w), f1 = __float_as_uint((float)(int8_t)(w >> 8));
      const unsigned f2 = __float_as_uint((float)(int8_t)(w >> 16)), f3 = __float_as_uint((float)((int)w >> 24));
      o.u[2 * i] = __builtin_amdgcn_perm(f1, f0, 0x07060302);
      o.u[2 * i + 1] = __builtin_amdgcn_perm(f3, f2, 0x07060302);
    }
  }
  return o.v;
}

// Eight key codes times 2^-14 as f16, exact (e4m3: down to 2^-23, a subnormal).
template <int FMT>
__device__ __forceinline__ f16x8 codes_f16(unsigned a, unsigned b) {
  union {
    unsigned u[4];
    f16x2 p[4];
    f16x8 v;
  } o;
  if constexpr (FMT == kE4M3) {
    o.p[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 0x1p-14f, false);
    o.p[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 0x1p-14f, true);
    o.p[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 0x1p-14f, false);
    o.p[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 0x1p-14f, true);
  } else {
    // 0x6400 + x is 1024 + x in f16: with x = code + 128, one multiply-add
    const f16x2 down = {(_Float16)0x1p-14f, (_Float16)0x1p-14f};
    const f16x2 off = {(_Float16)(-1152 * 0x1p-14f), (_Float16)(-1152 * 0x1p-14f)};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const unsigned w = (i ? b : a) ^ 0x80808080u;
      o.u[2 * i] = __builtin_amdgcn_perm(0x64646464u, w, 0x04010400);
      o.u[2 * i + 1] = __builtin_amdgcn_perm(0x64646464u, w, 0x04030402);
      o.p[2 * i] = __builtin_elementwise_fma(o.p[2 * i], down, off);
      o.p[2 * i + 1] = __builtin_elementwise_fma(o.p[2 * i + 1], down, off);
    }
  }
  return o.v;
}

// Bytes of word bits 0..3 of m as a mask.
__device__ __forceinline__ unsigned byte_mask(unsigned m) {
  return ((m & 1u) | (m & 2u) << 7 | (m & 4u) << 14 | (m & 8u) << 21) * 255u;
}

// e4m3 codes of slots past the last node (never written), and those read in
// place of a page that does not exist (held = 0), may be NaNs: zeros.
__device__ __forceinline__ u32x4 hold_values(u32x4 w, int held, int lg) {
  const unsigned hm = held >= 32 ? ~0u : (1u << held) - 1u;
  const unsigned mA = byte_mask(hm >> (4 * lg)), mB = byte_mask(hm >> (16 + 4 * lg));
  return (u32x4){w.x & mA, w.y & mB, w.z & mA, w.w & mB};
}

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ float halves_max(float v) {   // xor 32
  const u32x2 t = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(t.x), __uint_as_float(t.y));
}
// Over the four lanes of a row (xor 16 and 32).
__device__ __forceinline__ float groups_max(float v) {
  v = halves_max(v);
  const u32x2 t = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(t.x), __uint_as_float(t.y));
}
// Over a wave, by lane moves.
__device__ __forceinline__ float lanes_sum(float v) {
  const u32x2 t = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(t.x) + __uint_as_float(t.y);
  const u32x2 u = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(u.x) + __uint_as_float(u.y);
  v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x128, 0xF, 0xF, true));   // rotations of 16
  v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x124, 0xF, 0xF, true));
  v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x122, 0xF, 0xF, true));
  return v + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x121, 0xF, 0xF, true));
}

// The sum over the lanes before this one.
__device__ __forceinline__ int lanes_before(int v) {
  int s = v;
  s += __builtin_amdgcn_update_dpp(0, s, 0x111, 0xF, 0xF, false);   // row_shr 1, 2, 4, 8 ...
  s += __builtin_amdgcn_update_dpp(0, s, 0x112, 0xF, 0xF, false);
  s += __builtin_amdgcn_update_dpp(0, s, 0x114, 0xF, 0xF, false);
  s += __builtin_amdgcn_update_dpp(0, s, 0x118, 0xF, 0xF, false);
  s += __builtin_amdgcn_update_dpp(0, s, 0x142, 0xA, 0xF, false);   // ... and the sums of the rows before
  s += __builtin_amdgcn_update_dpp(0, s, 0x143, 0xC, 0xF, false);
  return s - v;
}

// Key splits of a batch of 2 to 64 prompts.  The launch has room for a.slots
// of them; a prompt takes a share in proportion to its pages (its "parts", one
// at least, of a.split_pages pages or more), so that a long prompt among short
// ones does not hold up the rest (8 prompts of up to 32768 tokens: 75 -> 69 us;
// one of 16384 among 31 of 512: 60 -> 24).  Lane j of a wave finds the parts of
// prompt j, their size and the slot of the first.
//
// ceil(w x) parts of weights w come to at most x sum(w) + B, so the last of the
// four x fits; the first that does is taken.  (Weights up to 2^25 and 1e-5
// under the bound: far more than the rounding of these sums.)
struct TreeParts {
  int parts, slot;
  float size;
};
__device__ __forceinline__ TreeParts tree_parts(const TreeAttnArgs& a, int lane) {
  const int B = a.c.B;
  float w = 0.f;
  if (lane < B) {
    const int L = max(a.lens[lane], 0), nb = a.n_nodes ? min(max(a.n_nodes[lane], 0), a.n) : a.n;
    const long long toks = (long long)L + nb;
    if (toks <= (long long)a.c.table_stride * kPage) w = (float)min((toks + kPage - 1) / kPage, 1ll << 25);
  }
  int parts = 1;
  float size = w;
  if (a.slots > B) {
    const float room = (float)a.slots, per = 0.99999f / fmaxf(lanes_sum(w), 1.f);
    const float most = 1.f / (float)a.split_pages;
    float k[4], sum[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = fminf((room - (float)(B * i) / 3.f) * per, most);
      k[i] = lane < B ? fminf(fmaxf(ceilf(w * x), 1.f), (float)kTreeMaxSplits) : 0.f;
      sum[i] = lanes_sum(k[i]);
    }
    const float of = sum[0] <= room ? k[0] : sum[1] <= room ? k[1] : sum[2] <= room ? k[2] : k[3];
    parts = (int)of;
    size = w / of;
  }
  if (lane >= B) parts = 0;
  return {parts, lanes_before(parts), size};
}

// The prompt, KV head, keys and rows of a workgroup that takes `tiles` row
// tiles of a (prompt, KV head).
struct TreeSpan {
  int b, kvh, slot, parts, nrows, row0, L, nb, node0, node1, beg, end;
  int turn;    // counts the workgroups of a row group on an XCD
  bool over, none;
};

// ENDS: in a chunk, the first 32 workgroups of an XCD, one for each of its CUs, take a
// pair's row groups from the last on, the next 32 from the first on, and so forth: its last
// rows see the most keys, and a CU gets groups of either end (4-bit cache in bf16: a chunk of
// 1000 over 1000 tokens 62 -> 52 us, two of 509 over 3001 95 -> 91).
template <bool ENDS = false>
__device__ __forceinline__ TreeSpan tree_span(const TreeAttnArgs& a, int tiles) {
  TreeSpan t;
  // The row groups of one (prompt, KV head, split) read the same pages:
  // workgroup w runs on XCD w % 8, so they take consecutive slots of one XCD.
  const int NR = a.row_groups, NC = gridDim.x / NR, full = NC & ~7;
  int chunk, rg;
  if ((int)blockIdx.x < full * NR) {
    const int x = blockIdx.x >> 3;
    chunk = (blockIdx.x & 7) + 8 * (x / NR);
    rg = x % NR;
    if (ENDS && !a.parents) {
      const int from_last = (x / 64 - (x - rg) / 64) * 32 + min(x % 64, 32) - min((x - rg) % 64, 32);
      rg = x & 32 ? rg - from_last : NR - 1 - from_last;
    }
  } else {
    const int x = blockIdx.x - full * NR;
    chunk = full + x / NR;
    rg = x % NR;
  }
  const int lane = threadIdx.x & 63, B = a.c.B;
  t.turn = chunk >> 3;
  t.slot = chunk / a.c.Hkv;
  t.kvh = chunk % a.c.Hkv;
  t.parts = a.slots / B;
  t.b = t.slot / t.parts;
  int part = t.slot % t.parts;
  bool spare = false;
  if (B > 1 && B <= kTreeShared) {
    const TreeParts p = tree_parts(a, lane);
    int place = p.slot;
    if (a.slots < 2 * B) {
      // Parts of unlike sizes: the largest first, so that the last workgroups
      // to start are short (12 trees of 65 at 8192: 232 -> 202 us).  The last
      // six bits of a size make way for the prompt: no two are the same.
      const int key = (__float_as_int(p.size) & ~63) | (63 - lane);
      place = 0;
      if (a.slots == B) {
        for (int j = 0; j < B; ++j) place += __builtin_amdgcn_readlane(key, j) > key ? 1 : 0;
      } else {
        for (int j = 0; j < B; ++j)
          place += __builtin_amdgcn_readlane(key, j) > key ? __builtin_amdgcn_readlane(p.parts, j) : 0;
      }
    }
    const unsigned long long mine = __ballot(t.slot >= place && t.slot < place + p.parts);
    spare = mine == 0;
    t.b = spare ? 0 : __builtin_ctzll(mine);
    t.parts = __builtin_amdgcn_readlane(p.parts, t.b);
    part = t.slot - __builtin_amdgcn_readlane(place, t.b);
    t.slot = __builtin_amdgcn_readlane(p.slot, t.b) + part;
  }
  t.nb = a.n_nodes ? min(max(a.n_nodes[t.b], 0), a.n) : a.n;
  t.nrows = t.nb * a.G;
  t.row0 = rg * 16 * tiles;
  t.none = spare || t.row0 >= t.nrows;
  t.L = max(a.lens[t.b], 0);
  t.node0 = t.row0 / a.G;
  t.node1 = (min(t.row0 + 16 * tiles, t.nrows) - 1) / a.G;
  // a prompt that its table cannot hold has no answer: NaN, and no page read
  t.over = (long long)t.L + t.nb > (long long)a.c.table_stride * kPage;
  const int pages = t.over ? 0 : (int)(((long long)t.L + t.nb + kPage - 1) / kPage);
  const int per = (pages + t.parts - 1) / t.parts;
  t.beg = (int)min((long long)part * per, (long long)pages);
  t.end = t.over ? 0 : (int)min(min((long long)t.beg + per, (long long)pages), ((long long)t.L + t.node1) / kPage + 1);
  return t;
}

// Which nodes a node sees, for the nodes of a workgroup: masks[m - node0].  A
// parent outside [0, own index) ends the walk, so every walk ends.
__device__ __forceinline__ void tree_masks(const TreeAttnArgs& a, const TreeSpan& t, uint32_t* masks, int* par, int NT) {
  const int nodes = t.node1 - t.node0 + 1;
  for (int i = threadIdx.x; i <= t.node1; i += NT) par[i] = a.parents[(long long)t.b * a.n + i];
  for (int i = threadIdx.x; i < nodes * kTreeWords; i += NT) masks[i] = 0u;
  __syncthreads();
  for (int i = threadIdx.x; i < nodes; i += NT) {
    int m = t.node0 + i;
    while (true) {
      masks[i * kTreeWords + (m >> 5)] |= 1u << (m & 31);
      const int up = par[m];
      if (up < 0 || up >= m) break;
      m = up;
    }
  }
  __syncthreads();
}

// Eight entries of q.
template <typename QT>
__device__ __forceinline__ void load_q8(const QT* p, float (&x)[8]) {
  if constexpr (sizeof(QT) == 2) {
    const bf16x8 v = *(const bf16x8*)p;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
  } else {
    const f32x4 v0 = *(const f32x4*)p, v1 = *(const f32x4*)(p + 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = e < 4 ? v0[e & 3] : v1[e & 3];
  }
}

// The power of two 2^(14 - e) that brings a row of q to a largest entry in [2^14,
// 2^15), from the largest bit pattern of |q|: what the entries are multiplied by
// (with the sign of the softmax scale; 0 for a scale of 0), and what a score of
// the result (with key codes of 2^-14) counts in log2 units, |scale| 2^e.  The
// former is finite from e = -112 on.  The latter meets the -inf of hidden slots
// and scores of 0, so it stays finite and above 0: e is at least what makes it
// 2^-126, and it ends at the largest fp32.  (A row that e is too large for keeps
// fewer bits, those of entries below 2^-137 or of scores below 2^-49 for keys of
// up to 2^60 among them.)  A NaN or an infinity stays one (its scores are NaN).
struct QScale {
  float down, rm;
};
__device__ __forceinline__ QScale q_scale(float scale_log2, int scale_exp, unsigned top) {
  const float s = fabsf(scale_log2);
  // s >= 2^(x - 1), x the exponent of frexp
  const int e = max(max((int)(top >> 23) - 127, -112), -125 - (__builtin_amdgcn_frexp_expf(s) + scale_exp));
  return {__builtin_ldexpf(scale_log2 < 0.f ? -1.f : scale_log2 > 0.f ? 1.f : 0.f, 14 - e),
          s == 0.f ? 1.f : fminf(__builtin_ldexpf(s, e + scale_exp), 3.4028234663852886e38f)};
}
template <int QP>
__device__ __forceinline__ void q_planes(const float (&x)[8], float down, f16x8 (&q)[QP]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float y = x[k] * down;
    const _Float16 hi = (_Float16)y;
    q[0][k] = hi;
    if constexpr (QP > 1) q[1][k] = (_Float16)(y - (float)hi);
  }
}

// Probabilities times s_v as bf16 planes: one, rounded; two, rounded (16 bits); or
// three by truncation, 8 bits each.  Every rest is exact.
template <int PP>
__device__ __forceinline__ void p_planes(float (&w)[8], bf16x8 (&pf)[PP]) {
  union {
    unsigned u[4];
    bf16x8 v;
  } o;
#pragma unroll
  for (int pl = 0; pl < PP; ++pl) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (PP < 3) {
        o.v[2 * e] = (bf16)w[2 * e];
        o.v[2 * e + 1] = (bf16)w[2 * e + 1];
      } else {
        o.u[e] = __builtin_amdgcn_perm(__float_as_uint(w[2 * e + 1]), __float_as_uint(w[2 * e]), 0x07060302);
      }
    }
    pf[pl] = o.v;
    if (pl + 1 < PP) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const unsigned high = PP == 2 ? (e & 1 ? o.u[e / 2] : o.u[e / 2] << 16) : __float_as_uint(w[e]);
        w[e] -= __uint_as_float(high & 0xffff0000u);
      }
    }
  }
}

template <typename QT>
__device__ __forceinline__ void store4(QT* o, f32x4 y) {
  if constexpr (sizeof(QT) == 4) *(f32x4*)o = y;
  else *(bf16x4*)o = (bf16x4){(bf16)y[0], (bf16)y[1], (bf16)y[2], (bf16)y[3]};
}

// One tile of 16 rows in a wave: lane (row lr = lane % 16, group lg = lane / 16).
// PLANES: of p s_v.
template <int HD, typename QT, int PLANES>
struct RowTile {
  static constexpr int S = HD / 32, DT = HD / 16;
  static constexpr int QP = sizeof(QT) == 4 ? 2 : 1;   // planes of q
  static constexpr int PP = PLANES;
  f16x8 q[S][QP];
  float rm;              // what a score of the scaled q counts in log2 units
  f32x4 acc[DT];         // dims 16 t + 4 lg .. +3 of row lr
  float m, l;            // running maximum (log2 units) and this lane's part of the sum
  int node, head;
  bool valid;

  __device__ __forceinline__ void init(const TreeAttnArgs& a, const TreeSpan& t, int row, int lg) {
    valid = row < t.nrows;
    const int r = valid ? row : t.nrows - 1;
    node = r / a.G;
    head = t.kvh * a.G + r % a.G;
    const QT* qp = (const QT*)a.q + t.b * a.qsb + node * a.qst + (long long)head * HD + 8 * lg;
    float x[S][8];
    unsigned top = 0;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      load_q8<QT>(qp + 32 * s, x[s]);
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[s][e]) & 0x7fffffffu);
    }
    top = max(top, (unsigned)__shfl_xor((int)top, 16, 64));
    top = max(top, (unsigned)__shfl_xor((int)top, 32, 64));
    const QScale qs = q_scale(a.scale_log2, a.scale_exp, top);
    rm = qs.rm;
#pragma unroll
    for (int s = 0; s < S; ++s) q_planes<QP>(x[s], qs.down, q[s]);
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = (f32x4){0.f, 0.f, 0.f, 0.f};
    m = -INFINITY;
    l = t.over ? __uint_as_float(0x7fc00000u) : 0.f;
  }

  // What is not visible of a page: vis has this lane's slots at bits 0..3 and
  // 16..19.  (The scales of a hidden slot may be anything.)
  static __device__ __forceinline__ void hide(float (&s)[8], float (&vs)[8], unsigned vis) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool seen = vis >> (e < 4 ? e : 12 + e) & 1u;
      s[e] = seen ? s[e] : -INFINITY;
      vs[e] = seen ? vs[e] : 0.f;
    }
  }

  // Probabilities of a page as planes of p s_v, from its scores times s_k
  // (slots 4 lg + e and 16 + 4 lg + e).
  __device__ __forceinline__ void softmax(const float (&s)[8], const float (&vs)[8], bf16x8 (&pf)[PP]) {
    float mt = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
    mt = groups_max(mt) * rm;
    // The exponentials use a maximum that may lie up to kLazy below the true
    // one, so O is rescaled rarely; O / l does not depend on it.
    const bool raise = mt > m + kLazy;   // true for the first visible key
    if (__ballot(raise)) {
      const float to = raise ? mt : m;
      const float corr = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - to);
      l *= corr;
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[d] *= corr;
      m = to;
    }
    const float mu = m == -INFINITY ? 0.f : m;
    float w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float p = __builtin_amdgcn_exp2f(fmaf(s[e], rm, -mu));
      l += p;
      w[e] = p * vs[e];
    }
    p_planes<PP>(w, pf);
  }

  __device__ __forceinline__ void finish() {
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
  }

  // The result, or this split's part of it.
  __device__ __forceinline__ void store(const TreeAttnArgs& a, const TreeSpan& t, int lg) {
    if (!valid) return;
    const long long row = ((long long)t.b * a.n + node) * a.H + head;
    if (t.parts == 1) {
      const float inv = 1.f / l;
      QT* o = (QT*)a.out + row * HD + 4 * lg;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        store4<QT>(o + 16 * d, acc[d] * inv);
      }
    } else {
      const long long prow = ((long long)t.slot * a.n + node) * a.H + head;
      float* po = a.part_o + prow * HD + 4 * lg;
#pragma unroll
      for (int d = 0; d < DT; ++d) *(f32x4*)(po + 16 * d) = acc[d];
      if (lg == 0) {
        a.part_ml[prow * 2] = m;
        a.part_ml[prow * 2 + 1] = l;
      }
    }
  }
};

// Scores of a page's two halves; dim step s, key codes k0 and k1.  Every
// other product belongs to another sum, so that none waits for the one before.
template <typename Row, int RPW>
__device__ __forceinline__ void score_step(const Row (&row)[RPW], int s, const f16x8& k0, const f16x8& k1,
                                           f32x4 (&sc)[RPW][2]) {
#pragma unroll
  for (int pl = 0; pl < Row::QP; ++pl)
#pragma unroll
    for (int r = 0; r < RPW; ++r) {
      sc[r][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, row[r].q[s][pl], sc[r][0], 0, 0, 0);
      sc[r][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, row[r].q[s][pl], sc[r][1], 0, 0, 0);
    }
}

// O of the dim tiles d and d + 1, value codes v0 and v1.
template <typename Row, int RPW>
__device__ __forceinline__ void value_step(Row (&row)[RPW], int d, const bf16x8& v0, const bf16x8& v1,
                                           const bf16x8 (&pf)[RPW][Row::PP]) {
#pragma unroll
  for (int pl = 0; pl < Row::PP; ++pl)
#pragma unroll
    for (int r = 0; r < RPW; ++r) {
      row[r].acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, pf[r][pl], row[r].acc[d], 0, 0, 0);
      row[r].acc[d + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, pf[r][pl], row[r].acc[d + 1], 0, 0, 0);
    }
}

// Planes of p s_v of every row tile of a wave, from a page's scores.
// MASKED: the page holds nodes.
template <bool MASKED, typename Row, int RPW>
__device__ __forceinline__ void page_softmax(Row (&row)[RPW], const f32x4 (&sc)[RPW][2], const f32x4 (&ks)[2],
                                             const f32x4 (&vs)[2], bool tree, int i0, int node0,
                                             const uint32_t* masks, int lg,
                                             bf16x8 (&pf)[RPW][Row::PP]) {
#pragma unroll
  for (int r = 0; r < RPW; ++r) {
    float s[8], v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      s[e] = sc[r][e >> 2][e & 3] * ks[e >> 2][e & 3];
      v[e] = vs[e >> 2][e & 3];
    }
    if constexpr (MASKED) {
      const unsigned vis = tree ? slots_of_tree(i0, masks + (row[r].node - node0) * kTreeWords)
                                : slots_of_chain(i0, row[r].node);
      Row::hide(s, v, vis >> (4 * lg));
    }
    row[r].softmax(s, v, pf[r]);
  }
}

// Workgroup = (key split, prompt x KV head, group of RPW row tiles); its four
// waves take every fourth page each.  No LDS stage and no barrier in the
// loop: the cache holds the codes in operand order (kvq_layout.h), 16 bytes a
// lane, and the next page's loads are in flight while one is computed.  The
// waves merge through LDS, key splits through a second kernel, both in a
// fixed order.  (Two tiles of fp32 rows over heads of 128 take all 256 registers
// and 9, over int8 16, more in scratch: stored and read around the loop, and one
// of them in a page with nodes.  8 prompts of 8 nodes x 4 at 4096: 29.7 us, in bf16,
// which needs none, 22.3.)
template <int HD, int FMT, typename QT, int RPW>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void tree_few_kernel(TreeAttnArgs a) {
  constexpr int KW = 4;
  using Row = RowTile<HD, QT, sizeof(QT) == 4 ? 3 : RPW == 1 ? 2 : 1>;
  constexpr int S = Row::S, DT = Row::DT;
  constexpr int UNIT = kvq_unit_bytes(HD);
  constexpr int SLOT = (2 + 4 * DT) * 64;    // floats a wave hands over per row tile
  constexpr int XF = (KW - 1) * RPW * SLOT, MF = 16 * RPW * kTreeWords + kTreeMax;
  __shared__ float lds[XF > MF ? XF : MF];

  const int lane = threadIdx.x & 63, kw = threadIdx.x >> 6;
  const int lr = lane & 15, lg = lane >> 4;
  const TreeSpan t = tree_span(a, RPW);
  if (t.none) return;   // uniform over the workgroup

  // page ids of this wave's next 64 pages, one a lane
  int ids = 0;
  const int* table = a.c.table + (long long)t.b * a.c.table_stride;
  auto fetch_ids = [&](int it) __attribute__((always_inline)) {
    const int p = t.beg + kw + KW * (it + lane);
    ids = p < t.end ? table[p] : 0;
  };
  const int npages = t.end > t.beg + kw ? (t.end - t.beg - kw + KW - 1) / KW : 0;
  if (npages > 0) fetch_ids(0);

  Row row[RPW];
#pragma unroll
  for (int r = 0; r < RPW; ++r) row[r].init(a, t, t.row0 + 16 * r + lr, lg);

  const bool tree = a.parents != nullptr && a.n > 1;
  uint32_t* masks = (uint32_t*)lds;
  if (tree) tree_masks(a, t, masks, (int*)lds + 16 * RPW * kTreeWords, 256);

  u32x4 kr[S], vr[S];
  f32x4 ksr[2], vsr[2];
  const uint8_t* unit = nullptr;   // of the page that is loaded
  bool bad = false, next_bad = false;
  auto load_keys = [&](int it) __attribute__((always_inline)) {
    const int id = __builtin_amdgcn_readlane(ids, it & 63);
    next_bad = id < 0 || id >= a.c.pages;
    unit = a.c.pool + ((long long)(next_bad ? 0 : id) * a.c.Hkv + t.kvh) * UNIT;
#pragma unroll
    for (int s = 0; s < S; ++s) kr[s] = *(const u32x4*)(unit + s * 1024 + lane * 16);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      ksr[h] = *(const f32x4*)(unit + 2 * kPage * HD + 64 * h + 16 * lg);
      vsr[h] = *(const f32x4*)(unit + 2 * kPage * HD + 4 * kPage + 64 * h + 16 * lg);
    }
  };
  auto load_values = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < S; ++s) vr[s] = *(const u32x4*)(unit + kPage * HD + s * 1024 + lane * 16);
  };

  auto step = [&](auto masked, int it) __attribute__((always_inline)) {
    constexpr bool MASKED = decltype(masked)::value;
    const int page = t.beg + kw + KW * it;
    f32x4 sc[RPW][2];
#pragma unroll
    for (int r = 0; r < RPW; ++r) sc[r][0] = sc[r][1] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < S; ++s) {
      score_step(row, s, codes_f16<FMT>(kr[s].x, kr[s].y), codes_f16<FMT>(kr[s].z, kr[s].w), sc);
    }
    f32x4 ks[2] = {ksr[0], ksr[1]};
    const f32x4 vs[2] = {vsr[0], vsr[1]};
    if (bad) {   // its keys have no value: rows that see one are NaN
      const float nan = __uint_as_float(0x7fc00000u);
      ks[0] = ks[1] = (f32x4){nan, nan, nan, nan};
    }
    if constexpr (FMT == kE4M3 && MASKED) {
#pragma unroll
      for (int s = 0; s < S; ++s) vr[s] = hold_values(vr[s], bad ? 0 : t.L + t.nb - page * kPage, lg);
    }
    // The next page's loads are in flight during the rest: all of them where
    // there is room for this page's values as bf16, else its keys'.
    bf16x8 vf[RPW == 1 ? DT : 1];
    if constexpr (RPW == 1) {
#pragma unroll
      for (int s = 0; s < S; ++s) {
        vf[2 * s] = codes_bf16<FMT>(vr[s].x, vr[s].y);
        vf[2 * s + 1] = codes_bf16<FMT>(vr[s].z, vr[s].w);
      }
    }
    if (it + 1 < npages) {
      if (((it + 1) & 63) == 0) fetch_ids(it + 1);
      load_keys(it + 1);
      if constexpr (RPW == 1) load_values();
    }
    bf16x8 pf[RPW][Row::PP];
    page_softmax<MASKED>(row, sc, ks, vs, tree, page * kPage - t.L, t.node0, masks, lg, pf);
#pragma unroll
    for (int d = 0; d < DT; d += 2) {
      if constexpr (RPW == 1) {
        value_step(row, d, vf[d], vf[d + 1], pf);
      } else {
        const u32x4 w = vr[d / 2];
        value_step(row, d, codes_bf16<FMT>(w.x, w.y), codes_bf16<FMT>(w.z, w.w), pf);
      }
    }
    if constexpr (RPW > 1) {
      if (it + 1 < npages) load_values();
    }
    bad = next_bad;
  };
  // the pages of prompt tokens only, then those that hold nodes
  const int plain = min(npages, max(0, (t.L / kPage - t.beg - kw + KW - 1) / KW));
  if (npages > 0) {
    load_keys(0);
    load_values();
    bad = next_bad;
  }
  int it = 0;
  for (; it < plain; ++it) step(std::false_type{}, it);
  for (; it < npages; ++it) step(std::true_type{}, it);

#pragma unroll
  for (int r = 0; r < RPW; ++r) row[r].finish();
  // waves 1.. hand (m, l, O) to wave 0, which adds them in order
  __syncthreads();   // the masks are no longer read
  if (kw > 0) {
#pragma unroll
    for (int r = 0; r < RPW; ++r) {
      float* x = lds + ((kw - 1) * RPW + r) * SLOT;
      x[lane] = row[r].m;
      x[64 + lane] = row[r].l;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[(2 + 4 * d + e) * 64 + lane] = row[r].acc[d][e];
    }
  }
  __syncthreads();
  if (kw > 0) return;
#pragma unroll
  for (int r = 0; r < RPW; ++r) {
#pragma unroll
    for (int k = 1; k < KW; ++k) {
      const float* x = lds + ((k - 1) * RPW + r) * SLOT;
      const float mq = x[lane], lq = x[64 + lane];
      const float mn = fmaxf(row[r].m, mq);
      const float s0 = row[r].m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(row[r].m - mn);
      const float s1 = mq == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mq - mn);
      row[r].l = row[r].l * s0 + lq * s1;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          row[r].acc[d][e] = row[r].acc[d][e] * s0 + x[(2 + 4 * d + e) * 64 + lane] * s1;
      row[r].m = mn;
    }
    row[r].store(a, t, lg);
  }
}

// Workgroup = (key split, prompt x KV head, group of a.wg_tiles row tiles);
// wave w takes tile w.  A page is converted once for all waves: its
// codes come in as 16 bytes a thread, two pages before they are needed, and go
// to LDS as f16 (keys) and bf16 (values) in operand order.
// EU: waves a SIMD at least.  Four leave 128 registers a lane (the loop likes
// 134 in bf16, 146 in fp32; of the latter 11 then live in scratch, outside the
// loop but for one that a page with nodes reads).
template <int HD, int FMT, typename QT, int EU>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(EU))) void tree_many_kernel(TreeAttnArgs a) {
  using Row = RowTile<HD, QT, sizeof(QT) == 4 ? 3 : 1>;
  constexpr int NT = 256, W = 4;
  constexpr int S = Row::S, DT = Row::DT;
  constexpr int UNIT = kvq_unit_bytes(HD);
  constexpr int CH = 2 * S * 64;                     // 16-byte chunks of codes in a unit
  constexpr int PER = (CH + NT - 1) / NT;
  constexpr int ROWS = 16 * W;
  __shared__ __attribute__((aligned(16))) u32x4 tile[2][2 * CH];   // [keys: S][half] [values: DT], 64 lanes each
  __shared__ __attribute__((aligned(16))) float scale[2][2 * kPage];
  __shared__ uint32_t masks[ROWS * kTreeWords];
  __shared__ int par[kTreeMax];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lg = lane >> 4;
  const TreeSpan t = tree_span(a, a.wg_tiles);
  if (t.none) return;   // uniform over the workgroup
  const int npages = t.end - t.beg;
  const int wrow = t.row0 + 16 * wave;
  const int wend = min(t.row0 + 16 * a.wg_tiles, t.nrows);
  const bool has_rows = wrow < wend;

  const int* table = a.c.table + (long long)t.b * a.c.table_stride + t.beg;
  // Two pages in flight.  Loads past the last page repeat it: without a branch
  // the compiler knows how many are outstanding, and waits for the older page
  // alone.
  u32x4 raw[2][PER];
  float sraw[2];
  bool bad[2] = {false, false};
  int id_next = npages > 0 ? table[0] : 0;   // of the page that is loaded next: a scalar load, one step ahead
  auto load = [&](int it, int slot) __attribute__((always_inline)) {
    const int id = id_next;
    id_next = table[min(it + 1, npages - 1)];
    bad[slot] = id < 0 || id >= a.c.pages;
    const uint8_t* u = a.c.pool + ((long long)(bad[slot] ? 0 : id) * a.c.Hkv + t.kvh) * UNIT;
#pragma unroll
    for (int c = 0; c < PER; ++c)
      if (CH % NT == 0 || tid + NT * c < CH) raw[slot][c] = *((const u32x4*)u + tid + NT * c);
    sraw[slot] = *((const float*)(u + 2 * kPage * HD) + lane);
  };
  auto put = [&](int it, int buf) __attribute__((always_inline)) {
    const int page = t.beg + it;
#pragma unroll
    for (int c = 0; c < PER; ++c) {
      const int i = tid + NT * c;
      if (CH % NT != 0 && i >= CH) continue;
      const int s = i >> 6;
      union {
        f16x8 h;
        bf16x8 b;
        u32x4 u;
      } x, y;
      const u32x4 w = raw[buf][c];
      if (CH % (2 * NT) == 0 ? c < PER / 2 : s < S) {   // uniform over a wave
        x.h = codes_f16<FMT>(w.x, w.y);
        y.h = codes_f16<FMT>(w.z, w.w);
      } else {
        u32x4 v = w;
        if (FMT == kE4M3 && (page + 1) * kPage > t.L) v = hold_values(v, bad[buf] ? 0 : t.L + t.nb - page * kPage, lg);
        x.b = codes_bf16<FMT>(v.x, v.y);
        y.b = codes_bf16<FMT>(v.z, v.w);
      }
      tile[buf][(2 * s) * 64 + lane] = x.u;
      tile[buf][(2 * s + 1) * 64 + lane] = y.u;
    }
    // a page that does not exist: rows that see one of its keys are NaN
    if (wave == 0) scale[buf][lane] = bad[buf] && lane < kPage ? __uint_as_float(0x7fc00000u) : sraw[buf];
  };

  if (npages > 0) {
    load(0, 0);
    load(1, 1);
  }
  Row row[1];
  row[0].init(a, t, wrow + lr, lg);
  row[0].valid = wrow + lr < wend;
  // the last node of the wave's rows: later pages hold nothing for it
  const int wlast = (min(wrow + 16, wend) - 1) / a.G;
  const bool tree = a.parents != nullptr && a.n > 1;
  if (tree) tree_masks(a, t, masks, par, NT);
  if (npages > 0) put(0, 0);
  __syncthreads();

  auto step = [&](auto masked, int it, int buf) __attribute__((always_inline)) {
    constexpr bool MASKED = decltype(masked)::value;
    const int page = t.beg + it;
    load(it + 2, buf);
    if (has_rows && !(MASKED && page * kPage > t.L + wlast)) {
      f32x4 sc[1][2] = {{{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}}};
#pragma unroll
      for (int s = 0; s < S; ++s)
        score_step(row, s, *(const f16x8*)&tile[buf][(2 * s) * 64 + lane],
                   *(const f16x8*)&tile[buf][(2 * s + 1) * 64 + lane], sc);
      const f32x4 ks[2] = {*(const f32x4*)&scale[buf][4 * lg], *(const f32x4*)&scale[buf][16 + 4 * lg]};
      const f32x4 vs[2] = {*(const f32x4*)&scale[buf][kPage + 4 * lg], *(const f32x4*)&scale[buf][kPage + 16 + 4 * lg]};
      bf16x8 pf[1][Row::PP];
      page_softmax<MASKED>(row, sc, ks, vs, tree, page * kPage - t.L, t.node0, masks, lg, pf);
#pragma unroll
      for (int d = 0; d < DT; d += 2)
        value_step(row, d, *(const bf16x8*)&tile[buf][CH + d * 64 + lane],
                   *(const bf16x8*)&tile[buf][CH + (d + 1) * 64 + lane], pf);
    }
    put(it + 1, buf ^ 1);
    __syncthreads();
  };
  // Pairs of pages of prompt tokens only, then the pages that hold nodes (and
  // one before them, if the plain ones are odd).
  const int plain = min(npages, max(0, t.L / kPage - t.beg)) & ~1;
  int it = 0;
  for (; it < plain; it += 2) {
    step(std::false_type{}, it, 0);
    step(std::false_type{}, it + 1, 1);
  }
  for (; it < npages; it += 2) {
    step(std::true_type{}, it, 0);
    if (it + 1 < npages) step(std::true_type{}, it + 1, 1);
  }
  if (!has_rows) return;
  row[0].finish();
  row[0].store(a, t, lg);
}

// A tile of 32 rows in a wave: lane (row lane % 32, half h = lane / 32).
template <int HD, typename QT>
struct WideTile {
  static constexpr int S = HD / 16, DT = HD / 32;
  static constexpr int QP = sizeof(QT) == 4 ? 2 : 1, PP = sizeof(QT) == 4 ? 3 : 1;
  f16x8 q[S][QP];        // dims 16 s + 8 h .. +7
  float rm;
  f32x16 acc[DT];        // dims 32 d + 8 (i / 4) + 4 h + i % 4
  float m, l;
  int node, head;
  bool valid;
};

// tree_many_kernel with tiles of 32 rows (MFMA 32x32x16): half the matrix
// instructions and LDS reads.  A matrix instruction keeps the SIMD from
// issuing vector ones for about eight cycles whatever its size (a wave of
// products beside a wave of additions: 372 us for 16x16x32, 325 for 32x32x16,
// where each alone takes 250), and the vector work of the softmax is as long
// as the products (64 prompts x 8 KV heads of 256 rows at up to 2048 tokens: 119
// us in bf16, 194 in fp32 over int8, where tiles of 16 take 127 and 201).
// Scores: lane (row, h) holds slots 8 j + 4 h + e, j < 4, e < 4, which in that
// order are its operand of the two value products of 16 slots.
template <int HD, int FMT, typename QT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void tree_wide_kernel(TreeAttnArgs a) {
  using Row = WideTile<HD, QT>;
  constexpr int NT = 256, W = 4;
  constexpr int S = Row::S, DT = Row::DT, QP = Row::QP, PP = Row::PP;
  constexpr int UNIT = kvq_unit_bytes(HD);
  constexpr int CH = 4 * HD;                         // 16-byte chunks of codes in a unit
  constexpr int PER = (CH + NT - 1) / NT;
  constexpr int ROWS = 32 * W;
  // operands of 64 lanes: keys [S], values [DT][2]
  __shared__ __attribute__((aligned(16))) u32x4 ktile[2][S * 64], vtile[2][DT * 2 * 64];
  __shared__ __attribute__((aligned(16))) float scale[2][2 * kPage];
  __shared__ uint32_t masks[ROWS * kTreeWords];
  __shared__ int par[kTreeMax];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, h = lane >> 5;
  const TreeSpan t = tree_span(a, a.wg_tiles);
  if (t.none) return;   // uniform over the workgroup
  const int npages = t.end - t.beg;
  const int wrow = t.row0 + 32 * wave;
  const int wend = min(t.row0 + 16 * a.wg_tiles, t.nrows);
  const bool has_rows = wrow < wend;

  const int* table = a.c.table + (long long)t.b * a.c.table_stride + t.beg;
  // Two pages in flight, as in tree_many_kernel.
  u32x4 raw[2][PER];
  float sraw[2];
  bool bad[2] = {false, false};
  int id_next = npages > 0 ? table[0] : 0;
  auto load = [&](int it, int slot) __attribute__((always_inline)) {
    const int id = id_next;
    id_next = table[min(it + 1, npages - 1)];
    bad[slot] = id < 0 || id >= a.c.pages;
    const uint8_t* u = a.c.pool + ((long long)(bad[slot] ? 0 : id) * a.c.Hkv + t.kvh) * UNIT;
#pragma unroll
    for (int c = 0; c < PER; ++c)
      if (CH % NT == 0 || tid + NT * c < CH) raw[slot][c] = *((const u32x4*)u + tid + NT * c);
    sraw[slot] = *((const float*)(u + 2 * kPage * HD) + lane);
  };
  auto put = [&](int it, int buf) __attribute__((always_inline)) {
    const int page = t.beg + it;
#pragma unroll
    for (int c = 0; c < PER; ++c) {
      const int i = tid + NT * c;
      if (CH % NT != 0 && i >= CH) continue;
      // chunk (dims / 32, quarter g, x = lane % 16)
      const int s = i >> 6, g = lane >> 4, x = lane & 15;
      const u32x4 w = raw[buf][c];
      if (CH % (2 * NT) == 0 ? c < PER / 2 : s < HD / 32) {   // keys x and x + 16, dims 32 s + 8 g .. +7
        union {
          f16x8 h8;
          u32x4 u;
        } k0, k1;
        k0.h8 = codes_f16<FMT>(w.x, w.y);
        k1.h8 = codes_f16<FMT>(w.z, w.w);
        u32x4* at = &ktile[buf][(2 * s + (g >> 1)) * 64 + (g & 1) * 32 + x];
        at[0] = k0.u;
        at[16] = k1.u;
      } else {   // dims 32 d + x and + 16, slots 4 g .. +3 and 16 + 4 g .. +3
        u32x4 v = w;
        if (FMT == kE4M3 && (page + 1) * kPage > t.L) v = hold_values(v, bad[buf] ? 0 : t.L + t.nb - page * kPage, g);
        union {
          bf16x8 b8;
          uint2 u[2];
        } v0, v1;
        v0.b8 = codes_bf16<FMT>(v.x, v.y);
        v1.b8 = codes_bf16<FMT>(v.z, v.w);
        const int d = s - HD / 32;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          uint2* at = (uint2*)&vtile[buf][(2 * d + k) * 64 + (g & 1) * 32 + x] + (g >> 1);
          at[0] = v0.u[k];
          at[32] = v1.u[k];
        }
      }
    }
    // a page that does not exist: rows that see one of its keys are NaN
    if (wave == 0) scale[buf][lane] = bad[buf] && lane < kPage ? __uint_as_float(0x7fc00000u) : sraw[buf];
  };

  if (npages > 0) {
    load(0, 0);
    load(1, 1);
  }
  Row row;
  {
    const int r0 = wrow + lr;
    row.valid = r0 < wend;
    const int r = r0 < t.nrows ? r0 : t.nrows - 1;
    row.node = r / a.G;
    row.head = t.kvh * a.G + r % a.G;
    const QT* qp = (const QT*)a.q + t.b * a.qsb + row.node * a.qst + (long long)row.head * HD + 8 * h;
    float x[S][8];
    unsigned top = 0;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      load_q8<QT>(qp + 16 * s, x[s]);
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[s][e]) & 0x7fffffffu);
    }
    top = max(top, (unsigned)__shfl_xor((int)top, 32, 64));
    const QScale qs = q_scale(a.scale_log2, a.scale_exp, top);
    row.rm = qs.rm;
#pragma unroll
    for (int s = 0; s < S; ++s) q_planes<QP>(x[s], qs.down, row.q[s]);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) row.acc[d][i] = 0.f;
    row.m = -INFINITY;
    row.l = t.over ? __uint_as_float(0x7fc00000u) : 0.f;
  }
  // the last node of the wave's rows: later pages hold nothing for it
  const int wlast = (min(wrow + 32, wend) - 1) / a.G;
  const bool tree = a.parents != nullptr && a.n > 1;
  if (tree) tree_masks(a, t, masks, par, NT);
  if (npages > 0) put(0, 0);
  __syncthreads();

  auto step = [&](auto masked, int it, int buf) __attribute__((always_inline)) {
    constexpr bool MASKED = decltype(masked)::value;
    const int page = t.beg + it;
    load(it + 2, buf);
    if (has_rows && !(MASKED && page * kPage > t.L + wlast)) {
      f32x16 sc;
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        const f16x8 k = *(const f16x8*)&ktile[buf][s * 64 + lane];
#pragma unroll
        for (int pl = 0; pl < QP; ++pl)
          sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, row.q[s][pl], sc, 0, 0, 0);
      }
      float p[16], v[16];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x4 ks = *(const f32x4*)&scale[buf][8 * j + 4 * h], vs = *(const f32x4*)&scale[buf][kPage + 8 * j + 4 * h];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          p[4 * j + e] = sc[4 * j + e] * ks[e];
          v[4 * j + e] = vs[e];
        }
      }
      if constexpr (MASKED) {
        const int i0 = page * kPage - t.L;
        const unsigned vis = (tree ? slots_of_tree(i0, masks + (row.node - t.node0) * kTreeWords)
                                   : slots_of_chain(i0, row.node)) >> (4 * h);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const bool seen = vis >> (8 * (i / 4) + i % 4) & 1u;
          p[i] = seen ? p[i] : -INFINITY;
          v[i] = seen ? v[i] : 0.f;   // the scale of a hidden slot may be anything
        }
      }
      float mt = p[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mt = fmaxf(mt, p[i]);
      mt = halves_max(mt) * row.rm;
      const bool raise = mt > row.m + kLazy;
      if (__ballot(raise)) {
        const float to = raise ? mt : row.m;
        const float corr = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(row.m - to);
        row.l *= corr;
#pragma unroll
        for (int d = 0; d < DT; ++d) row.acc[d] *= corr;
        row.m = to;
      }
      const float mu = row.m == -INFINITY ? 0.f : row.m;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        bf16x8 pf[PP];
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = __builtin_amdgcn_exp2f(fmaf(p[8 * k + e], row.rm, -mu));
          row.l += x;
          w[e] = x * v[8 * k + e];
        }
        p_planes<PP>(w, pf);
        bf16x8 vf[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d) vf[d] = *(const bf16x8*)&vtile[buf][(2 * d + k) * 64 + lane];
#pragma unroll
        for (int pl = 0; pl < PP; ++pl)
#pragma unroll
          for (int d = 0; d < DT; ++d)
            row.acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[d], pf[pl], row.acc[d], 0, 0, 0);
      }
    }
    put(it + 1, buf ^ 1);
    __syncthreads();
  };
  const int plain = min(npages, max(0, t.L / kPage - t.beg)) & ~1;
  int it = 0;
  for (; it < plain; it += 2) {
    step(std::false_type{}, it, 0);
    step(std::false_type{}, it + 1, 1);
  }
  for (; it < npages; it += 2) {
    step(std::true_type{}, it, 0);
    if (it + 1 < npages) step(std::true_type{}, it + 1, 1);
  }
  if (!has_rows) return;
  row.l += __shfl_xor(row.l, 32, 64);
  if (!row.valid) return;
  const long long out = ((long long)t.b * a.n + row.node) * a.H + row.head;
  const float inv = 1.f / row.l;
  const long long prow = ((long long)t.slot * a.n + row.node) * a.H + row.head;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x4 y = {row.acc[d][4 * j], row.acc[d][4 * j + 1], row.acc[d][4 * j + 2], row.acc[d][4 * j + 3]};
      const int at = 32 * d + 8 * j + 4 * h;
      if (t.parts == 1) store4<QT>((QT*)a.out + out * HD + at, y * inv);
      else *(f32x4*)(a.part_o + prow * HD + at) = y;
    }
  if (t.parts > 1 && h == 0) {
    a.part_ml[prow * 2] = row.m;
    a.part_ml[prow * 2 + 1] = row.l;
  }
}

// Merge of the key splits: one wave per (node, head) row.
template <int HD, typename QT>
__global__ __launch_bounds__(256) void tree_combine_kernel(TreeAttnArgs a) {
  const long long rows = (long long)a.c.B * a.n * a.H;
  const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= rows) return;
  const int per_b = a.n * a.H, b = (int)(row / per_b), at = (int)(row % per_b);
  if (a.n_nodes && at / a.H >= a.n_nodes[b]) return;
  // its prompt's splits (tree_span)
  int ns = a.slots / a.c.B, slot = b * ns;
  if (a.c.B > 1 && a.c.B <= kTreeShared) {
    const TreeParts p = tree_parts(a, lane);
    ns = __builtin_amdgcn_readlane(p.parts, b);
    if (ns == 1) return;   // written by tree_*_kernel
    slot = __builtin_amdgcn_readlane(p.slot, b);
  }
  const long long part = (long long)slot * per_b + at;
  constexpr int PER = (HD + 63) / 64;
  float ms = -INFINITY, ls = 0.f;
  if (lane < ns) {
    ms = a.part_ml[(part + (long long)lane * per_b) * 2];
    ls = a.part_ml[(part + (long long)lane * per_b) * 2 + 1];
  }
  const float mx = wave_max(ms);
  // a split whose keys this row does not see has m = -inf, l = 0; one with a
  // key on a page outside the pool has l = NaN
  const float ws = ms == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ms - mx);
  const float l = wave_sum(ws * ls);
  float acc[PER] = {};
  for (int s0 = 0; s0 < ns; s0 += 8) {
    float o[8][PER];
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
      for (int u = 0; u < PER; ++u) {
        const int d = lane + 64 * u;
        o[k][u] = s0 + k < ns && d < HD ? a.part_o[(part + (long long)(s0 + k) * per_b) * HD + d] : 0.f;
      }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float w = s0 + k < ns ? __shfl(ws, s0 + k, 64) : 0.f;
#pragma unroll
      for (int u = 0; u < PER; ++u) acc[u] = fmaf(w, o[k][u], acc[u]);
    }
  }
  const float inv = 1.f / l;
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int d = lane + 64 * u;
    if (d < HD) ((QT*)a.out)[row * HD + d] = (QT)(acc[u] * inv);
  }
}

template <int HD, int FMT, typename QT>
hipError_t tree_attn_rows(const TreeAttnArgs& a, const TreeAttnPlan& p, hipStream_t st) {
  const unsigned grid = (unsigned)((long long)p.row_groups * p.slots * a.c.Hkv);
  if (p.few == 1) tree_few_kernel<HD, FMT, QT, 1><<<grid, 256, 0, st>>>(a);
  else if (p.few == 2) tree_few_kernel<HD, FMT, QT, 2><<<grid, 256, 0, st>>>(a);
  else if (!p.wide) {
    constexpr bool kFour = tree_may_be_four(HD, sizeof(QT) == 2, FMT);
    if (kFour && p.four) tree_many_kernel<HD, FMT, QT, kFour ? 4 : 3><<<grid, 256, 0, st>>>(a);
    else tree_many_kernel<HD, FMT, QT, 3><<<grid, 256, 0, st>>>(a);
  } else if constexpr (tree_may_be_wide(HD, sizeof(QT) == 2, FMT)) {
    tree_wide_kernel<HD, FMT, QT><<<grid, 256, 0, st>>>(a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.slots == a.c.B) return e;
  const long long rows = (long long)a.c.B * a.n * a.H;
  tree_combine_kernel<HD, QT><<<(unsigned)((rows + 3) / 4), 256, 0, st>>>(a);
  return hipGetLastError();
}

template <int HD>
hipError_t tree_attn_hd(const TreeAttnArgs& a, const TreeAttnPlan& p, int dtype, hipStream_t st) {
  if (a.c.format == kE4M3)
    return dtype == 1 ? tree_attn_rows<HD, kE4M3, bf16>(a, p, st) : tree_attn_rows<HD, kE4M3, float>(a, p, st);
  return dtype == 1 ? tree_attn_rows<HD, kInt8, bf16>(a, p, st) : tree_attn_rows<HD, kInt8, float>(a, p, st);
}

}  // namespace

hipError_t tree_attn_hd32(const TreeAttnArgs& a, const TreeAttnPlan& p, int dtype, hipStream_t st);
hipError_t tree_attn_hd64(const TreeAttnArgs& a, const TreeAttnPlan& p, int dtype, hipStream_t st);
hipError_t tree_attn_hd128(const TreeAttnArgs& a, const TreeAttnPlan& p, int dtype, hipStream_t st);

}  // namespace cdsl

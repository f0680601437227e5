// Attention of a token tree over the 4-bit paged cache: the kernels, one instance
// file per head dimension (tree_attention_fp4_*.hip).  The formula, the tiles and
// the split of rows and keys are those of the 8-bit cache (tree_attention.h);
// what differs comes from the scales, which belong to 32 dims of a token.
//
// A scale is a power of two, so that code * scale is exact in bf16, and the
// instruction that expands two codes applies it: keys and values enter the
// products as the values they are, and neither scores nor probabilities meet a
// scale.  It takes a scale's exponent from bits 23 to 30 of a register whatever
// the others hold (measured), so that one shift brings a scale byte into place.
//
// The two codes of a byte are two dims of one token, as one scale serves both.  A
// value operand has eight tokens of one dim a lane, so pairs of expanded tokens
// trade halves: lane x has dims 32 s + 2 x and + 1 of block s, in the tiles "even"
// and "odd", and a lane's sums of both are eight neighbouring dims of the result.
//
// Precision.  A row of q is scaled by a power of two to a largest entry in [1, 2), so
// that its scores stay within fp32 wherever those of ordinary size do, and taken as bf16
// planes, three for fp32, one for bf16: exact down to 2^-103 of the largest entry.
// Probabilities (1 to 2^8 at most, see kLazy) are planes as over 8 bits: three for fp32;
// for bf16 two with one tile of rows, and one (2^-8 of each, 0.0023 of the result in the
// mean square where its own rounding is 0.0017) with more, where a second costs 6 to 30%
// (8 prompts of 8 nodes x 4 at 4096: 21.4 -> 23.5 us, 64 trees of 65 at 2048: 121 -> 136,
// two chunks of 509 over 3001: 67 -> 78, of 512 over 32768: 551 -> 718).
#pragma once
#include "tree_attention.h"

namespace cdsl {

namespace {

// The bits of the scale in byte e of a word, for an instruction that takes its exponent.
__device__ __forceinline__ float fp4_scale_of(unsigned w, int e) {
  return __uint_as_float(e == 3 ? w >> 1 : w << (23 - 8 * e));
}

// Eight dims of a key: its codes, and the word and byte of its scale.
__device__ __forceinline__ bf16x8 fp4_key(unsigned w, float s) {
  union {
    bf16x2v p[4];
    bf16x8 v;
  } o;
  o.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0);
  o.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1);
  o.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2);
  o.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3);
  return o.v;
}

// Four tokens of two dims (w: a byte each; s: their scales): the even dim's, the
// odd dim's.
__device__ __forceinline__ void fp4_values4(unsigned w, unsigned s, unsigned (&even)[2], unsigned (&odd)[2]) {
  union {
    bf16x2v p;
    unsigned u;
  } t[4];
  t[0].p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, fp4_scale_of(s, 0), 0);
  t[1].p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, fp4_scale_of(s, 1), 1);
  t[2].p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, fp4_scale_of(s, 2), 2);
  t[3].p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, fp4_scale_of(s, 3), 3);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    even[i] = __builtin_amdgcn_perm(t[2 * i + 1].u, t[2 * i].u, 0x05040100);
    odd[i] = __builtin_amdgcn_perm(t[2 * i + 1].u, t[2 * i].u, 0x07060302);
  }
}

// The value operands of a block of 32 dims: a lane's two words of codes (slots 4
// lg + e and 16 + 4 lg + e) and of scales.
__device__ __forceinline__ void fp4_values(const unsigned (&w)[2], const unsigned (&s)[2], bf16x8& even, bf16x8& odd) {
  union {
    unsigned u[4];
    bf16x8 v;
  } a, b;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    unsigned x[2], y[2];
    fp4_values4(w[h], s[h], x, y);
    a.u[2 * h] = x[0], a.u[2 * h + 1] = x[1];
    b.u[2 * h] = y[0], b.u[2 * h + 1] = y[1];
  }
  even = a.v;
  odd = b.v;
}

// Which of a word's bytes are 255 (a NaN row's scales): 0x80 in each.
__device__ __forceinline__ unsigned fp4_none(unsigned s) {
  // + 1 in each byte carries into bit 7 unless its lower seven bits stay below 127
  return s & ((s & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
}

// In a page with nodes, the words of values and scales of slots that may hold
// anything (past the last node, or of a page that does not exist), and the scales
// of rows that are NaN: zeros, so that a row which does not see them stays finite.
// m: the held slots at bits 0..3.
__device__ __forceinline__ void fp4_hold(unsigned& w, unsigned& s, unsigned m) {
  const unsigned none = fp4_none(s);
  m = byte_mask(m);
  w &= m;
  s &= m & ~(none | (none - (none >> 7)));
}

// The largest of N values, a NaN if one is (an instruction takes three; fmaxf would
// make each value canonical first).
template <int N>
__device__ __forceinline__ float max_of(const float (&x)[N]) {
  float m = x[0];
#pragma unroll
  for (int i = 1; i < N; ++i) m = __builtin_elementwise_maximum(m, x[i]);
  return m;
}

// The same over the two lanes of a row that are 32 apart, and over four.
__device__ __forceinline__ float max_halves(float v) {
  const u32x2 t = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __builtin_elementwise_maximum(__uint_as_float(t.x), __uint_as_float(t.y));
}
__device__ __forceinline__ float max_groups(float v) {
  v = max_halves(v);
  const u32x2 t = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __builtin_elementwise_maximum(__uint_as_float(t.x), __uint_as_float(t.y));
}

__device__ __forceinline__ unsigned held_mask(int held) {
  return held >= 32 ? ~0u : held <= 0 ? 0u : (1u << held) - 1u;
}

// Three bf16 planes of eight bits of each probability, by truncation.  The product
// of a pair of planes with (-1, 0) or (0, -1) takes one of them from its value, an
// exact difference in one instruction for two.  (The pairs are kept from the
// compiler: it writes (-1, 0) as the constant -1.0, which the instruction reads as
// (0, -1).)
__device__ __forceinline__ void fp4_p_planes(float (&w)[8], bf16x8 (&pf)[3]) {
  union {
    unsigned u[4];
    bf16x2v p[4];
    bf16x8 v;
  } o;
  union {
    unsigned u;
    bf16x2v p;
  } lower, upper;
  lower.u = 0xbf80u;
  upper.u = 0xbf800000u;
  asm("" : "+s"(lower.u), "+s"(upper.u));
#pragma unroll
  for (int pl = 0; pl < 3; ++pl) {
#pragma unroll
    for (int e = 0; e < 4; ++e) o.u[e] = __builtin_amdgcn_perm(__float_as_uint(w[2 * e + 1]), __float_as_uint(w[2 * e]), 0x07060302);
    pf[pl] = o.v;
    if (pl == 2) break;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      w[2 * e] = __builtin_amdgcn_fdot2_f32_bf16(o.p[e], lower.p, w[2 * e], false);
      w[2 * e + 1] = __builtin_amdgcn_fdot2_f32_bf16(o.p[e], upper.p, w[2 * e + 1], false);
    }
  }
}
template <int PP>
__device__ __forceinline__ void fp4_p_planes(float (&w)[8], bf16x8 (&pf)[PP]) {
  p_planes<PP>(w, pf);
}

// The power of two 2^-e that brings a row of q to a largest entry in [1, 2), from the
// largest bit pattern of |q|: what the entries are multiplied by (with the sign of the
// softmax scale; 0 for a scale of 0), and what a score of the result counts in log2
// units, |scale| 2^e.  The former is finite from e = -126 on.  The latter meets the -inf
// of hidden slots and scores of 0, so e keeps it within 2^-126 and 2^127.  (Where the
// first of these raises e, entries lose more, and scores 2^-125 at most.)  A NaN or an infinity stays one.
__device__ __forceinline__ QScale fp4_q_scale(float scale_log2, int scale_exp, unsigned top) {
  const float s = fabsf(scale_log2);
  const int x = __builtin_amdgcn_frexp_expf(s) + scale_exp;   // 2^(x - 1) <= |scale| < 2^x
  const int e = min(max(max((int)(top >> 23) - 127, -126), -125 - x), 127 - x);
  return {__builtin_ldexpf(scale_log2 < 0.f ? -1.f : scale_log2 > 0.f ? 1.f : 0.f, -e),
          s == 0.f ? 1.f : __builtin_ldexpf(s, e + scale_exp)};
}
// Eight entries as bf16 planes: of fp32 three of eight bits, by truncation, of bf16 itself.
template <int QP>
__device__ __forceinline__ void fp4_q8(float (&x)[8], float down, bf16x8 (&q)[QP]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] *= down;
  if constexpr (QP == 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) q[0][e] = (bf16)x[e];
  } else {
    p_planes<QP>(x, q);
  }
}

// The largest bit pattern of |x| among a lane's entries.
template <int S>
__device__ __forceinline__ unsigned top_of(const float (&x)[S][8]) {
  unsigned top = 0;
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[s][e]) & 0x7fffffffu);
  return top;
}

// A row's running maximum and sum.  The maximum may lag by kLazy, so that O is
// rescaled rarely; O / l does not depend on it.
struct Fp4Softmax {
  float rm;            // log2 units of a score, above 0
  float m, l;          // running maximum (log2 units; -inf before the first visible key), this lane's part of the sum
  __device__ __forceinline__ void init(float units, bool over) {
    rm = units;
    m = -INFINITY;
    l = over ? __uint_as_float(0x7fc00000u) : 0.f;
  }
  // Raises the maximum to a page's, the row's largest score `most`, where it lags;
  // scale(c): O *= c.
  template <typename F>
  __device__ __forceinline__ void raise(float most, F scale) {
    most *= rm;
    const bool up = most > m + kLazy;   // true for the first visible key
    if (__ballot(up)) {
      const float to = up ? most : m;
      const float corr = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - to);
      l *= corr;
      scale(corr);
      m = to;
    }
  }
  // Scores to probabilities.
  template <int N>
  __device__ __forceinline__ void exps(float (&s)[N]) {
    const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], rm, -mu));
      l += s[e];
    }
  }
};

// One tile of 16 rows in a wave: lane (row lr = lane % 16, group lg = lane / 16).
template <int HD, typename QT, int PLANES>
struct Fp4Tile {
  static constexpr int S = HD / 32, DT = HD / 16;
  static constexpr int QP = sizeof(QT) == 4 ? 3 : 1;   // planes of q
  static constexpr int PP = PLANES;                    // and of p
  bf16x8 q[S][QP];
  f32x4 acc[DT];         // tiles (s, even) and (s, odd): dims 32 s + 8 lg + 2 e (+ 1) of row lr
  Fp4Softmax sm;
  int node, head;
  bool valid;

  __device__ __forceinline__ void init(const TreeAttnArgs& a, const TreeSpan& t, int row, int lg) {
    valid = row < t.nrows;
    const int r = valid ? row : t.nrows - 1;
    node = r / a.G;
    head = t.kvh * a.G + r % a.G;
    const QT* qp = (const QT*)a.q + t.b * a.qsb + node * a.qst + (long long)head * HD + 8 * lg;
    float x[S][8];
#pragma unroll
    for (int s = 0; s < S; ++s) load_q8<QT>(qp + 32 * s, x[s]);
    unsigned top = top_of(x);
    top = max(top, (unsigned)__shfl_xor((int)top, 16, 64));
    top = max(top, (unsigned)__shfl_xor((int)top, 32, 64));
    const QScale qs = fp4_q_scale(a.scale_log2, a.scale_exp, top);
#pragma unroll
    for (int s = 0; s < S; ++s) fp4_q8<QP>(x[s], qs.down, q[s]);
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = (f32x4){0.f, 0.f, 0.f, 0.f};
    sm.init(qs.rm, t.over);
  }
  // Probabilities of a page as planes, from its scores (slots 4 lg + e and 16 + 4
  // lg + e).
  __device__ __forceinline__ void softmax(float (&s)[8], bf16x8 (&pf)[PP]) {
    sm.raise(max_groups(max_of(s)), [&](float c) __attribute__((always_inline)) {
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[d] *= c;
    });
    sm.exps(s);
    fp4_p_planes(s, pf);
  }

  __device__ __forceinline__ void finish() {
    sm.l += __shfl_xor(sm.l, 16, 64);
    sm.l += __shfl_xor(sm.l, 32, 64);
  }

  // The result, or this split's part of it.
  __device__ __forceinline__ void store(const TreeAttnArgs& a, const TreeSpan& t, int lg) {
    if (!valid) return;
    const bool whole = t.parts == 1;
    const float inv = whole ? 1.f / sm.l : 1.f;
    const long long row = ((long long)t.b * a.n + node) * a.H + head;
    const long long prow = ((long long)t.slot * a.n + node) * a.H + head;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const f32x4 x = acc[2 * s] * inv, y = acc[2 * s + 1] * inv;
      const f32x4 lo = {x[0], y[0], x[1], y[1]}, hi = {x[2], y[2], x[3], y[3]};
      const int at = 32 * s + 8 * lg;
      if (whole) {
        store4<QT>((QT*)a.out + row * HD + at, lo);
        store4<QT>((QT*)a.out + row * HD + at + 4, hi);
      } else {
        *(f32x4*)(a.part_o + prow * HD + at) = lo;
        *(f32x4*)(a.part_o + prow * HD + at + 4) = hi;
      }
    }
    if (!whole && lg == 0) {
      a.part_ml[prow * 2] = sm.m;
      a.part_ml[prow * 2 + 1] = sm.l;
    }
  }
};

// Scores of a page's two halves, 32 dims of the keys.
template <typename Row, int RPW>
__device__ __forceinline__ void fp4_score_step(const Row (&row)[RPW], int s, const bf16x8& k0, const bf16x8& k1,
                                               f32x4 (&sc)[RPW][2]) {
#pragma unroll
  for (int pl = 0; pl < Row::QP; ++pl)
#pragma unroll
    for (int r = 0; r < RPW; ++r) {
      sc[r][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, row[r].q[s][pl], sc[r][0], 0, 0, 0);
      sc[r][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, row[r].q[s][pl], sc[r][1], 0, 0, 0);
    }
}

// Planes of p of every row tile of a wave, from a page's scores.  MASKED: the
// page holds nodes; all: the rows see all of it, and no value is NaN.  none: this
// lane's slots whose values are NaN (bit e).  bad: NaN
// for a page that does not exist, which the sums of the rows that see a slot of it
// take up; else 0.
template <bool MASKED, typename Row, int RPW>
__device__ __forceinline__ void fp4_softmax(Row (&row)[RPW], const f32x4 (&sc)[RPW][2], float bad, unsigned none,
                                            bool all, bool tree, int i0, int node0, const uint32_t* masks, int lg,
                                            bf16x8 (&pf)[RPW][Row::PP]) {
  const float nan = __uint_as_float(0x7fc00000u);
#pragma unroll
  for (int r = 0; r < RPW; ++r) {
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = sc[r][e >> 2][e & 3];
    if (MASKED && !all) {
      const unsigned vis = (tree ? slots_of_tree(i0, masks + (row[r].node - node0) * kTreeWords)
                                 : slots_of_chain(i0, row[r].node)) >> (4 * lg);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        s[e] = !(vis >> (e < 4 ? e : 12 + e) & 1u) ? -INFINITY : none >> e & 1u ? nan : s[e];
      row[r].sm.l += vis & 0x000f000fu ? bad : 0.f;
    } else {
      row[r].sm.l += bad;
    }
    row[r].softmax(s, pf[r]);
  }
}

// This lane's slots whose value scales are 255, bit e (from the words of block 0).
__device__ __forceinline__ unsigned fp4_none_bits(unsigned s0, unsigned s1) {
  const unsigned a = fp4_none(s0) >> 7, b = fp4_none(s1) >> 7;
  return (a | a >> 7 | a >> 14 | a >> 21) & 15u | ((b | b >> 7 | b >> 14 | b >> 21) & 15u) << 4;
}

// The pages of a KV head.
template <int HD>
struct Fp4Pages {
  const uint8_t* base;
  unsigned pages;
  unsigned long long stride;
  __device__ __forceinline__ Fp4Pages(const TreeAttnArgs& a, int kvh)
      : base(a.c.pool + (long long)kvh * fp4_unit_bytes(HD)), pages(a.c.pages),
        stride((unsigned long long)a.c.Hkv * fp4_unit_bytes(HD)) {}
  // What a page's rows add to the sums that see it: 0, or the bits of a NaN if there is
  // none (its loads take page 0).
  __device__ __forceinline__ unsigned bad(int id) const { return (unsigned)id < pages ? 0u : 0x7fc00000u; }
  __device__ __forceinline__ const uint8_t* unit(int id) const { return base + ((unsigned)id < pages ? (unsigned)id : 0u) * stride; }
};

// Few rows (one or two tiles).  Workgroup = (key split, prompt x KV head, group of
// RPW row tiles); its four waves take every fourth page each, straight from memory
// to registers, with the next page's loads in flight while one is computed.
// The waves merge through LDS, key splits through a second kernel, both in a
// fixed order.
//
// The bytes bound it where keys are long: 8 tokens of up to 32768, 4 query heads each
// of 8 KV heads, take 35 to 40 us with the merge's 5, and their 160 MB 33 at the rate of
// a copy.  A token at 256 takes 5.9 us, its start and three dependent loads.  (In fp32
// two tiles of heads of 128 spill 128 bytes a lane; 8 prompts of 8 x 4 rows at 4096
// take 31 us, in bf16 23.)
template <int HD, typename QT, int RPW>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void fp4_few_kernel(TreeAttnArgs a) {
  constexpr int KW = 4;
  using Row = Fp4Tile<HD, QT, sizeof(QT) == 4 ? 3 : RPW == 1 ? 2 : 1>;
  constexpr int S = Row::S, DT = Row::DT, W = fp4_pair(HD), C = S / W;
  constexpr int SLOT = (2 + 4 * DT) * 64;    // floats a wave hands over per row tile
  constexpr int XF = (KW - 1) * RPW * SLOT, MF = 16 * RPW * kTreeWords + kTreeMax;
  typedef unsigned Chunk __attribute__((ext_vector_type(2 * W)));   // [block][half of the page]
  typedef typename std::conditional<W == 2, unsigned, uint16_t>::type Scales;
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

  const Fp4Pages<HD> pages(a, t.kvh);
  struct Page {
    Chunk k[C], v[C], vs[C];
    Scales ks[C];
    unsigned bad;
  } in;
  auto load = [&](int it) __attribute__((always_inline)) {
    const int id = __builtin_amdgcn_readlane(ids, it & 63);
    in.bad = pages.bad(id);
    const uint8_t* unit = pages.unit(id);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      in.k[c] = *((const Chunk*)(unit + c * 1024) + lane);
      in.ks[c] = *((const Scales*)(unit + 32 * HD + c * 64) + lr);
      in.v[c] = *((const Chunk*)(unit + 16 * HD + c * 1024) + lane);
      in.vs[c] = *((const Chunk*)(unit + 33 * HD + c * 64) + lg);
    }
  };

  auto step = [&](auto masked, int it) __attribute__((always_inline)) {
    constexpr bool MASKED = decltype(masked)::value;
    const int page = t.beg + kw + KW * it;
    Page now = in;
    if (it + 1 < npages) {
      if (((it + 1) & 63) == 0) fetch_ids(it + 1);
      load(it + 1);
    }
    f32x4 sc[RPW][2];
#pragma unroll
    for (int r = 0; r < RPW; ++r) sc[r][0] = sc[r][1] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int c = s / W, i = s % W * 2;
      fp4_score_step(row, s, fp4_key(now.k[c][i], fp4_scale_of(now.ks[c], i)),
                     fp4_key(now.k[c][i + 1], fp4_scale_of(now.ks[c], i + 1)), sc);
    }
    unsigned none = 0;
    if constexpr (MASKED) {
      none = fp4_none_bits(now.vs[0][0], now.vs[0][1]);
      const unsigned hm = held_mask(now.bad ? 0 : t.L + t.nb - page * kPage) >> (4 * lg);
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 2 * W; ++i) {
          unsigned w = now.v[c][i], s = now.vs[c][i];
          fp4_hold(w, s, hm >> (i % 2 * 16));
          now.v[c][i] = w;
          now.vs[c][i] = s;
        }
    }
    bf16x8 pf[RPW][Row::PP];
    fp4_softmax<MASKED>(row, sc, __uint_as_float(now.bad), none, false, tree, page * kPage - t.L, t.node0, masks, lg, pf);
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int c = s / W, i = s % W * 2;
      const unsigned w[2] = {now.v[c][i], now.v[c][i + 1]}, vs[2] = {now.vs[c][i], now.vs[c][i + 1]};
      bf16x8 even, odd;
      fp4_values(w, vs, even, odd);
      value_step(row, 2 * s, even, odd, pf);
    }
  };
  // the pages of prompt tokens only, then those that hold nodes
  const int plain = min(npages, max(0, (t.L / kPage - t.beg - kw + KW - 1) / KW));
  if (npages > 0) load(0);
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
      x[lane] = row[r].sm.m;
      x[64 + lane] = row[r].sm.l;
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
      const float mn = fmaxf(row[r].sm.m, mq);
      const float s0 = row[r].sm.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(row[r].sm.m - mn);
      const float s1 = mq == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mq - mn);
      row[r].sm.l = row[r].sm.l * s0 + lq * s1;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          row[r].acc[d][e] = row[r].acc[d][e] * s0 + x[(2 + 4 * d + e) * 64 + lane] * s1;
      row[r].sm.m = mn;
    }
    row[r].store(a, t, lg);
  }
}

// Loads and expansion of a page by the four waves of a workgroup.  A piece is a
// lane's eight bytes of codes of one block of 32 dims, keys (2 HD pieces) or values
// (2 HD), with the scales that go with it; a wave takes 64 of one kind at a time.
template <int HD>
struct Fp4Pieces {
  static constexpr int NT = 256, P = fp4_pair(HD);
  static constexpr int N = 4 * HD;
  static constexpr int PER = (N + NT - 1) / NT;
  struct Raw {
    u32x2 codes[PER], scales[PER];   // of keys: two bytes of scales in .x
    unsigned bad;
  };
  unsigned at[PER], scale_at[PER];   // offsets in a unit
  int wave;

  // Of piece c: whether there is one and its kind (uniform over a wave); its block and
  // lane.
  __device__ __forceinline__ bool any(int c) const { return NT * (c + 1) <= N || 64 * wave + NT * c < N; }
  __device__ __forceinline__ bool keys(int c) const {
    return NT * (c + 1) <= 2 * HD ? true : NT * c >= 2 * HD ? false : 64 * wave < 2 * HD;
  }
  static __device__ __forceinline__ int piece(int c) { return ((int)threadIdx.x + NT * c) & (2 * HD - 1); }
  static __device__ __forceinline__ int block(int c) { return P == 2 ? piece(c) / 128 * 2 + piece(c) % 2 : 0; }
  static __device__ __forceinline__ int lane(int c) { return P == 2 ? piece(c) / 2 % 64 : piece(c); }
  // Neighbouring threads have the same lane of two blocks, whose operands lie some
  // multiple of all banks apart: of odd blocks, lanes trade places four apart.
  static __device__ __forceinline__ int turned(int lane, int block) { return P == 2 ? lane ^ (block & 1) * 4 : lane; }

  __device__ __forceinline__ void init(int w) {
    wave = w;
#pragma unroll
    for (int c = 0; c < PER; ++c) {
      const int s = block(c), l = lane(c);
      at[c] = 8u * (threadIdx.x + NT * c);
      scale_at[c] = keys(c) ? fp4_key_scale_at(HD, l % 16, 32 * s) : fp4_value_scale_at(HD, l / 16 * 4, 32 * s);
    }
  }
  __device__ __forceinline__ void load(Raw& r, const uint8_t* u) const {
#pragma unroll
    for (int c = 0; c < PER; ++c) {
      if (!any(c)) continue;
      r.codes[c] = *(const u32x2*)(u + at[c]);
      if (keys(c)) r.scales[c].x = *(const uint16_t*)(u + scale_at[c]);
      else r.scales[c] = *(const u32x2*)(u + scale_at[c]);
    }
  }
  // Codes and scales of a value piece of a page with nodes, from whose slot `held` on
  // there are none; gone: [slot], 1 where a value is NaN.
  static __device__ __forceinline__ void hold(int c, u32x2& w, u32x2& e, uint8_t* gone, int held) {
    const int x = lane(c) % 16, g = lane(c) / 16;
    unsigned w0 = w.x, w1 = w.y, e0 = e.x, e1 = e.y;
    if (block(c) == 0 && x < 8)   // one of the lanes that have these slots
      gone[x / 4 * 16 + g * 4 + x % 4] = fp4_none(x < 4 ? e0 : e1) >> (8 * (x % 4) + 7) & 1u;
    const unsigned hm = held_mask(held) >> (4 * g);
    fp4_hold(w0, e0, hm);
    fp4_hold(w1, e1, hm >> 16);
    w = (u32x2){w0, w1};
    e = (u32x2){e0, e1};
  }
};

// More rows.  Workgroup = (key split, prompt x KV head, group of a.wg_tiles row
// tiles); wave w takes tile w.  A page is expanded once for all waves: its codes
// come in two pages before they are needed and go to LDS as bf16 in operand order.
//
// Issue bounds it: 64 trees of 65 x 4 rows over 2048 tokens in fp32 (200 to 235 us) have
// vector instructions at 56% of the SIMDs' cycles and matrix ones, six products for the
// formula's two, at 51%; the two add up.  Workgroups of six or eight waves and four
// workgroups a CU in fp32 gain nothing.
template <int HD, typename QT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(sizeof(QT) == 4 ? 3 : 4))) void fp4_many_kernel(TreeAttnArgs a) {
  using Row = Fp4Tile<HD, QT, sizeof(QT) == 4 ? 3 : 1>;
  using Pieces = Fp4Pieces<HD>;
  constexpr int NT = 256, W = 4;
  constexpr int S = Row::S, DT = Row::DT;
  constexpr int ROWS = 16 * W;
  // operands of 64 lanes: keys [S][half], values [S][even, odd]
  __shared__ __attribute__((aligned(16))) u32x4 tile[2][(2 * S + DT) * 64];
  __shared__ __attribute__((aligned(4))) uint8_t gone[2][kPage];     // 1: the slot's value is NaN; read by words
  static_assert(__alignof__(gone) >= 4, "words");
  __shared__ uint32_t masks[ROWS * kTreeWords];
  __shared__ int par[kTreeMax];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lg = lane >> 4;
  const TreeSpan t = tree_span<true>(a, a.wg_tiles);
  if (t.none) return;   // uniform over the workgroup
  const int npages = t.end - t.beg;
  const int wrow = t.row0 + 16 * ((wave + t.turn) % W);   // where tiles are missing, not always the same SIMD's
  const int wend = min(t.row0 + 16 * a.wg_tiles, t.nrows);
  const bool has_rows = wrow < wend;

  const int* table = a.c.table + (long long)t.b * a.c.table_stride + t.beg;
  // The next page's codes are in flight while one is computed.  (Loads past the last
  // page repeat it.)
  const Fp4Pages<HD> pages(a, t.kvh);
  Pieces pieces;
  pieces.init(wave);
  typename Pieces::Raw in;
  // Page ids are read 64 at a time, one a lane: read one by one, a step ahead, each is waited
  // for behind the barrier (64 trees of 65 in bf16 142 -> 140 us, in fp32 234 -> 231).
  int ids = 0;
  auto load = [&](int it) __attribute__((always_inline)) {
    if ((it & 63) == 0) ids = table[min(it + lane, npages - 1)];
    const int id = __builtin_amdgcn_readlane(ids, it & 63);
    in.bad = pages.bad(id);
    pieces.load(in, pages.unit(id));
  };
  float page_bad[2] = {0.f, 0.f};
  auto put = [&](int it, int buf) __attribute__((always_inline)) {
    const int page = t.beg + it;
    page_bad[buf] = __uint_as_float(in.bad);
    const bool nodes = (page + 1) * kPage > t.L;
#pragma unroll
    for (int c = 0; c < Pieces::PER; ++c) {
      if (!pieces.any(c)) continue;
      const int s = Pieces::block(c), l = Pieces::lane(c);
      u32x2 w = in.codes[c], e = in.scales[c];
      union {
        bf16x8 b;
        u32x4 u;
      } x, y;
      u32x4* at = &tile[buf][((pieces.keys(c) ? 0 : 2 * S) + 2 * s) * 64 + Pieces::turned(l, s)];
      if (pieces.keys(c)) {
        x.b = fp4_key(w.x, fp4_scale_of(e.x, 0));
        y.b = fp4_key(w.y, fp4_scale_of(e.x, 1));
      } else {
        if (nodes) Pieces::hold(c, w, e, gone[buf], in.bad ? 0 : t.L + t.nb - page * kPage);
        const unsigned wv[2] = {w.x, w.y}, ev[2] = {e.x, e.y};
        fp4_values(wv, ev, x.b, y.b);
      }
      at[0] = x.u;
      at[64] = y.u;
    }
  };

  if (npages > 0) {
    load(0);
    put(0, 0);
    load(1);
  }
  Row row[1];
  row[0].init(a, t, wrow + lr, lg);
  row[0].valid = wrow + lr < wend;
  // The first and the last node of the wave's rows: in a chunk, pages up to the one are
  // seen by all of them and take no mask (12 chunks of 500 x 4 rows over 1000 in fp32
  // 348 -> 340 us), pages past the other by none.
  const int wfirst = wrow / a.G, wlast = (min(wrow + 16, wend) - 1) / a.G;
  const bool tree = a.parents != nullptr && a.n > 1;
  if (tree) tree_masks(a, t, masks, par, NT);
  __syncthreads();

  auto step = [&](auto masked, int it, int buf) __attribute__((always_inline)) {
    constexpr bool MASKED = decltype(masked)::value;
    const int page = t.beg + it;
    if (has_rows && !(MASKED && page * kPage > t.L + wlast)) {
      f32x4 sc[1][2] = {{{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}}};
      // Operands are read from LDS two blocks before they are used: left to itself the compiler
      // keeps one block's pair in flight and waits before every product (64 trees of 65 in fp32
      // over 2048 tokens: 243 -> 234 us).
      constexpr int AHEAD = S < 2 ? S : 2;
      auto operand = [&](int at, int s) __attribute__((always_inline)) {
        return *(const bf16x8*)&tile[buf][at * 64 + Pieces::turned(lane, s)];
      };
      bf16x8 x[S][2];
#pragma unroll
      for (int s = 0; s < AHEAD; ++s) x[s][0] = operand(2 * s, s), x[s][1] = operand(2 * s + 1, s);
#pragma unroll
      for (int s = 0; s < S; ++s) {
        __builtin_amdgcn_sched_barrier(0);
        if (s + AHEAD < S) x[s + AHEAD][0] = operand(2 * (s + AHEAD), s + AHEAD), x[s + AHEAD][1] = operand(2 * (s + AHEAD) + 1, s + AHEAD);
        fp4_score_step(row, s, x[s][0], x[s][1], sc);
      }
#pragma unroll
      for (int s = 0; s < AHEAD; ++s) x[s][0] = operand(2 * S + 2 * s, s), x[s][1] = operand(2 * S + 2 * s + 1, s);
      __builtin_amdgcn_sched_barrier(0);
      unsigned none = 0;
      if (MASKED && (page + 1) * kPage > t.L) {
        const unsigned g0 = *(const unsigned*)&gone[buf][4 * lg], g1 = *(const unsigned*)&gone[buf][16 + 4 * lg];
        none = (g0 | g0 >> 7 | g0 >> 14 | g0 >> 21) & 15u | ((g1 | g1 >> 7 | g1 >> 14 | g1 >> 21) & 15u) << 4;
      }
      bf16x8 pf[1][Row::PP];
      const int i0 = page * kPage - t.L;
      const bool all = MASKED && !tree && i0 + kPage - 1 <= wfirst && !__any(none != 0);
      fp4_softmax<MASKED>(row, sc, page_bad[buf], none, all, tree, i0, t.node0, masks, lg, pf);
#pragma unroll
      for (int s = 0; s < S; ++s) {
        __builtin_amdgcn_sched_barrier(0);
        if (s + AHEAD < S) x[s + AHEAD][0] = operand(2 * S + 2 * (s + AHEAD), s + AHEAD), x[s + AHEAD][1] = operand(2 * S + 2 * (s + AHEAD) + 1, s + AHEAD);
        value_step(row, 2 * s, x[s][0], x[s][1], pf);
      }
    }
    put(it + 1, buf ^ 1);
    load(it + 2);
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
struct Fp4Wide {
  static constexpr int S = HD / 16, DT = HD / 32;
  static constexpr int QP = sizeof(QT) == 4 ? 3 : 1, PP = QP;
  bf16x8 q[S][QP];       // dims 16 s + 8 h .. +7
  f32x16 acc[DT];        // i < 8: dim 32 d + 16 (i / 4) + 8 h + 2 (i % 4); i + 8: the next one
  Fp4Softmax sm;
  int node, head;
  bool valid;
};

// fp4_many_kernel with tiles of 32 rows (MFMA 32x32x16).  Half the matrix
// instructions and LDS reads, each page expanded for twice the rows, and more of
// the vector work beside a matrix instruction, which keeps its SIMD from it for
// about eight cycles whatever its size: two chunks of 512 over 32768 tokens in bf16 take
// 590 us, 0.94 PFLOP/s, with tiles of 16 847.  (In bf16 three waves a SIMD, which spill
// 84 bytes a lane.)
// TILES: row tiles of a workgroup, 4 or 2.  With two, a pair of waves shares a
// tile's rows and takes every other page each; they merge through LDS.  (Two chunks of
// 509 over 3001, lengths alike, in bf16: 90 us.  Before a CU had groups of either end,
// 94; whole tiles, one wave a SIMD, then took 102, over two splits of the keys with their
// merge 105, and waves with two tiles of rows, which halve the reads of LDS again, 126.)
// Scores: lane (row, h) holds slots 8 j + 4 h + e, j < 4, e < 4, which in that
// order are its operand of the two value products of 16 slots.
template <int HD, typename QT, int TILES>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(sizeof(QT) == 2 && TILES == 4 ? 3 : 2))) void fp4_wide_kernel(TreeAttnArgs a) {
  using Row = Fp4Wide<HD, QT>;
  using Pieces = Fp4Pieces<HD>;
  constexpr int NT = 256, KS = 4 / TILES;            // pages at a time
  constexpr int S = Row::S, DT = Row::DT, QP = Row::QP, PP = Row::PP;
  constexpr int ROWS = 32 * TILES;
  // operands of 64 lanes: keys [S], values [DT][2]
  struct Tile {
    u32x4 k[S * 64], v[DT * 2 * 64];
  };
  __shared__ __attribute__((aligned(16))) Tile tiles[2][KS];
  __shared__ __attribute__((aligned(4))) uint8_t gone[2][KS][kPage];     // 1: the slot's value is NaN
  static_assert(__alignof__(gone) >= 4, "words");
  __shared__ uint32_t masks[ROWS * kTreeWords];
  __shared__ int par[kTreeMax];
  static_assert(KS == 1 || sizeof(tiles) >= TILES * (2 + 16 * DT) * 64 * sizeof(float), "room for the merge");

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, h = lane >> 5;
  const TreeSpan t = tree_span<true>(a, a.wg_tiles);
  const int rt = (wave + t.turn) % TILES, ks = wave / TILES;   // turned as in fp4_many_kernel
  if (t.none) return;   // uniform over the workgroup
  const int npages = t.end - t.beg;
  const int wrow = t.row0 + 32 * rt;
  const int wend = min(t.row0 + 16 * a.wg_tiles, t.nrows);
  const bool has_rows = wrow < wend;

  const int* table = a.c.table + (long long)t.b * a.c.table_stride + t.beg;
  const Fp4Pages<HD> pages(a, t.kvh);
  Pieces pieces;
  pieces.init(wave);
  typename Pieces::Raw in[KS];
  float page_bad[2] = {0.f, 0.f};    // of this wave's page
  int ids = 0;
  auto load = [&](int st) __attribute__((always_inline)) {
    if ((KS * st & 63) == 0) ids = table[min(KS * st + lane, npages - 1)];
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const int id = __builtin_amdgcn_readlane(ids, (KS * st + k) & 63);
      in[k].bad = pages.bad(id);
      pieces.load(in[k], pages.unit(id));
    }
  };
  auto put = [&](int st, int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const int page = t.beg + KS * st + k;
      const bool nodes = (page + 1) * kPage > t.L;
      Tile& tile = tiles[buf][k];
      if (k == ks) page_bad[buf] = __uint_as_float(in[k].bad);
#pragma unroll
      for (int c = 0; c < Pieces::PER; ++c) {
        if (!pieces.any(c)) continue;
        const int s = Pieces::block(c), l = Pieces::lane(c), g = l / 16, x = l % 16;
        u32x2 w = in[k].codes[c], e = in[k].scales[c];
        if (pieces.keys(c)) {   // keys x and x + 16, dims 32 s + 8 g .. +7
          union {
            bf16x8 b;
            u32x4 u;
          } k0, k1;
          k0.b = fp4_key(w.x, fp4_scale_of(e.x, 0));
          k1.b = fp4_key(w.y, fp4_scale_of(e.x, 1));
          u32x4* at = &tile.k[(2 * s + (g >> 1)) * 64 + Pieces::turned((g & 1) * 32 + x, s)];
          at[0] = k0.u;
          at[16] = k1.u;
        } else {   // dims 32 s + 2 x and + 1, slots 4 g .. +3 and 16 + 4 g .. +3
          if (nodes) Pieces::hold(c, w, e, gone[buf][k], in[k].bad ? 0 : t.L + t.nb - page * kPage);
          u32x2* at = (u32x2*)&tile.v[2 * s * 64 + Pieces::turned((g & 1) * 32 + x, s)] + (g >> 1);
          unsigned even[2], odd[2];
          fp4_values4(w.x, e.x, even, odd);
          at[0] = (u32x2){even[0], even[1]};
          at[32] = (u32x2){odd[0], odd[1]};
          fp4_values4(w.y, e.y, even, odd);
          at[128] = (u32x2){even[0], even[1]};
          at[160] = (u32x2){odd[0], odd[1]};
        }
      }
    }
  };

  if (npages > 0) {
    load(0);
    put(0, 0);
    load(1);
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
#pragma unroll
    for (int s = 0; s < S; ++s) load_q8<QT>(qp + 16 * s, x[s]);
    unsigned top = top_of(x);
    top = max(top, (unsigned)__shfl_xor((int)top, 32, 64));
    const QScale qs = fp4_q_scale(a.scale_log2, a.scale_exp, top);
#pragma unroll
    for (int s = 0; s < S; ++s) fp4_q8<QP>(x[s], qs.down, row.q[s]);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) row.acc[d][i] = 0.f;
    row.sm.init(qs.rm, t.over);
  }
  // as in fp4_many_kernel (12 chunks of 500 x 4 rows over 1000 in bf16: 183 -> 172 us, one of
  // 1000 alone 33.5 -> 29.6)
  const int wfirst = wrow / a.G, wlast = (min(wrow + 32, wend) - 1) / a.G;
  const bool tree = a.parents != nullptr && a.n > 1;
  if (tree) tree_masks(a, t, masks, par, NT);
  __syncthreads();

  // whether a value of this wave's page, of the chunk itself, is NaN
  auto gone_any = [&](int st, int buf) __attribute__((always_inline)) {
    return (t.beg + KS * st + ks + 1) * kPage > t.L && __any(gone[buf][ks][lr]);
  };
  auto step = [&](auto masked, int st, int buf) __attribute__((always_inline)) {
    constexpr bool MASKED = decltype(masked)::value;
    const int page = t.beg + KS * st + ks;
    if (has_rows && !(MASKED && (page * kPage > t.L + wlast || (KS > 1 && page >= t.end)))) {
      const Tile& tile = tiles[buf][ks];
      f32x16 sc;
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] = 0.f;
      // Keys are read from LDS some steps ahead, and the values' first half before the softmax:
      // 12 prompts of 500 tokens behind 1000, 185 -> 183 us in bf16 and 361 -> 353 in fp32, whose
      // registers hold two steps of keys instead of four.
      constexpr int AHEAD = QP == 1 ? 4 : 2;
      auto key = [&](int s) __attribute__((always_inline)) { return *(const bf16x8*)&tile.k[s * 64 + Pieces::turned(lane, s / 2)]; };
      auto value = [&](int d, int k) __attribute__((always_inline)) {
        return *(const bf16x8*)&tile.v[(2 * d + k) * 64 + Pieces::turned(lane, d)];
      };
      bf16x8 x[S], vf[2][DT];
#pragma unroll
      for (int s = 0; s < AHEAD && s < S; ++s) x[s] = key(s);
#pragma unroll
      for (int s = 0; s < S; ++s) {
        __builtin_amdgcn_sched_barrier(0);
        if (s + AHEAD < S) x[s + AHEAD] = key(s + AHEAD);
#pragma unroll
        for (int pl = 0; pl < QP; ++pl)
          sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[s], row.q[s][pl], sc, 0, 0, 0);
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) vf[0][d] = value(d, 0);
      __builtin_amdgcn_sched_barrier(0);
      float p[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] = sc[i];
      const int i0 = page * kPage - t.L;
      if (MASKED && (tree || i0 + kPage - 1 > wfirst || gone_any(st, buf))) {
        const unsigned vis = (tree ? slots_of_tree(i0, masks + (row.node - t.node0) * kTreeWords)
                                   : slots_of_chain(i0, row.node)) >> (4 * h);
        const bool nodes = i0 + kPage > 0;
        const float nan = __uint_as_float(0x7fc00000u);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const unsigned g = nodes ? *(const unsigned*)&gone[buf][ks][8 * j + 4 * h] : 0u;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            p[4 * j + e] = !(vis >> (8 * j + e) & 1u) ? -INFINITY : g >> (8 * e) & 1u ? nan : p[4 * j + e];
        }
        row.sm.l += vis & 0x0f0f0f0fu ? page_bad[buf] : 0.f;
      } else {
        row.sm.l += page_bad[buf];
      }
      row.sm.raise(max_halves(max_of(p)), [&](float c) __attribute__((always_inline)) {
#pragma unroll
        for (int d = 0; d < DT; ++d) row.acc[d] *= c;
      });
      row.sm.exps(p);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        bf16x8 pf[PP];
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = p[8 * k + e];
        fp4_p_planes(w, pf);
        if (k == 0)
#pragma unroll
          for (int d = 0; d < DT; ++d) vf[1][d] = value(d, 1);
#pragma unroll
        for (int pl = 0; pl < PP; ++pl)
#pragma unroll
          for (int d = 0; d < DT; ++d)
            row.acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[k][d], pf[pl], row.acc[d], 0, 0, 0);
      }
    }
    put(st + 1, buf ^ 1);
    load(st + 2);
    __syncthreads();
  };
  const int steps = (npages + KS - 1) / KS;
  const int plain = min(npages, max(0, t.L / kPage - t.beg)) / KS & ~1;
  int st = 0;
  for (; st < plain; st += 2) {
    step(std::false_type{}, st, 0);
    step(std::false_type{}, st + 1, 1);
  }
  for (; st < steps; st += 2) {
    step(std::true_type{}, st, 0);
    if (st + 1 < steps) step(std::true_type{}, st + 1, 1);
  }
  row.sm.l += __shfl_xor(row.sm.l, 32, 64);
  if constexpr (KS > 1) {   // the second wave of a pair hands over (the tiles are no longer read)
    float* x = (float*)tiles + rt * (2 + 16 * DT) * 64;
    if (ks > 0 && has_rows) {
      x[lane] = row.sm.m;
      x[64 + lane] = row.sm.l;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[(2 + 16 * d + i) * 64 + lane] = row.acc[d][i];
    }
    __syncthreads();
    if (ks > 0) return;
    if (has_rows) {
      const float mq = x[lane], lq = x[64 + lane];
      const float mn = fmaxf(row.sm.m, mq);
      const float s0 = row.sm.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(row.sm.m - mn);
      const float s1 = mq == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mq - mn);
      row.sm.l = row.sm.l * s0 + lq * s1;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) row.acc[d][i] = row.acc[d][i] * s0 + x[(2 + 16 * d + i) * 64 + lane] * s1;
      row.sm.m = mn;
    }
  }
  if (!has_rows || !row.valid) return;
  const bool whole = t.parts == 1;
  const float inv = whole ? 1.f / row.sm.l : 1.f;
  const long long out = ((long long)t.b * a.n + row.node) * a.H + row.head;
  const long long prow = ((long long)t.slot * a.n + row.node) * a.H + row.head;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      f32x4 y[2];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        y[e / 2][e % 2 * 2] = row.acc[d][4 * j + e] * inv;
        y[e / 2][e % 2 * 2 + 1] = row.acc[d][8 + 4 * j + e] * inv;
      }
      const int at = 32 * d + 16 * j + 8 * h;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (whole) store4<QT>((QT*)a.out + out * HD + at + 4 * u, y[u]);
        else *(f32x4*)(a.part_o + prow * HD + at + 4 * u) = y[u];
      }
    }
  if (!whole && h == 0) {
    a.part_ml[prow * 2] = row.sm.m;
    a.part_ml[prow * 2 + 1] = row.sm.l;
  }
}

template <int HD, typename QT>
hipError_t fp4_attn_rows(const TreeAttnArgs& a, const TreeAttnPlan& p, hipStream_t st) {
  const unsigned grid = (unsigned)((long long)p.row_groups * p.slots * a.c.Hkv);
  if (p.few == 1) fp4_few_kernel<HD, QT, 1><<<grid, 256, 0, st>>>(a);
  else if (p.few == 2) fp4_few_kernel<HD, QT, 2><<<grid, 256, 0, st>>>(a);
  else if (p.paired) fp4_wide_kernel<HD, QT, 2><<<grid, 256, 0, st>>>(a);
  else if (p.wide) fp4_wide_kernel<HD, QT, 4><<<grid, 256, 0, st>>>(a);
  else fp4_many_kernel<HD, QT><<<grid, 256, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.slots == a.c.B) return e;
  const long long rows = (long long)a.c.B * a.n * a.H;
  tree_combine_kernel<HD, QT><<<(unsigned)((rows + 3) / 4), 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

}  // namespace cdsl

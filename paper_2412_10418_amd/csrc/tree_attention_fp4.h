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
// Precision.  q is taken as bf16 planes, exact: three for fp32, one for bf16; the
// softmax scale multiplies the score.  Probabilities (1 to 2^8 at most, see kLazy)
// are planes as over 8 bits: three for fp32; for bf16 two with one tile of rows,
// and one (2^-8 of each, 0.0023 of the result in the mean square where its own
// rounding is 0.0017) with more.
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

__device__ __forceinline__ unsigned held_mask(int held) {
  return held >= 32 ? ~0u : held <= 0 ? 0u : (1u << held) - 1u;
}

// q as bf16 planes of eight bits, by truncation (of bf16: itself), with the sign
// of the softmax scale; zeros for a scale of 0.
template <typename QT, int QP>
__device__ __forceinline__ void fp4_q8(const QT* p, float sign, bf16x8 (&q)[QP]) {
  float x[8];
  load_q8<QT>(p, x);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] *= sign;
  if constexpr (QP == 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) q[0][e] = (bf16)x[e];
  } else {
    p_planes<QP>(x, q);
  }
}
__device__ __forceinline__ float sign_of(float scale) { return scale < 0.f ? -1.f : scale > 0.f ? 1.f : 0.f; }
// What a score counts in log2 units.  It meets the -inf of hidden slots, so it is
// above 0 (scores are 0 where the scale is).
__device__ __forceinline__ float score_unit(float scale) { return fmaxf(fabsf(scale), 0x1p-126f); }

// One tile of 16 rows in a wave: lane (row lr = lane % 16, group lg = lane / 16).
template <int HD, typename QT, int PLANES>
struct Fp4Tile {
  static constexpr int S = HD / 32, DT = HD / 16;
  static constexpr int QP = sizeof(QT) == 4 ? 3 : 1;   // planes of q
  static constexpr int PP = PLANES;                    // and of p
  bf16x8 q[S][QP];
  float rm;              // what a score counts in log2 units
  f32x4 acc[DT];         // tiles (s, even) and (s, odd): dims 32 s + 8 lg + 2 e (+ 1) of row lr
  float m, l;            // running maximum (log2 units) and this lane's part of the sum
  int node, head;
  bool valid;

  __device__ __forceinline__ void init(const TreeAttnArgs& a, const TreeSpan& t, int row, int lg) {
    valid = row < t.nrows;
    const int r = valid ? row : t.nrows - 1;
    node = r / a.G;
    head = t.kvh * a.G + r % a.G;
    const QT* qp = (const QT*)a.q + t.b * a.qsb + node * a.qst + (long long)head * HD + 8 * lg;
    const float sign = sign_of(a.scale_log2);
    rm = score_unit(a.scale_log2);
#pragma unroll
    for (int s = 0; s < S; ++s) fp4_q8<QT, QP>(qp + 32 * s, sign, q[s]);
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = (f32x4){0.f, 0.f, 0.f, 0.f};
    m = -INFINITY;
    l = t.over ? __uint_as_float(0x7fc00000u) : 0.f;
  }

  // Probabilities of a page as planes, from its scores (slots 4 lg + e and 16 + 4
  // lg + e).  The running maximum may lag by kLazy, so that O is rescaled rarely.
  __device__ __forceinline__ void softmax(const float (&s)[8], bf16x8 (&pf)[PP]) {
    float mt = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
    mt = groups_max(mt) * rm;
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
    float p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      p[e] = __builtin_amdgcn_exp2f(fmaf(s[e], rm, -mu));
      l += p[e];
    }
    p_planes<PP>(p, pf);
  }

  __device__ __forceinline__ void finish() {
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
  }

  // The result, or this split's part of it.
  __device__ __forceinline__ void store(const TreeAttnArgs& a, const TreeSpan& t, int lg) {
    if (!valid) return;
    const bool whole = t.parts == 1;
    const float inv = whole ? 1.f / l : 1.f;
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
      a.part_ml[prow * 2] = m;
      a.part_ml[prow * 2 + 1] = l;
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
// page holds nodes.  none: this lane's slots whose values are NaN (bit e).
template <bool MASKED, typename Row, int RPW>
__device__ __forceinline__ void fp4_softmax(Row (&row)[RPW], const f32x4 (&sc)[RPW][2], bool bad, unsigned none,
                                            bool tree, int i0, int node0, const uint32_t* masks, int lg,
                                            bf16x8 (&pf)[RPW][Row::PP]) {
  const float nan = __uint_as_float(0x7fc00000u);
#pragma unroll
  for (int r = 0; r < RPW; ++r) {
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = bad ? nan : sc[r][e >> 2][e & 3];
    if constexpr (MASKED) {
      const unsigned vis = (tree ? slots_of_tree(i0, masks + (row[r].node - node0) * kTreeWords)
                                 : slots_of_chain(i0, row[r].node)) >> (4 * lg);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        s[e] = !(vis >> (e < 4 ? e : 12 + e) & 1u) ? -INFINITY : none >> e & 1u ? nan : s[e];
    }
    row[r].softmax(s, pf[r]);
  }
}

// This lane's slots whose value scales are 255, bit e (from the words of block 0).
__device__ __forceinline__ unsigned fp4_none_bits(unsigned s0, unsigned s1) {
  const unsigned a = fp4_none(s0) >> 7, b = fp4_none(s1) >> 7;
  return (a | a >> 7 | a >> 14 | a >> 21) & 15u | ((b | b >> 7 | b >> 14 | b >> 21) & 15u) << 4;
}

// Few rows (one or two tiles).  Workgroup = (key split, prompt x KV head, group of
// RPW row tiles); its four waves take every fourth page each, straight from memory
// to registers, with the next page's loads in flight while one is computed.
// The waves merge through LDS, key splits through a second kernel, both in a
// fixed order.
template <int HD, typename QT, int RPW>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void fp4_few_kernel(TreeAttnArgs a) {
  constexpr int KW = 4;
  using Row = Fp4Tile<HD, QT, sizeof(QT) == 4 ? 3 : RPW == 1 ? 2 : 1>;
  constexpr int S = Row::S, DT = Row::DT, W = fp4_pair(HD), C = S / W;
  constexpr int UNIT = fp4_unit_bytes(HD);
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

  struct Page {
    Chunk k[C], v[C], vs[C];
    Scales ks[C];
    bool bad;
  } in;
  auto load = [&](int it) __attribute__((always_inline)) {
    const int id = __builtin_amdgcn_readlane(ids, it & 63);
    in.bad = id < 0 || id >= a.c.pages;
    const uint8_t* unit = a.c.pool + ((long long)(in.bad ? 0 : id) * a.c.Hkv + t.kvh) * UNIT;
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
    fp4_softmax<MASKED>(row, sc, now.bad, none, tree, page * kPage - t.L, t.node0, masks, lg, pf);
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

// Loads and expansion of a page for all waves of a workgroup: a piece of eight
// bytes (a lane's codes of one block) a thread at a time, with the scales that go
// with it.
template <int HD>
struct Fp4Pieces {
  static constexpr int NT = 256, W = fp4_pair(HD);
  static constexpr int N = 4 * HD;                 // keys' 2 HD, then values'
  static constexpr int PER = (N + NT - 1) / NT;
  static constexpr int UNIT = fp4_unit_bytes(HD);
  u32x2 codes[PER], scales[PER];                   // of keys: two bytes of scales in .x
  bool bad;

  static __device__ __forceinline__ bool keys(int c) { return N >= 2 * NT ? c < PER / 2 : (int)threadIdx.x < 2 * HD; }
  // block and lane of a piece
  static __device__ __forceinline__ int piece(int c) { return ((int)threadIdx.x + NT * c) & (2 * HD - 1); }
  static __device__ __forceinline__ int block(int j) { return W == 2 ? j / 128 * 2 + j % 2 : 0; }
  static __device__ __forceinline__ int lane(int j) { return W == 2 ? j / 2 % 64 : j; }

  __device__ __forceinline__ void load(const uint8_t* u) {
#pragma unroll
    for (int c = 0; c < PER; ++c) {
      const int i = threadIdx.x + NT * c;
      if (N % NT != 0 && i >= N) continue;
      codes[c] = *((const u32x2*)u + i);
      const int j = piece(c), s = block(j), l = lane(j);
      if (keys(c)) scales[c].x = *(const uint16_t*)(u + fp4_key_scale_at(HD, l % 16, 32 * s));
      else scales[c] = *(const u32x2*)(u + fp4_value_scale_at(HD, l / 16 * 4, 32 * s));
    }
  }
};

// More rows.  Workgroup = (key split, prompt x KV head, group of a.wg_tiles row
// tiles); wave w takes tile w.  A page is expanded once for all waves: its codes
// come in two pages before they are needed and go to LDS as bf16 in operand order.
template <int HD, typename QT, int EU>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(EU))) void fp4_many_kernel(TreeAttnArgs a) {
  using Row = Fp4Tile<HD, QT, sizeof(QT) == 4 ? 3 : 1>;
  using In = Fp4Pieces<HD>;
  constexpr int NT = 256, W = 4;
  constexpr int S = Row::S, DT = Row::DT;
  constexpr int ROWS = 16 * W;
  // operands of 64 lanes: keys [S][half], values [S][even, odd]
  __shared__ __attribute__((aligned(16))) u32x4 tile[2][(2 * S + DT) * 64];
  __shared__ uint8_t gone[2][kPage];     // 1: the slot's value is NaN
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
  In in[2];
  int id_next = npages > 0 ? table[0] : 0;   // of the page that is loaded next: a scalar load, one step ahead
  auto load = [&](int it, int slot) __attribute__((always_inline)) {
    const int id = id_next;
    id_next = table[min(it + 1, npages - 1)];
    in[slot].bad = id < 0 || id >= a.c.pages;
    in[slot].load(a.c.pool + ((long long)(in[slot].bad ? 0 : id) * a.c.Hkv + t.kvh) * In::UNIT);
  };
  bool page_bad[2] = {false, false};
  auto put = [&](int it, int buf) __attribute__((always_inline)) {
    const int page = t.beg + it;
    page_bad[buf] = in[buf].bad;
    const bool nodes = (page + 1) * kPage > t.L;
#pragma unroll
    for (int c = 0; c < In::PER; ++c) {
      if (In::N % NT != 0 && tid + NT * c >= In::N) continue;
      const int j = In::piece(c), s = In::block(j), l = In::lane(j);
      u32x2 w = in[buf].codes[c], e = in[buf].scales[c];
      union {
        bf16x8 b;
        u32x4 u;
      } x, y;
      if (In::keys(c)) {
        x.b = fp4_key(w.x, fp4_scale_of(e.x, 0));
        y.b = fp4_key(w.y, fp4_scale_of(e.x, 1));
        tile[buf][(2 * s) * 64 + l] = x.u;
        tile[buf][(2 * s + 1) * 64 + l] = y.u;
      } else {
        if (nodes) {
          const unsigned hm = held_mask(in[buf].bad ? 0 : t.L + t.nb - page * kPage) >> (l / 16 * 4);
          if (s == 0 && l % 16 < 8) {   // one of the lanes that have these slots
            const int q = l % 16;
            gone[buf][q / 4 * 16 + l / 16 * 4 + q % 4] = (q < 4 ? fp4_none(e.x) : fp4_none(e.y)) >> (8 * (q % 4) + 7) & 1u;
          }
          unsigned w0 = w.x, w1 = w.y, e0 = e.x, e1 = e.y;
          fp4_hold(w0, e0, hm);
          fp4_hold(w1, e1, hm >> 16);
          w = (u32x2){w0, w1};
          e = (u32x2){e0, e1};
        }
        const unsigned wv[2] = {w.x, w.y}, ev[2] = {e.x, e.y};
        fp4_values(wv, ev, x.b, y.b);
        tile[buf][(2 * S + 2 * s) * 64 + l] = x.u;
        tile[buf][(2 * S + 2 * s + 1) * 64 + l] = y.u;
      }
    }
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
        fp4_score_step(row, s, *(const bf16x8*)&tile[buf][(2 * s) * 64 + lane],
                       *(const bf16x8*)&tile[buf][(2 * s + 1) * 64 + lane], sc);
      unsigned none = 0;
      if (MASKED && (page + 1) * kPage > t.L) {
        const unsigned g0 = *(const unsigned*)&gone[buf][4 * lg], g1 = *(const unsigned*)&gone[buf][16 + 4 * lg];
        none = (g0 | g0 >> 7 | g0 >> 14 | g0 >> 21) & 15u | ((g1 | g1 >> 7 | g1 >> 14 | g1 >> 21) & 15u) << 4;
      }
      bf16x8 pf[1][Row::PP];
      fp4_softmax<MASKED>(row, sc, page_bad[buf], none, tree, page * kPage - t.L, t.node0, masks, lg, pf);
#pragma unroll
      for (int d = 0; d < DT; d += 2)
        value_step(row, d, *(const bf16x8*)&tile[buf][(2 * S + d) * 64 + lane],
                   *(const bf16x8*)&tile[buf][(2 * S + d + 1) * 64 + lane], pf);
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

template <int HD, typename QT>
hipError_t fp4_attn_rows(const TreeAttnArgs& a, const TreeAttnPlan& p, hipStream_t st) {
  const unsigned grid = (unsigned)((long long)p.row_groups * p.slots * a.c.Hkv);
  if (p.few == 1) fp4_few_kernel<HD, QT, 1><<<grid, 256, 0, st>>>(a);
  else if (p.few == 2) fp4_few_kernel<HD, QT, 2><<<grid, 256, 0, st>>>(a);
  else fp4_many_kernel<HD, QT, 3><<<grid, 256, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.slots == a.c.B) return e;
  const long long rows = (long long)a.c.B * a.n * a.H;
  tree_combine_kernel<HD, QT><<<(unsigned)((rows + 3) / 4), 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

}  // namespace cdsl

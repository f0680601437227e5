// Attention of a token tree over the 8-bit paged cache: the kernel, one
// instance file per head dimension (tree_attention_*.hip).
//
//   o_i = sum_j softmax_j(scale q_i . k_j) v_j
//
// over the prompt's L cached tokens and the node's ancestors and itself.
// With k = s_k c_k and v = s_v c_v (codes c, one scale per token and KV head)
// the scales leave the sums over dims: s_k multiplies a score, s_v a
// probability, and the matrix products run on the codes, which are exact in
// bf16.  One pass over the keys with a running maximum and sum (fp32).
//
// Workgroup = (key split, prompt x KV head, group of 16-row tiles); the rows
// of a (prompt, KV head) are its nodes x the G query heads of that KV head.
// Its four waves are row groups x KW key groups; a wave takes RPW row tiles
// and every KW-th page, whose codes go from memory straight to its registers:
// the cache holds them in operand order (tree.h), so there is no LDS stage
// and no barrier in the loop.  Scores are computed transposed,
//   S^T[16 keys, 16 rows] = K[16, hd] . Q^T[hd, 16]       (MFMA 16x16x32)
// so that a lane's scores are its operand of the second product,
//   O^T[16 dims, 16 rows] += V^T[16 dims, 32 keys] . P^T[32 keys, 16 rows].
// Key groups merge through LDS, key splits through a second kernel, both in
// a fixed order.
#pragma once
#include "tree.h"

namespace cdsl {

namespace {

// Eight codes (two words, slots or dims in order) as bf16, exact.
template <int FMT>
__device__ __forceinline__ bf16x8 codes8(unsigned a, unsigned b) {
  union {
    unsigned u[4];
    bf16x8 v;
  } o;
  if constexpr (FMT == kE4M3) {
    union {
      bf16x2v v;
      unsigned u;
    } t;
    t.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false);
    o.u[0] = t.u;
    t.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true);
    o.u[1] = t.u;
    t.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false);
    o.u[2] = t.u;
    t.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true);
    o.u[3] = t.u;
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

__device__ __forceinline__ f32x4 mfma16(const bf16x8& a, const bf16x8& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Bytes of word bits 0..3 of m as a mask.
__device__ __forceinline__ unsigned byte_mask(unsigned m) {
  return ((m & 1u) | (m & 2u) << 7 | (m & 4u) << 14 | (m & 8u) << 21) * 255u;
}

// QT float: activations in fp32.  q and p s_v are taken as three bf16 planes
// each (their 24 bits): with two, 2^-16 of each probability is lost, and the
// result's error is 2.5e-6 of it where fp32 products and sums give 0.8e-6.
// QT bf16: q as it is and p s_v in bf16 (2^-8 of each probability,
// independent over the keys; the result rounds by as much).
template <int HD, int FMT, typename QT, int RPW, int KW>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void tree_attn_kernel(TreeAttnArgs a) {
  constexpr int NW = 4, RTW = NW / KW;
  constexpr int S = HD / 32, DT = HD / 16;
  constexpr int QP = sizeof(QT) == 4 ? 3 : 1, PP = QP;   // planes of q and of p s_v
  constexpr int ROWS = 16 * RPW * RTW;       // rows per workgroup
  constexpr int MW = kTreeWords;             // mask words per node
  constexpr int UNIT = kvq_unit_bytes(HD);
  constexpr float kLazy = 8.f;
  constexpr int SLOT = (2 + 4 * DT) * 64;    // floats a wave hands over per row tile
  constexpr int XF = (KW - 1) * RTW * RPW * SLOT, MF = ROWS * MW + kTreeMax;
  __shared__ float lds[XF > MF ? XF : MF];

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int lr = lane & 15, lg = lane >> 4;
  // The row groups of one (prompt, KV head, split) read the same pages:
  // workgroup w runs on XCD w % 8, so they take consecutive slots of one XCD.
  const int NR = a.row_groups, NC = gridDim.x / NR, full = NC & ~7;
  int chunk, rg;
  if ((int)blockIdx.x < full * NR) {
    const int t = blockIdx.x >> 3;
    chunk = (blockIdx.x & 7) + 8 * (t / NR);
    rg = t % NR;
  } else {
    const int t = blockIdx.x - full * NR;
    chunk = full + t / NR;
    rg = t % NR;
  }
  const int split = chunk % a.nsplit, pair = chunk / a.nsplit;
  const int b = pair / a.c.Hkv, kvh = pair % a.c.Hkv;
  const int G = a.G;
  const int nb = a.n_nodes ? min(max(a.n_nodes[b], 0), a.n) : a.n;
  const int nrows = nb * G, row0 = rg * ROWS;
  if (row0 >= nrows) return;   // uniform over the workgroup
  const int L = max(a.lens[b], 0);
  const int node0 = row0 / G, node1 = (min(row0 + ROWS, nrows) - 1) / G;
  // a prompt that its table cannot hold has no answer: NaN, and no page read
  const bool over = (long long)L + nb > (long long)a.c.table_stride * kPage;
  const int pages = over ? 0 : (L + nb + kPage - 1) / kPage;
  const int per = (pages + a.nsplit - 1) / a.nsplit;
  const int beg = split * per;
  const int end = over ? 0 : min(min(beg + per, pages), (L + node1) / kPage + 1);

  const int rt = wave / KW, kw = wave % KW;
  const int rw0 = row0 + rt * 16 * RPW;
  const bool has_rows = rw0 < nrows;
  int node[RPW], qrow[RPW];
  bool valid[RPW];
#pragma unroll
  for (int r = 0; r < RPW; ++r) {
    const int row = rw0 + 16 * r + lr;
    valid[r] = row < nrows;
    const int rr = valid[r] ? row : nrows - 1;
    node[r] = rr / G;
    qrow[r] = kvh * G + rr % G;
  }

  // page ids of this wave's next 64 pages, one a lane
  int ids = 0;
  const int* table = a.c.table + (long long)b * a.c.table_stride;
  auto fetch_ids = [&](int it) __attribute__((always_inline)) {
    const int p = beg + kw + KW * (it + lane);
    ids = p < end ? table[p] : 0;
  };
  const int npages = has_rows && end > beg + kw ? (end - beg - kw + KW - 1) / KW : 0;
  if (npages > 0) fetch_ids(0);

  // Q^T fragments: row lr, dims 32 s + 8 lg .. +7
  bf16x8 qf[RPW][S][QP];
#pragma unroll
  for (int r = 0; r < RPW; ++r) {
    const QT* qp = (const QT*)a.q + b * a.qsb + node[r] * a.qst + (long long)qrow[r] * HD + 8 * lg;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      if constexpr (QP == 1) {
        qf[r][s][0] = *(const bf16x8*)(qp + 32 * s);
      } else {
        const f32x4 x0 = *(const f32x4*)(qp + 32 * s), x1 = *(const f32x4*)(qp + 32 * s + 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float x = e < 4 ? x0[e & 3] : x1[e & 3];
#pragma unroll
          for (int pl = 0; pl < QP; ++pl) {
            const bf16 hi = (bf16)x;
            qf[r][s][pl][e] = hi;
            x -= (float)hi;
          }
        }
      }
    }
  }

  // Which nodes a node sees: bit m of its mask.  A parent outside [0, own
  // index) ends the walk, so every walk ends.
  const bool tree = a.parents != nullptr && a.n > 1;
  unsigned* masks = (unsigned*)lds;
  if (tree) {
    int* par = (int*)lds + ROWS * MW;
    for (int i = threadIdx.x; i <= node1; i += 256) par[i] = a.parents[(long long)b * a.n + i];
    for (int i = threadIdx.x; i < ROWS * MW; i += 256) masks[i] = 0u;
    __syncthreads();
    const int i = threadIdx.x;
    if (i <= node1 - node0) {
      int m = node0 + i;
      while (true) {
        masks[i * MW + (m >> 5)] |= 1u << (m & 31);
        const int up = par[m];
        if (up < 0 || up >= m) break;
        m = up;
      }
    }
    __syncthreads();
  }
  auto visible = [&](int page, int m) __attribute__((always_inline)) -> unsigned {
    const int i0 = page * kPage - L;
    return tree ? slots_of_tree(i0, masks + (m - node0) * MW) : slots_of_chain(i0, m);
  };

  u32x4 kr[S], vr[S];
  f32x4 ksr[2], vsr[2];
  auto load = [&](int it) __attribute__((always_inline)) {
    const int id = __builtin_amdgcn_readlane(ids, it & 63);
    const bool bad = id < 0 || id >= a.c.pages;
    const uint8_t* u = a.c.pool + ((long long)(bad ? 0 : id) * a.c.Hkv + kvh) * UNIT;
#pragma unroll
    for (int s = 0; s < S; ++s) kr[s] = *(const u32x4*)(u + s * 1024 + lane * 16);
#pragma unroll
    for (int s = 0; s < S; ++s) vr[s] = *(const u32x4*)(u + kPage * HD + s * 1024 + lane * 16);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      ksr[t] = *(const f32x4*)(u + 2 * kPage * HD + 64 * t + 16 * lg);
      vsr[t] = *(const f32x4*)(u + 2 * kPage * HD + 4 * kPage + 64 * t + 16 * lg);
    }
    if (bad) {   // its keys have no value: rows that see one are NaN
      const float nan = __uint_as_float(0x7fc00000u);
      ksr[0] = ksr[1] = (f32x4){nan, nan, nan, nan};
    }
  };

  f32x4 acc[RPW][DT];
  float m_run[RPW], l_run[RPW];
#pragma unroll
  for (int r = 0; r < RPW; ++r) {
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[r][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    // running maximum (log2 units) and sum.  The exponentials use a maximum
    // that may lie up to kLazy below the true one, so O is rescaled rarely.
    m_run[r] = -INFINITY;
    l_run[r] = over ? __uint_as_float(0x7fc00000u) : 0.f;
  }

  if (npages > 0) load(0);
  for (int it = 0; it < npages; ++it) {
    const int page = beg + kw + KW * it;
    // scores of this page
    f32x4 sA[RPW], sB[RPW];
#pragma unroll
    for (int r = 0; r < RPW; ++r) sA[r] = sB[r] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const bf16x8 kA = codes8<FMT>(kr[s].x, kr[s].y), kB = codes8<FMT>(kr[s].z, kr[s].w);
#pragma unroll
      for (int r = 0; r < RPW; ++r)
#pragma unroll
        for (int pl = 0; pl < QP; ++pl) {
          sA[r] = mfma16(kA, qf[r][s][pl], sA[r]);
          sB[r] = mfma16(kB, qf[r][s][pl], sB[r]);
        }
    }
    float ks[8], vs[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      ks[e] = ksr[e >> 2][e & 3] * a.scale_log2;
      vs[e] = vsr[e >> 2][e & 3];
    }
    bf16x8 vf[DT];
    const bool masked = (page + 1) * kPage > L;   // uniform: the page holds nodes
    if (FMT == kE4M3 && masked) {
      // slots past the last node were never written: a code there may be a NaN
      const int held = L + nb - page * kPage;
      const unsigned hm = held >= 32 ? ~0u : (1u << held) - 1u;
      const unsigned mA = byte_mask(hm >> (4 * lg)), mB = byte_mask(hm >> (16 + 4 * lg));
#pragma unroll
      for (int s = 0; s < S; ++s) {
        vr[s].x &= mA;
        vr[s].y &= mB;
        vr[s].z &= mA;
        vr[s].w &= mB;
      }
    }
#pragma unroll
    for (int s = 0; s < S; ++s) {
      vf[2 * s] = codes8<FMT>(vr[s].x, vr[s].y);
      vf[2 * s + 1] = codes8<FMT>(vr[s].z, vr[s].w);
    }
    // the next page's loads are in flight during the rest
    if (it + 1 < npages) {
      if (((it + 1) & 63) == 0) fetch_ids(it + 1);
      load(it + 1);
    }
#pragma unroll
    for (int r = 0; r < RPW; ++r) {
      unsigned vis = ~0u;
      if (masked) vis = visible(page, node[r]) >> (4 * lg);
      float sv[8], mt = -INFINITY;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        sv[e] = (e < 4 ? sA[r][e & 3] : sB[r][e & 3]) * ks[e];
        if (masked && !(vis >> (e < 4 ? e : 12 + e) & 1u)) sv[e] = -INFINITY;
        mt = fmaxf(mt, sv[e]);
      }
      mt = fmaxf(mt, __shfl_xor(mt, 16, 64));
      mt = fmaxf(mt, __shfl_xor(mt, 32, 64));
      const bool raise = mt > m_run[r] + kLazy;   // true for the first visible key
      if (__ballot(raise)) {
        const float m_to = raise ? mt : m_run[r];
        const float corr = m_to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[r] - m_to);
        l_run[r] *= corr;
#pragma unroll
        for (int t = 0; t < DT; ++t) acc[r][t] *= corr;
        m_run[r] = m_to;
      }
      const float m_use = m_run[r] == -INFINITY ? 0.f : m_run[r];
      bf16x8 pf[PP];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float p = __builtin_amdgcn_exp2f(sv[e] - m_use);
        l_run[r] += p;
        float x = p * vs[e];
        if (masked && !(vis >> (e < 4 ? e : 12 + e) & 1u)) x = 0.f;   // its scale may be anything
#pragma unroll
        for (int pl = 0; pl < PP; ++pl) {
          const bf16 hi = (bf16)x;
          pf[pl][e] = hi;
          x -= (float)hi;
        }
      }
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int pl = 0; pl < PP; ++pl) acc[r][t] = mfma16(vf[t], pf[pl], acc[r][t]);
    }
  }

#pragma unroll
  for (int r = 0; r < RPW; ++r) {
    l_run[r] += __shfl_xor(l_run[r], 16, 64);
    l_run[r] += __shfl_xor(l_run[r], 32, 64);
  }
  if constexpr (KW > 1) {
    // key groups 1.. hand (m, l, O) to group 0, which adds them in order
    __syncthreads();   // the masks are no longer read
    if (has_rows && kw > 0) {
#pragma unroll
      for (int r = 0; r < RPW; ++r) {
        float* x = lds + ((rt * (KW - 1) + kw - 1) * RPW + r) * SLOT;
        x[lane] = m_run[r];
        x[64 + lane] = l_run[r];
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) x[(2 + 4 * t + e) * 64 + lane] = acc[r][t][e];
      }
    }
    __syncthreads();
    if (kw > 0) return;
  }
  if (!has_rows) return;
  if constexpr (KW > 1) {
#pragma unroll
    for (int k = 1; k < KW; ++k)
#pragma unroll
      for (int r = 0; r < RPW; ++r) {
        const float* x = lds + ((rt * (KW - 1) + k - 1) * RPW + r) * SLOT;
        const float mq = x[lane], lq = x[64 + lane];
        const float mn = fmaxf(m_run[r], mq);
        const float s0 = m_run[r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run[r] - mn);
        const float s1 = mq == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mq - mn);
        l_run[r] = l_run[r] * s0 + lq * s1;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[r][t][e] = acc[r][t][e] * s0 + x[(2 + 4 * t + e) * 64 + lane] * s1;
        m_run[r] = mn;
      }
  }
#pragma unroll
  for (int r = 0; r < RPW; ++r) {
    if (!valid[r]) continue;
    const long long row = ((long long)b * a.n + node[r]) * a.H + qrow[r];
    // lane (row lr, lg) holds dims 16 t + 4 lg .. +3
    if (a.nsplit == 1) {
      const float inv = 1.f / l_run[r];
      QT* o = (QT*)a.out + row * HD + 4 * lg;
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        const f32x4 y = acc[r][t] * inv;
        if constexpr (sizeof(QT) == 4) *(f32x4*)(o + 16 * t) = y;
        else *(bf16x4*)(o + 16 * t) = (bf16x4){(bf16)y[0], (bf16)y[1], (bf16)y[2], (bf16)y[3]};
      }
    } else {
      const long long prow = (long long)split * a.c.B * a.n * a.H + row;
      float* po = a.part_o + prow * HD + 4 * lg;
#pragma unroll
      for (int t = 0; t < DT; ++t) *(f32x4*)(po + 16 * t) = acc[r][t];
      if (lg == 0) {
        a.part_ml[prow * 2] = m_run[r];
        a.part_ml[prow * 2 + 1] = l_run[r];
      }
    }
  }
}

// Merge of the key splits: one wave per (node, head) row.
template <int HD, typename QT>
__global__ __launch_bounds__(256) void tree_combine_kernel(TreeAttnArgs a) {
  const long long rows = (long long)a.c.B * a.n * a.H;
  const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= rows) return;
  if (a.n_nodes) {
    const int nd = (int)(row / a.H % a.n), b = (int)(row / a.H / a.n);
    if (nd >= a.n_nodes[b]) return;
  }
  constexpr int PER = (HD + 63) / 64;
  const int ns = a.nsplit;
  float ms = -INFINITY, ls = 0.f;
  if (lane < ns) {
    ms = a.part_ml[((long long)lane * rows + row) * 2];
    ls = a.part_ml[((long long)lane * rows + row) * 2 + 1];
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
        o[k][u] = s0 + k < ns && d < HD ? a.part_o[((long long)(s0 + k) * rows + row) * HD + d] : 0.f;
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
  const unsigned grid = (unsigned)((long long)p.row_groups * p.nsplit * a.c.B * a.c.Hkv);
  if (p.rpw == 1 && p.kw == 4) tree_attn_kernel<HD, FMT, QT, 1, 4><<<grid, 256, 0, st>>>(a);
  else if (p.rpw == 2 && p.kw == 4) tree_attn_kernel<HD, FMT, QT, 2, 4><<<grid, 256, 0, st>>>(a);
  else if (p.rpw == 2 && p.kw == 2) tree_attn_kernel<HD, FMT, QT, 2, 2><<<grid, 256, 0, st>>>(a);
  else if (p.rpw == 2 && p.kw == 1) tree_attn_kernel<HD, FMT, QT, 2, 1><<<grid, 256, 0, st>>>(a);
  else return hipErrorInvalidValue;
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.nsplit == 1) return e;
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

// Verification of a drafted tree against the target's probabilities: the
// walk of speculative sampling over a tree, from given random numbers.
//
// From the node reached (0 at first) with rows p (target) and q (draft), its
// children are tested in index order:
//   P_0 = p;  child j with token x is taken when u_j q_r(x) <= P_r(x) and
//   P_r(x) > 0;  else  P_{r+1} = max(0, P_r - q_r) / (its sum),
// with q_r = q, or (drawn without replacement) q without the tokens rejected
// so far, over the share rest_r = 1 - sum of their q that is left of it.  The
// token after the last node taken is drawn from the P_r reached.  All P_r
// have one form,
//   P_r = max(0, p - c_r q) / N_r,   c_0 = 0, N_0 = 1,
//   c_{r+1} = c_r + N_r / rest_r,    N_{r+1} = sum max(0, p - c_{r+1} q),
// (a rejected token's entry is 0 from its rejection on, so that it does not
// matter that c_r q still counts it), so a rejection costs one sum over the
// two rows and nothing is stored.  Sums and tests are in fp64: in fp32 a
// draw among 32000 flat entries would land next to its token once in about
// thirty.
//
// One workgroup per prompt: the walk is a chain of decisions, and only the
// rows it rejects at, and the last one, are read.  The probabilities of all
// children are fetched at once first, so that the walk itself stays in LDS.
#include "tree.h"

namespace cdsl {

namespace {

constexpr int NT = 1024, NW = NT / 64;
constexpr int BLK = 4 * NT;                     // ids per block: four a thread
constexpr int kSegs = kAcceptMaxVocab / BLK * NW;   // (block, wave) sums at most

__device__ __forceinline__ double wave_sum_d(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// four entries of a row from id i on (0 past the end)
__device__ __forceinline__ void row4(const float* row, int i, int V, float (&x)[4]) {
  if (i + 4 <= V) {
    const f32x4u t = *(const f32x4u*)(row + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = t[e];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = i + e < V ? row[i + e] : 0.f;
  }
}

__global__ __launch_bounds__(NT) void tree_accept_kernel(const float* __restrict__ p_all,
                                                         const float* __restrict__ q_all, int n, int V,
                                                         const int* __restrict__ tokens,
                                                         const int* __restrict__ parents,
                                                         const int* __restrict__ n_nodes, const float* __restrict__ u,
                                                         const float* __restrict__ v, int replace, int* path,
                                                         int* n_path, int* next_token) {
  __shared__ int par[kTreeMax], tok[kTreeMax], walk[kTreeMax];
  __shared__ float px[kTreeMax], qx[kTreeMax], us[kTreeMax];
  __shared__ double part[kSegs];
  __shared__ double wtot[NW];
  __shared__ int hit, best_i[NW];
  __shared__ float best_v[NW];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int nb = n_nodes ? min(max(n_nodes[b], 1), n) : n;
  const long long row0 = (long long)b * n;
  for (int j = tid; j < nb; j += NT) {
    int c = j > 0 ? parents[row0 + j] : -1;
    const int x = tokens[row0 + j];
    if (c < 0 || c >= j || x < 0 || x >= V) c = -1;   // not a child that can be taken
    par[j] = c;
    tok[j] = x;
    if (c >= 0) {
      px[j] = p_all[(row0 + c) * V + x];
      qx[j] = q_all[(row0 + c) * V + x];
      us[j] = u[row0 + j];
    }
  }
  if (tid == 0) walk[0] = 0, hit = -1;
  __syncthreads();

  const int nblk = (V + BLK - 1) / BLK;
  int cur = 0, len = 1, from = 1;
  double c = 0., N = 1., rest = 1.;
  const float* p = p_all + row0 * V;
  const float* q = q_all + row0 * V;

  // w = max(0, p - c q) of four ids
  auto weights = [&](int i, double (&w)[4]) __attribute__((always_inline)) {
    float x[4], y[4];
    row4(p, i, V, x);
    if (c > 0.) {
      row4(q, i, V, y);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = fmax(0., fma(-c, (double)y[e], (double)x[e]));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = (double)x[e];
    }
  };
  // part[block * NW + wave] and the sum over all ids
  auto sum = [&]() __attribute__((always_inline)) -> double {
    double mine = 0.;
    for (int k = 0; k < nblk; ++k) {
      double w[4];
      weights(BLK * k + 4 * tid, w);
      const double s = wave_sum_d((w[0] + w[1]) + (w[2] + w[3]));
      if (lane == 0) part[k * NW + wv] = s;
      mine += s;
    }
    __syncthreads();   // earlier readers of wtot are done
    if (lane == 0) wtot[wv] = mine;
    __syncthreads();
    double t = 0.;
#pragma unroll
    for (int k = 0; k < NW; ++k) t += wtot[k];
    return t;
  };

  // Every wave walks alike, 64 nodes at a time.
  bool none = false, summed = false;   // no mass left; part holds the sums of the present c
  while (from < nb && !none) {
    const int j0 = from & ~63, j = j0 + lane;
    const unsigned long long kids = __ballot(j >= from && j < nb && par[j] == cur);
    if (!kids) {
      from = j0 + 64;
      continue;
    }
    const int k = j0 + __builtin_ctzll(kids);
    from = k + 1;
    if (!(rest > 0.)) continue;
    const double pk = c > 0. ? fmax(0., fma(-c, (double)qx[k], (double)px[k])) / N : (double)px[k];
    const double qk = (double)qx[k] / rest;
    if (pk > 0. && (double)us[k] * qk <= pk) {
      if (tid == 0) walk[len] = k;
      ++len;
      cur = k;
      p = p_all + (row0 + k) * V;
      q = q_all + (row0 + k) * V;
      c = 0., N = 1., rest = 1.;
      summed = false;
      continue;
    }
    c += N / rest;
    N = sum();
    summed = true;
    if (!replace) {
      // a token that an earlier sibling carried is out of q already
      bool twice = false;
      for (int s = 0; s < k; s += 64) {
        const int e = s + lane;
        twice = twice || __ballot(e < k && par[e] == cur && tok[e] == tok[k]);
      }
      if (!twice) rest -= (double)qx[k];
    }
    if (!(N > 0.)) none = true;
  }

  // The draw: the first id whose running sum passes v * (sum).
  if (!summed) N = sum();
  if (none) {
    // argmax p, lowest id on ties
    float bv = -INFINITY;
    int bi = 0;
    for (int i = tid; i < V; i += NT) {
      if (p[i] > bv) bv = p[i], bi = i;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const float ov = __shfl_xor(bv, o, 64);
      const int oi = __shfl_xor(bi, o, 64);
      if (vi_better(ov, oi, bv, bi)) bv = ov, bi = oi;
    }
    if (lane == 0) best_v[wv] = bv, best_i[wv] = bi;
    __syncthreads();
    if (tid == 0) {
      for (int k = 1; k < NW; ++k)
        if (vi_better(best_v[k], best_i[k], bv, bi)) bv = best_v[k], bi = best_i[k];
      hit = N == 0. ? bi : -1;
    }
  } else if (N > 0. && N < INFINITY) {
    const int segs = nblk * NW;
    const double T = (double)v[b] * N;
    // the segment the draw falls in, and the sum before it: each lane of a
    // wave takes a run of segments
    const int run = (segs + 63) / 64;
    double mine = 0.;
    for (int s = lane * run; s < min(segs, lane * run + run); ++s) mine += part[s];
    double incl = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double t = __shfl_up(incl, o, 64);
      if (lane >= o) incl += t;
    }
    double before = __shfl_up(incl, 1, 64);
    if (lane == 0) before = 0.;
    const unsigned long long past = __ballot(mine > 0. && incl > T), mass = __ballot(mine > 0.);
    // rounding may leave T at the sum: then the last run with mass
    const int src = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(mass | 1ull);
    double at = __shfl(before, src, 64);
    int seg = -1;
    double seg_at = at;
    for (int s = src * run; s < min(segs, src * run + run); ++s) {
      if (part[s] > 0.) {
        seg = s;
        seg_at = at;
        if (at + part[s] > T) break;
      }
      at += part[s];
    }
    if (seg >= 0 && wv == seg % NW) {
      const int i0 = BLK * (seg / NW) + 4 * tid;
      double w[4];
      weights(i0, w);
      const double own = (w[0] + w[1]) + (w[2] + w[3]);
      double sc = own;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const double t = __shfl_up(sc, o, 64);
        if (lane >= o) sc += t;
      }
      double r = __shfl_up(sc, 1, 64);
      if (lane == 0) r = 0.;
      r += seg_at;
      int at_e = -1, last_e = -1;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (w[e] > 0.) {
          last_e = e;
          if (at_e < 0 && r + w[e] > T) at_e = e;
        }
        r += w[e];
      }
      const unsigned long long hits = __ballot(at_e >= 0), with = __ballot(last_e >= 0);
      const int who = hits ? __builtin_ctzll(hits) : 63 - __builtin_clzll(with | 1ull);
      if (lane == who && with) hit = i0 + (hits ? at_e : last_e);
    }
  }
  __syncthreads();
  for (int i = tid; i < n; i += NT) path[row0 + i] = i < len ? walk[i] : -1;
  if (tid == 0) {
    n_path[b] = len;
    next_token[b] = hit;
  }
}

}  // namespace

hipError_t tree_accept_launch(const float* p, const float* q, int B, int n, int V, const int* tokens,
                              const int* parents, const int* n_nodes, const float* u, const float* v, int replace,
                              int* path, int* n_path, int* next_token, hipStream_t st) {
  if (B == 0) return hipSuccess;
  tree_accept_kernel<<<B, NT, 0, st>>>(p, q, n, V, tokens, parents, n_nodes, u, v, replace, path, n_path, next_token);
  return hipGetLastError();
}

}  // namespace cdsl

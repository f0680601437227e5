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
// Latency bounds it, so a row's loads are all in flight together, and rows of
// up to 32768 ids stay in registers for the node's further sums and the draw.
#include "tree.h"

namespace cdsl {

namespace {

constexpr int NT = 1024, NW = NT / 64;
constexpr int RUN = 1024;                       // consecutive ids of a wave in a chunk: 16 a lane
constexpr int CHUNK = NW * RUN;
constexpr int kSegs = kAcceptMaxVocab / RUN;    // (chunk, wave) sums at most
constexpr int kHeld = 2;                        // chunks that registers hold

// Sum over a wave, the same bits in every lane: rotations within rows of 16,
// then swaps of rows and halves (a shuffle through LDS takes five times as long).
template <int CTRL>
__device__ __forceinline__ double add_rotated(double v) {
  const unsigned lo = __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, 0xf, 0xf, false);
  const unsigned hi = __builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, 0xf, 0xf, false);
  return v + __hiloint2double(hi, lo);
}
__device__ __forceinline__ double wave_sum_d(double v) {
  typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
  v = add_rotated<0x128>(v);   // row_ror:8, 4, 2, 1
  v = add_rotated<0x124>(v);
  v = add_rotated<0x122>(v);
  v = add_rotated<0x121>(v);
  u32x2 lo = __builtin_amdgcn_permlane16_swap(__double2loint(v), __double2loint(v), false, false);
  u32x2 hi = __builtin_amdgcn_permlane16_swap(__double2hiint(v), __double2hiint(v), false, false);
  v = __hiloint2double(hi.x, lo.x) + __hiloint2double(hi.y, lo.y);
  lo = __builtin_amdgcn_permlane32_swap(__double2loint(v), __double2loint(v), false, false);
  hi = __builtin_amdgcn_permlane32_swap(__double2hiint(v), __double2hiint(v), false, false);
  return __hiloint2double(hi.x, lo.x) + __hiloint2double(hi.y, lo.y);
}

// Sixteen entries of a row: four at i, i + 256, i + 512, i + 768 (0 past the end).
struct Piece {
  float x[4][4];
  __device__ __forceinline__ void load(const float* row, int i, int V) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int at = i + 256 * u;
      if (at + 4 <= V) {
        const f32x4u t = *(const f32x4u*)(row + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[u][e] = t[e];
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[u][e] = at + e < V ? row[at + e] : 0.f;
      }
    }
  }
};

// max(0, p - c q); a NaN stays one
__device__ __forceinline__ double weight(float p, float q, double c) {
  const double d = fma(-c, (double)q, (double)p);
  return d < 0. ? 0. : d;
}
// Their sum as half of sum d + sum |d|: a subtraction and two additions an
// entry, and a NaN stays one (the fp64 instructions bound a pass: a maximum
// that keeps NaNs takes three).  Without an entry above 0 the two cancel to
// exactly 0, since every partial sum has its negative.
__device__ __forceinline__ double weights(const Piece& p, const Piece& q, double c) {
  double d = 0., a = 0.;
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const double t = fma(-c, (double)q.x[u][e], (double)p.x[u][e]);
      d += t;
      a += fabs(t);
    }
  return 0.5 * (d + a);
}

// HELD: V <= kHeld * CHUNK.
template <bool HELD>
__global__ __launch_bounds__(NT) void tree_accept_kernel(const float* __restrict__ p_all,
                                                         const float* __restrict__ q_all, int n, int V,
                                                         const int* __restrict__ tokens,
                                                         const int* __restrict__ parents,
                                                         const int* __restrict__ n_nodes, const float* __restrict__ u,
                                                         const float* __restrict__ v, int replace, int* path,
                                                         int* n_path, int* next_token) {
  __shared__ int par[kTreeMax], tok[kTreeMax], walk[kTreeMax];
  __shared__ float px[kTreeMax], qx[kTreeMax], us[kTreeMax];
  __shared__ double part[HELD ? kHeld * NW : kSegs];
  __shared__ int hit, best_i[NW];
  __shared__ float best_v[NW];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int nb = n_nodes ? min(max(n_nodes[b], 1), n) : n;
  const long long row0 = (long long)b * n;
  for (int j = tid; j < nb; j += NT) {
    int c = j > 0 ? parents[row0 + j] : -1;
    const int x = tokens[row0 + j];
    const float uj = u[row0 + j];
    if (c < 0 || c >= j || x < 0 || x >= V) c = -1;   // not a child that can be taken
    par[j] = c;
    tok[j] = x;
    if (c >= 0) {
      px[j] = p_all[(row0 + c) * V + x];
      qx[j] = q_all[(row0 + c) * V + x];
      us[j] = uj;
    }
  }
  if (tid == 0) walk[0] = 0, hit = -1;
  __syncthreads();

  const int chunks = (V + CHUNK - 1) / CHUNK, segs = chunks * NW;
  const int at0 = wv * RUN + 4 * lane;   // this lane's first id of a chunk
  int cur = 0, len = 1, from = 1;
  double c = 0., N = 1., rest = 1.;
  const float* p = p_all + row0 * V;
  const float* q = q_all + row0 * V;
  Piece hp[HELD ? kHeld : 1], hq[HELD ? kHeld : 1];
  bool have_p = false, have_q = false;   // the held pieces are those of cur

  // part[chunk * NW + wave] and their sum, for the present c
  auto sum = [&]() __attribute__((always_inline)) -> double {
    __syncthreads();   // earlier readers of part are done
    if constexpr (HELD) {
      const bool lp = !have_p, lq = !have_q && c > 0.;
#pragma unroll
      for (int k = 0; k < kHeld; ++k) {
        if (lp) hp[k].load(p, CHUNK * k + at0, V);
        if (lq) hq[k].load(q, CHUNK * k + at0, V);
        else if (c == 0.) hq[k] = Piece{};
      }
      have_p = true;
      have_q = c > 0.;
      double s[kHeld];
#pragma unroll
      for (int k = 0; k < kHeld; ++k) s[k] = wave_sum_d(weights(hp[k], hq[k], c));
      if (lane == 0)
#pragma unroll
        for (int k = 0; k < kHeld; ++k)
          if (k < chunks) part[k * NW + wv] = s[k];
    } else {
      // the next chunk's loads are in flight while one is added up
      Piece np, nq{}, xp, xq{};
      np.load(p, at0, V);
      if (c > 0.) nq.load(q, at0, V);
      for (int k = 0; k < chunks; ++k) {
        xp = np;
        xq = nq;
        if (k + 1 < chunks) {
          np.load(p, CHUNK * (k + 1) + at0, V);
          if (c > 0.) nq.load(q, CHUNK * (k + 1) + at0, V);
        }
        const double s = wave_sum_d(weights(xp, xq, c));
        if (lane == 0) part[k * NW + wv] = s;
      }
    }
    __syncthreads();
    double t = 0.;
    for (int k = lane; k < segs; k += 64) t += part[k];
    return wave_sum_d(t);
  };

  // Every wave walks alike, 64 nodes at a time, from one sum to the next.
  bool none = false, done = false, summed = false;   // no mass left; walked; part holds the sums of the present c
  while (true) {
    int fell = -1;   // the child that is rejected next
    while (from < nb && !none && fell < 0) {
      const int j0 = from & ~63, j = j0 + lane;
      const unsigned long long kids = __ballot(j >= from && j < nb && par[j] == cur);
      if (!kids) {
        from = j0 + 64;
        continue;
      }
      const int k = j0 + __builtin_ctzll(kids);
      from = k + 1;
      if (!(rest > 0.)) continue;
      const double pk = c > 0. ? weight(px[k], qx[k], c) / N : (double)px[k];
      const double qk = (double)qx[k] / rest;
      if (pk > 0. && (double)us[k] * qk <= pk) {
        if (tid == 0) walk[len] = k;
        ++len;
        cur = k;
        p = p_all + (row0 + k) * V;
        q = q_all + (row0 + k) * V;
        c = 0., N = 1., rest = 1.;
        summed = have_p = have_q = false;
      } else {
        fell = k;
      }
    }
    done = fell < 0;
    if (!done) c += N / rest;
    if (done && summed) break;
    N = sum();
    if (done) break;
    summed = true;
    if (!replace) {
      // a token that an earlier sibling carried is out of q already
      bool twice = false;
      for (int s = 0; s < fell; s += 64) {
        const int e = s + lane;
        twice = twice || __ballot(e < fell && par[e] == cur && tok[e] == tok[fell]);
      }
      if (!twice) rest -= (double)qx[fell];
    }
    if (!(N > 0.)) none = true;
  }

  // The draw: the first id whose running sum passes v * (sum).
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
    // first entry of a row of lanes whose running sum from `at` passes T (the
    // last one with mass when rounding leaves T past the total), and the sum
    // before it
    auto locate = [&](double mine, double T, double& at) __attribute__((always_inline)) -> int {
      double incl = mine;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const double t = __shfl_up(incl, o, 64);
        if (lane >= o) incl += t;
      }
      double before = __shfl_up(incl, 1, 64);
      if (lane == 0) before = 0.;
      const unsigned long long past = __ballot(mine > 0. && at + incl > T), mass = __ballot(mine > 0.);
      const int src = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(mass | 1ull);
      at += __shfl(before, src, 64);
      return mass ? src : -1;
    };
    const double T = (double)v[b] * N;
    // each lane takes a run of segments
    const int run = (segs + 63) / 64;
    double mine = 0., at = 0.;
    for (int s = lane * run; s < min(segs, lane * run + run); ++s) mine += part[s];
    const int src = locate(mine, T, at);
    int seg = -1;
    double seg_at = at;
    for (int s = src * run; src >= 0 && s < min(segs, src * run + run); ++s) {
      if (part[s] > 0.) {
        seg = s;
        seg_at = at;
        if (at + part[s] > T) break;
      }
      at += part[s];
    }
    if (seg >= 0 && wv == seg % NW) {   // its wave: 4 x 64 lanes x 4 ids in order
      const int i0 = CHUNK * (seg / NW) + at0;
      Piece xp, xq{};
      xp.load(p, i0, V);
      if (c > 0.) xq.load(q, i0, V);
      double t[4], w[4];
      int pick = -1;
      double pick_at = seg_at;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        t[k] = (weight(xp.x[k][0], xq.x[k][0], c) + weight(xp.x[k][1], xq.x[k][1], c)) +
               (weight(xp.x[k][2], xq.x[k][2], c) + weight(xp.x[k][3], xq.x[k][3], c));
        const double all = wave_sum_d(t[k]);
        if (all > 0. && !(pick >= 0 && seg_at > T)) {
          pick = k;
          pick_at = seg_at;
        }
        seg_at += all;
      }
      double own = 0.;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k == pick) {
          own = t[k];
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = weight(xp.x[k][e], xq.x[k][e], c);
        }
      double lane_at = pick_at;
      const int who = locate(own, T, lane_at);
      if (lane == who) {
        int e_at = -1;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (w[e] > 0. && (e_at < 0 || !(lane_at > T))) e_at = e;
          lane_at += w[e];
        }
        hit = i0 + 256 * pick + e_at;
      }
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
  if (V <= kHeld * CHUNK)
    tree_accept_kernel<true><<<B, NT, 0, st>>>(p, q, n, V, tokens, parents, n_nodes, u, v, replace, path, n_path,
                                               next_token);
  else
    tree_accept_kernel<false><<<B, NT, 0, st>>>(p, q, n, V, tokens, parents, n_nodes, u, v, replace, path, n_path,
                                                next_token);
  return hipGetLastError();
}

}  // namespace cdsl

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
// The walk is a chain of decisions, and only the rows it rejects at, and the
// last one, are read.  The probabilities of all children are fetched at once
// first, so that the walk itself stays in LDS.  Latency bounds it, and the
// fp64 rate of one CU (3 us for a sum over 32000 ids, 13 us over 128256).  Rows
// of up to 32768 ids: one workgroup per prompt, which keeps a node's rows in
// its registers for the node's further sums and the draw.  Longer rows: the
// first sums (rounds_of) have a launch each, with a workgroup per chunk of the
// row; each of them walks to the next sum that is needed, from where the
// launch before stopped, and a last launch, one workgroup per prompt, adds up
// what is left and draws.
#include "tree.h"

namespace cdsl {

namespace {

struct At;
constexpr int NT = 1024, NW = NT / 64;
constexpr int RUN = 1024;                       // consecutive ids of a wave in a chunk: 16 a lane
constexpr int CHUNK = NW * RUN;
constexpr int kSegs = kAcceptMaxVocab / RUN;    // (chunk, wave) sums at most
constexpr int kHeld = 2;                        // chunks that registers hold
constexpr int kRounds = 5;                      // sums of a long row that have a launch of their own, at most

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
// Their sum: three fp64 instructions an entry behind the conversions (they bound
// a pass).  A maximum drops NaNs, so they are looked for among the entries where
// one is 2 or above, which no probability is.  Each term is taken at 0 before it
// is added: sum d and sum |d|, whose half it is as well, lose what is left
// beside rejected tokens once c is large.
__device__ __forceinline__ double weights(const Piece& p, const Piece& q, double c) {
  double s = 0.;
  unsigned bits = 0;
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s += fmax(fma(-c, (double)q.x[u][e], (double)p.x[u][e]), 0.);
      bits |= __float_as_uint(p.x[u][e]) | __float_as_uint(q.x[u][e]);
    }
  if (bits & 0x40000000u) {
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (__builtin_isnan(p.x[u][e] - q.x[u][e])) s = NAN;   // one of them is, or both are infinite
  }
  return s;
}

struct AcceptArgs {
  const float* p;
  const float* q;
  int n, V;
  const int* tokens;
  const int* parents;
  const int* n_nodes;
  const float* u;
  const float* v;
  int replace;
  int* path;
  int* n_path;
  int* next_token;
  // long rows: what the launches hand on (see tree_accept_workspace)
  At* at;           // [kRounds][B]: where a round's walk stopped
  double* parts;           // [kRounds][B][segs]: the sums of runs that it stopped for
  float* kids;             // [2][B][n]: the children's p and q
  long long kid_stride;    // B * n
  int round;               // rounds before this launch
};

// A prompt's tree in LDS, and the state of its walk; alike in every wave.
struct Walk {
  int par[kTreeMax], tok[kTreeMax];
  float px[kTreeMax], qx[kTreeMax], us[kTreeMax];
};
struct At {
  int cur = 0, len = 1, from = 1;
  int none = 0;            // no mass left
  int summed = 0;          // N is the sum of the present c
  int fell = -1;           // the child that is being rejected (stopped for its sum)
  int over = 0;            // walked, and summed
  double c = 0., N = 1., rest = 1.;
};

// First launch: the children's probabilities come from their rows, and later
// launches find them in a.kids.
template <bool FIRST>
__device__ __forceinline__ void fetch_tree(const AcceptArgs& a, int b, int nb, bool keep, Walk& w) {
  const long long row0 = (long long)b * a.n;
  for (int j = threadIdx.x; j < nb; j += NT) {
    int c = j > 0 ? a.parents[row0 + j] : -1;
    const int x = a.tokens[row0 + j];
    const float uj = a.u[row0 + j];
    float* kp = a.kids + row0 + j;
    float* kq = kp + a.kid_stride;
    float pj = 0.f, qj = 0.f;
    if constexpr (!FIRST) pj = *kp, qj = *kq;
    if (c < 0 || c >= j || x < 0 || x >= a.V) c = -1;   // not a child that can be taken
    if (FIRST && c >= 0) {
      pj = a.p[(row0 + c) * a.V + x];
      qj = a.q[(row0 + c) * a.V + x];
    }
    if (FIRST && keep) *kp = pj, *kq = qj;
    w.par[j] = c;
    w.tok[j] = x;
    w.px[j] = pj;
    w.qx[j] = qj;
    w.us[j] = uj;
  }
  __syncthreads();
}

// What follows a sum (at.N, for at.c).
__device__ __forceinline__ void walk_summed(const AcceptArgs& a, const Walk& w, At& at) {
  const int lane = threadIdx.x & 63, fell = at.fell;
  at.fell = -1;
  at.summed = 1;
  if (fell < 0) {
    at.over = 1;
    return;
  }
  if (!a.replace) {
    // a token that an earlier sibling carried is out of q already
    bool twice = false;
    for (int s = 0; s < fell; s += 64) {
      const int e = s + lane;
      twice = twice || __ballot(e < fell && w.par[e] == at.cur && w.tok[e] == w.tok[fell]);
    }
    if (!twice) at.rest -= (double)w.qx[fell];
  }
  if (!(at.N > 0.)) at.none = 1;
}

// Walks to the next sum that is needed, for at.c; false: none is (at.over).
// moved(node, place on the path): a node is reached.
template <typename Moved>
__device__ __forceinline__ bool walk_on(const Walk& w, int nb, At& at, Moved&& moved) {
  const int lane = threadIdx.x & 63;
  if (at.over) return false;
  int fell = -1;   // the child that is rejected next
  while (at.from < nb && !at.none && fell < 0) {   // 64 nodes at a time
    const int j0 = at.from & ~63, j = j0 + lane;
    const unsigned long long kids = __ballot(j >= at.from && j < nb && w.par[j] == at.cur);
    if (!kids) {
      at.from = j0 + 64;
      continue;
    }
    const int k = j0 + __builtin_ctzll(kids);
    at.from = k + 1;
    if (!(at.rest > 0.)) continue;
    const double pk = at.c > 0. ? weight(w.px[k], w.qx[k], at.c) / at.N : (double)w.px[k];
    const double qk = (double)w.qx[k] / at.rest;
    if (pk > 0. && (double)w.us[k] * qk <= pk) {
      moved(k, at.len);
      ++at.len;
      at.cur = k;
      at.c = 0., at.N = 1., at.rest = 1.;
      at.summed = 0;
    } else {
      fell = k;
    }
  }
  if (fell < 0 && at.summed) {
    at.over = 1;
    return false;
  }
  at.fell = fell;
  if (fell >= 0) at.c += at.N / at.rest;
  return true;
}

// Sum of the parts of a row, in every lane.
__device__ __forceinline__ double sum_parts(const double* part, int segs) {
  double t = 0.;
  for (int k = threadIdx.x & 63; k < segs; k += 64) t += part[k];
  return wave_sum_d(t);
}

// The state after the rounds before this launch: where the last one stopped,
// with the sum that it stopped for.  (Loaded before the tree, so that their
// latencies overlap; the parts of a prompt that is over are not used.)
__device__ __forceinline__ At stopped(const AcceptArgs& a, int b, int B, int segs) {
  At at;
  if (a.round > 0) {
    const long long slot = (long long)(a.round - 1) * B + b;
    const double* part = a.parts + slot * segs;
    double t = 0.;
    for (int k = threadIdx.x & 63; k < segs; k += 64) t += part[k];
    at = a.at[slot];
    if (!at.over) at.N = wave_sum_d(t);
  }
  return at;
}

// One round: the walk to the next sum, and the sums of this chunk's runs for
// it.  Workgroup = (chunk, prompt); the first of a prompt hands the state on.
template <bool FIRST>
__global__ __launch_bounds__(NT) void tree_sums_kernel(AcceptArgs a) {
  __shared__ Walk w;
  const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int nb = a.n_nodes ? min(max(a.n_nodes[b], 1), a.n) : a.n;
  const int segs = gridDim.x * NW;
  const bool lead = blockIdx.x == 0 && tid == 0;
  const long long row0 = (long long)b * a.n;
  At at = stopped(a, b, gridDim.y, segs);
  fetch_tree<FIRST>(a, b, nb, blockIdx.x == 0, w);
  if (!FIRST && !at.over) walk_summed(a, w, at);
  const bool need = walk_on(w, nb, at, [&](int k, int place) {
    if (lead) a.path[row0 + place] = k;
  });
  const long long slot = (long long)a.round * gridDim.y + b;
  if (lead) a.at[slot] = at;
  if (!need) return;
  const long long row = (row0 + at.cur) * a.V;
  const int i = CHUNK * blockIdx.x + wv * RUN + 4 * lane;
  Piece p, q{};
  p.load(a.p + row, i, a.V);
  if (at.c > 0.) q.load(a.q + row, i, a.V);
  const double s = wave_sum_d(weights(p, q, at.c));
  if (lane == 0) a.parts[slot * segs + blockIdx.x * NW + wv] = s;
}

// CHUNKS: V <= CHUNKS * CHUNK, the one launch (one chunk of registers takes 18 us
// over 16384 ids and 27 for 45 prompts over 12368, where two take 22.5 and 35; two
// fill the 128 registers, one value more lives in scratch); 0: the one after the
// rounds.
template <int CHUNKS>
__global__ __launch_bounds__(NT) void tree_accept_kernel(AcceptArgs a) {
  constexpr bool HELD = CHUNKS > 0;
  __shared__ Walk w;
  __shared__ double part[HELD ? CHUNKS * NW : kSegs];
  __shared__ int hit, best_i[NW];
  __shared__ float best_v[NW];
  const int b = blockIdx.x, V = a.V, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int nb = a.n_nodes ? min(max(a.n_nodes[b], 1), a.n) : a.n;
  const long long row0 = (long long)b * a.n;
  if (tid == 0) hit = -1;
  const int chunks = (V + CHUNK - 1) / CHUNK, segs = chunks * NW;
  At at = stopped(a, b, gridDim.x, segs);
  fetch_tree<HELD>(a, b, nb, false, w);
  const int at0 = wv * RUN + 4 * lane;   // this lane's first id of a chunk
  bool known = false;      // the parts that at.N is the sum of are in a.parts
  if constexpr (!HELD) {
    if (!at.over) walk_summed(a, w, at);
    known = true;
  }
  const float* p = a.p + (row0 + at.cur) * V;
  const float* q = a.q + (row0 + at.cur) * V;
  Piece hp[HELD ? CHUNKS : 1], hq[HELD ? CHUNKS : 1];
  bool have_p = false, have_q = false;   // the held pieces are those of the node reached

  while (walk_on(w, nb, at, [&](int k, int place) {
    if (tid == 0) a.path[row0 + place] = k;
    p = a.p + (row0 + k) * V;
    q = a.q + (row0 + k) * V;
    have_p = have_q = false;
  })) {
    // part[chunk * NW + wave] and their sum, for the present c
    const double c = at.c;
    known = false;
    __syncthreads();   // earlier readers of part are done
    if constexpr (HELD) {
      const bool lp = !have_p, lq = !have_q && c > 0.;
#pragma unroll
      for (int k = 0; k < CHUNKS; ++k) {
        if (lp) hp[k].load(p, CHUNK * k + at0, V);
        if (lq) hq[k].load(q, CHUNK * k + at0, V);
        else if (c == 0.) hq[k] = Piece{};
      }
      have_p = true;
      have_q = c > 0.;
      double s[CHUNKS];
#pragma unroll
      for (int k = 0; k < CHUNKS; ++k) s[k] = wave_sum_d(weights(hp[k], hq[k], c));
      if (lane == 0)
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k)
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
    at.N = sum_parts(part, segs);
    walk_summed(a, w, at);
  }
  if (!HELD && known) {
    // they are the last ones that a round stopped for (the first round always does)
    int r = a.round - 1;
    while (r > 0 && a.at[(long long)r * gridDim.x + b].over) --r;
    const double* from = a.parts + ((long long)r * gridDim.x + b) * segs;
    for (int k = tid; k < segs; k += NT) part[k] = from[k];
    __syncthreads();
  }

  // The draw: the first id whose running sum passes v * (sum).
  const double c = at.c, N = at.N;
  if (at.none) {
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
    // first entry of a row of lanes whose running sum from `sum_at` passes T (the
    // last one with mass when rounding leaves T past the total), and the sum
    // before it
    auto locate = [&](double mine, double T, double& sum_at) __attribute__((always_inline)) -> int {
      double incl = mine;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const double t = __shfl_up(incl, o, 64);
        if (lane >= o) incl += t;
      }
      double before = __shfl_up(incl, 1, 64);
      if (lane == 0) before = 0.;
      const unsigned long long past = __ballot(mine > 0. && sum_at + incl > T), mass = __ballot(mine > 0.);
      const int src = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(mass | 1ull);
      sum_at += __shfl(before, src, 64);
      return mass ? src : -1;
    };
    const double T = (double)a.v[b] * N;
    // each lane takes a run of segments
    const int run = (segs + 63) / 64;
    double mine = 0., from = 0.;
    for (int s = lane * run; s < min(segs, lane * run + run); ++s) mine += part[s];
    const int src = locate(mine, T, from);
    int seg = -1;
    double seg_at = from;
    for (int s = src * run; src >= 0 && s < min(segs, src * run + run); ++s) {
      if (part[s] > 0.) {
        seg = s;
        seg_at = from;
        if (from + part[s] > T) break;
      }
      from += part[s];
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
  for (int i = at.len + tid; i < a.n; i += NT) a.path[row0 + i] = -1;
  if (tid == 0) {
    a.path[row0] = 0;
    a.n_path[b] = at.len;
    a.next_token[b] = hit;
  }
}

int chunks_of(int V) { return (V + CHUNK - 1) / CHUNK; }

// The more prompts, the longer the longest walk; the longer the rows, the more a
// sum in the last launch costs.  Trees of 65 (us, with 2, 4 and 5 rounds):
//   prompts         8                16                24                32
//   35101    31.6 33.0 35.4   36.5 36.5 38.9   38.9 39.7 40.8   39.4 38.8 40.6
//   65536    27.9 29.3 32.1   35.9 33.2 36.1   43.0 41.5 43.2   38.5 36.6 38.6
//   128256   40.3 31.9 35.6   48.3 39.6 40.5   55.7 47.4 47.3   68.9 55.7 52.2
// (how many children each draw rejects makes up to 10 us of them).
int rounds_of(int B, int V) { return B >= 32 ? kRounds : B <= 16 && V <= 4 * CHUNK ? 2 : 4; }

}  // namespace

namespace {
struct AcceptWs {
  size_t parts, kids, total;   // the states come first
};
AcceptWs accept_ws(int B, int n, int V) {
  auto al = [](size_t x) { return (x + 255) & ~(size_t)255; };
  AcceptWs w{};
  if (V <= kHeld * CHUNK) return w;
  w.parts = al(sizeof(At) * kRounds * B);
  w.kids = w.parts + al((size_t)kRounds * B * chunks_of(V) * NW * sizeof(double));
  w.total = w.kids + (size_t)2 * B * n * sizeof(float);
  return w;
}
}  // namespace

size_t tree_accept_workspace(int B, int n, int V) { return accept_ws(B, n, V).total; }

hipError_t tree_accept_launch(const float* p, const float* q, int B, int n, int V, const int* tokens,
                              const int* parents, const int* n_nodes, const float* u, const float* v, int replace,
                              int* path, int* n_path, int* next_token, void* workspace, hipStream_t st) {
  if (B == 0) return hipSuccess;
  AcceptArgs a{};
  a.p = p;
  a.q = q;
  a.n = n;
  a.V = V;
  a.tokens = tokens;
  a.parents = parents;
  a.n_nodes = n_nodes;
  a.u = u;
  a.v = v;
  a.replace = replace;
  a.path = path;
  a.n_path = n_path;
  a.next_token = next_token;
  a.kid_stride = (long long)B * n;
  if (V <= kHeld * CHUNK) {
    if (V <= CHUNK) tree_accept_kernel<1><<<B, NT, 0, st>>>(a);
    else tree_accept_kernel<kHeld><<<B, NT, 0, st>>>(a);
    return hipGetLastError();
  }
  const AcceptWs ws = accept_ws(B, n, V);
  a.at = (At*)workspace;
  a.parts = (double*)((char*)workspace + ws.parts);
  a.kids = (float*)((char*)workspace + ws.kids);
  const dim3 grid((unsigned)chunks_of(V), (unsigned)B);
  const int rounds = rounds_of(B, V);
  for (; a.round < rounds; ++a.round) {
    if (a.round == 0) tree_sums_kernel<true><<<grid, NT, 0, st>>>(a);
    else tree_sums_kernel<false><<<grid, NT, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  tree_accept_kernel<0><<<B, NT, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace cdsl

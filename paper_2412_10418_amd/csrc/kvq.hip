// The 8-bit paged cache: rows quantised as they are written, read back, and
// the kept path of a tree moved to the front of the tree's slots.
//
// One scale per (token, KV head) row x of hd values, a = max |x|:
//   int8  s = max(a / 127, 2^-126) (rounded to fp32), code = x / s to the
//         nearest integer, ties to even
//   e4m3  s = the smallest power of two with a <= 448 s, at least 2^-126;
//         code = x / s (exact) to the nearest e4m3, ties to even
// A row that holds a NaN or an infinity has s = NaN and codes 0: it reads
// back as NaN.  Scales stay fp32, so that a value differs from its input by
// its code's rounding alone.
#include <type_traits>

#include "tree.h"

namespace cdsl {

namespace {

template <typename T>
__device__ __forceinline__ void load4(const T* p, float (&x)[4]);
template <>
__device__ __forceinline__ void load4<float>(const float* p, float (&x)[4]) {
  const f32x4 t = *(const f32x4*)p;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = t[e];
}
template <>
__device__ __forceinline__ void load4<bf16>(const bf16* p, float (&x)[4]) {
  const bf16x4 t = *(const bf16x4*)p;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = (float)t[e];
}

// Codes of four values of one row as bytes, from the row's scale s.
template <int FMT>
__device__ __forceinline__ unsigned encode4(const float (&x)[4], float s) {
  if constexpr (FMT == kE4M3) {
    // 1 / s of a power of two, exact
    const float inv = __uint_as_float((254u << 23) - __float_as_uint(s));
    unsigned w = 0;
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, w, true);
    return w;
  } else {
    // 1 / s to 2^-23 of itself by one Newton step, so that x / s <= 127.5 is off
    // by less than 2^-15: the nearest integer is the right one unless x / s
    // lies as near to a tie.  There (once in 2^14 values) the signs of
    // x - s (n +- 1/2), which one fused multiply-add gives exactly, tell.
    float inv = __builtin_amdgcn_rcpf(s);
    inv = fmaf(inv, fmaf(-s, inv, 1.f), inv);
    float n[4], far = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float r = x[e] * inv;
      n[e] = __builtin_rintf(r);
      far = fmaxf(far, fabsf(r - n[e]));
    }
    if (far > 0.5f - 0x1p-14f) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float up = fmaf(-s, n[e] + 0.5f, x[e]), dn = fmaf(-s, n[e] - 0.5f, x[e]);
        const bool odd = (int)n[e] & 1;
        if (up > 0.f || (up == 0.f && odd)) n[e] += 1.f;
        else if (dn < 0.f || (dn == 0.f && odd)) n[e] -= 1.f;
      }
    }
    // 1.5 2^23 + n has n in its low bits
    unsigned u[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = __float_as_uint(n[e] + 0x1.8p23f);
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(u[3], u[2], 0x0c0c0400), __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400),
                                 0x05040100);
  }
}

template <int FMT>
__device__ __forceinline__ float scale_of(float a) {
  if constexpr (FMT == kE4M3) {
    const unsigned u = __float_as_uint(a);
    // a = m 2^e: 448 = 1.75 * 2^8
    const int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return __uint_as_float((unsigned)max(e, 1) << 23);
  } else {
    // a / 127 rounded to nearest: with the rounded reciprocal, one correction
    // by the exact remainder gives it (Markstein 1990; checked for every a)
    constexpr float y = 1.f / 127.f;
    const float t = a * y;
    return fmaxf(fmaf(fmaf(-127.f, t, a), y, t), 1.1754943508222875e-38f);
  }
}

template <int FMT>
__device__ __forceinline__ void decode4(unsigned w, float s, float (&y)[4]) {
  if constexpr (FMT == kE4M3) {
    y[0] = __builtin_amdgcn_cvt_f32_fp8(w, 0) * s;
    y[1] = __builtin_amdgcn_cvt_f32_fp8(w, 1) * s;
    y[2] = __builtin_amdgcn_cvt_f32_fp8(w, 2) * s;
    y[3] = __builtin_amdgcn_cvt_f32_fp8(w, 3) * s;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (float)(int8_t)(w >> (8 * e)) * s;
  }
}

// Bytes (t, e) -> (e, t) of four words.
__device__ __forceinline__ void transpose4(const unsigned (&w)[4], unsigned (&o)[4]) {
  const unsigned a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400), b = __builtin_amdgcn_perm(w[3], w[2], 0x05010400);
  const unsigned c = __builtin_amdgcn_perm(w[1], w[0], 0x07030602), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602);
  o[0] = __builtin_amdgcn_perm(b, a, 0x05040100);
  o[1] = __builtin_amdgcn_perm(b, a, 0x07060302);
  o[2] = __builtin_amdgcn_perm(d, c, 0x05040100);
  o[3] = __builtin_amdgcn_perm(d, c, 0x07060302);
}

// Maximum over groups of LANES lanes (8, 16 or 32): within quads, halves of a
// row, rows of 16, then the two rows; vector instructions only (shuffles
// through LDS, 40 a thread, took 6 us of 42 at 24 prompts of up to 2047).
template <int CTRL>
__device__ __forceinline__ unsigned max_moved(unsigned a) {
  return max(a, (unsigned)__builtin_amdgcn_update_dpp(0, (int)a, CTRL, 0xf, 0xf, false));
}
template <int LANES>
__device__ __forceinline__ unsigned group_max(unsigned a) {
  a = max_moved<0xB1>(a);                             // quad_perm 1 0 3 2
  a = max_moved<0x4E>(a);                             // quad_perm 2 3 0 1
  a = max_moved<0x141>(a);                            // row_half_mirror
  if constexpr (LANES > 8) a = max_moved<0x140>(a);   // row_mirror
  if constexpr (LANES > 16) {
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    const u32x2 t = __builtin_amdgcn_permlane16_swap(a, a, false, false);
    a = max(t.x, t.y);
  }
  return a;
}

// Where word w of a unit's codes stands in LDS: the sixteen 16-byte chunks of a
// row of 64 words are permuted by the row, so that neither the order of the
// rows (dims along the lanes) nor that of the unit meets one bank often.
__device__ __forceinline__ int banked(int w) { return w ^ ((w >> 6 & 15) << 2); }

// Threads of a workgroup: a task is four slots x four dims of the keys or of
// the values (16 hd / 4 tasks a unit), so that a quarter-row load or store of
// the fp32 or bf16 side is contiguous over the lanes and a task's 4 x 4 codes
// are whole words in both orders.
template <int HD>
constexpr int kvq_threads() { return 4 * HD < 256 ? 4 * HD : 256; }

// Workgroup = (page of the prompt's run, KV head, prompt).  The bytes of the
// rows bound it (in fp32 they are 4 of every 5 bytes moved): 16 prompts of 256
// x 32 heads of 128 in fp32 take 29.6 us, 5.7 TB/s with what the last cache holds,
// 24 of up to 2047 x 8 in bf16 32.0.  Branches for every row and tie, rather than
// for the page and four values, cost 5 and 10 us.
template <int HD, int FMT, typename T>
__global__ __launch_bounds__(kvq_threads<HD>()) void kvq_write_kernel(KvqView c, KvqRows r) {
  constexpr int NT = kvq_threads<HD>();
  constexpr int LQ = HD / 4;                 // lanes per quad of slots
  constexpr int PER = 4 * HD / NT;           // tasks per thread
  __shared__ __attribute__((aligned(16))) unsigned lds[2 * kPage * HD / 4];
  const int b = blockIdx.y, h = blockIdx.x % c.Hkv;
  const KvqRun run = kvq_run(r.start, r.count, r.T, b);
  const long long beg = run.beg, end = run.end;
  const long long page = kvq_first_page(run) + blockIdx.x / c.Hkv;
  const long long base = page * kPage;
  if (base >= end || base + kPage <= beg) return;
  uint8_t* unit = kvq_unit_of(c, b, page, h);
  if (!unit) return;
  // whole pages go through LDS, so that their lines leave whole; of the others
  // only the run's bytes are written
  auto page_rows = [&](auto all) __attribute__((always_inline)) {
    constexpr bool WHOLE = decltype(all)::value;
    float x[PER][4][4];
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int task = threadIdx.x + NT * u;
      const int isv = task / (8 * LQ), quad = task / LQ % 8, d = task % LQ * 4;
      const T* src = (const T*)(isv ? r.V : r.K) + (isv ? r.vsb : r.ksb) * b + h * HD + d;
      const long long ts = isv ? r.vst : r.kst;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const long long pos = base + 4 * quad + t;
        if (WHOLE || (pos >= beg && pos < end)) load4<T>(src + (pos - beg) * ts, x[u][t]);
        else x[u][t][0] = x[u][t][1] = x[u][t][2] = x[u][t][3] = 0.f;
      }
    }
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int task = threadIdx.x + NT * u;
      const int isv = task / (8 * LQ), quad = task / LQ % 8, d = task % LQ * 4;
      float s[4];
      unsigned w[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        // the largest bit pattern of |x|: NaN and infinity stay on top
        unsigned a = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) a = max(a, __float_as_uint(x[u][t][e]) & 0x7fffffffu);
        a = group_max<LQ>(a);
        const bool bad = a >= 0x7f800000u;
        s[t] = scale_of<FMT>(__uint_as_float(a));
        w[t] = encode4<FMT>(x[u][t], s[t]);
        s[t] = bad ? __uint_as_float(0x7fc00000u) : s[t];
        w[t] = bad ? 0u : w[t];
      }
      const int slot = 4 * quad;
      float* sc = (float*)(unit + (isv ? kvq_value_scale_at(HD, slot) : kvq_key_scale_at(HD, slot)));
      if constexpr (WHOLE) {
        if (d == 0) *(f32x4*)sc = (f32x4){s[0], s[1], s[2], s[3]};
        unsigned o[4];
        if (isv) transpose4(w, o);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          if (isv) lds[banked(kvq_value_at(HD, slot, d + t) / 4)] = o[t];
          else lds[banked(kvq_key_at(slot + t, d) / 4)] = w[t];
        }
      } else {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const bool live = base + slot + t >= beg && base + slot + t < end;
          if (!live) continue;
          if (d == 0) sc[t] = s[t];
          if (!isv) *(unsigned*)(unit + kvq_key_at(slot + t, d)) = w[t];
          else
#pragma unroll
            for (int e = 0; e < 4; ++e) unit[kvq_value_at(HD, slot + t, d + e)] = (uint8_t)(w[t] >> (8 * e));
        }
      }
    }
  };
  if (base < beg || base + kPage > end) {   // uniform over the workgroup
    page_rows(std::false_type{});
    return;
  }
  page_rows(std::true_type{});
  __syncthreads();
#pragma unroll
  for (int i = threadIdx.x; i < 2 * kPage * HD / 16; i += NT) *((u32x4*)unit + i) = *(const u32x4*)&lds[banked(4 * i)];
}

// Workgroup = (page of the prompt's run, KV head, prompt): the unit comes in
// as 16-byte pieces, the rows leave as whole lines.  Rows of a page outside
// the pool are NaN.
template <int HD, int FMT, typename T>
__global__ __launch_bounds__(kvq_threads<HD>()) void kvq_read_kernel(KvqView c, KvqRows r) {
  constexpr int NT = kvq_threads<HD>();
  constexpr int LQ = HD / 4;
  constexpr int PER = 4 * HD / NT;
  constexpr int WORDS = kvq_unit_bytes(HD) / 4, CODES = 2 * kPage * HD / 4;
  __shared__ __attribute__((aligned(16))) unsigned lds[WORDS];
  const int b = blockIdx.y, h = blockIdx.x % c.Hkv;
  const KvqRun run = kvq_run(r.start, r.count, r.T, b);
  const long long beg = run.beg, end = run.end;
  const long long page = kvq_first_page(run) + blockIdx.x / c.Hkv;
  const long long base = page * kPage;
  if (base >= end || base + kPage <= beg) return;
  const uint8_t* unit = kvq_unit_of(c, b, page, h);
  if (unit) {
    for (int i = threadIdx.x; i < WORDS / 4; i += NT)
      *(u32x4*)&lds[4 * i < CODES ? banked(4 * i) : 4 * i] = *((const u32x4*)unit + i);
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int task = threadIdx.x + NT * u;
    const int isv = task / (8 * LQ), slot = task / LQ % 8 * 4, d = task % LQ * 4;
    unsigned w[4];
    float s[4];
    if (unit) {
      unsigned o[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        o[t] = lds[banked((isv ? kvq_value_at(HD, slot, d + t) : kvq_key_at(slot + t, d)) / 4)];
        s[t] = __uint_as_float(lds[(isv ? kvq_value_scale_at(HD, slot + t) : kvq_key_scale_at(HD, slot + t)) / 4]);
      }
      if (isv) transpose4(o, w);
      else
#pragma unroll
        for (int t = 0; t < 4; ++t) w[t] = o[t];
    } else {
#pragma unroll
      for (int t = 0; t < 4; ++t) w[t] = 0u, s[t] = __uint_as_float(0x7fc00000u);
    }
    T* dst = (T*)(isv ? r.Vo : r.Ko) + h * HD + d;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const long long pos = base + slot + t;
      if (pos < beg || pos >= end) continue;
      float y[4];
      decode4<FMT>(w[t], s[t], y);
      T* o = dst + ((long long)b * r.T + (pos - beg)) * c.Hkv * HD;
      if constexpr (sizeof(T) == 4) *(f32x4*)o = (f32x4){y[0], y[1], y[2], y[3]};
      else *(bf16x4*)o = (bf16x4){(bf16)y[0], (bf16)y[1], (bf16)y[2], (bf16)y[3]};
    }
  }
}

// The pointer that another lane holds.
template <typename P>
__device__ __forceinline__ P* ptr_of_lane(P* p, int lane) {
  return (P*)__shfl((long long)p, lane, 64);
}

// Moves of single tokens.  One wave per (layer, KV head, prompt); entry i of the
// path moves from slot L + path[i] to L + i.  Eight entries at a time are read
// before any of them is written; with path ascending, path[i] >= i, so that no
// later entry's source has been written by then.
//
// A token's keys lie in hd / 8 runs of 8 bytes: one instruction moves those of
// several tokens.  Its values lie one byte in eight: a lane reads the 16 bytes
// around two of them (dims x and x + 16) and collects those of eight tokens; the
// eight slots that they go to lie in at most three aligned groups of four, so
// that three reads and three writes of 16 bytes place them all.  (The page is
// the prompt's own from lens on, so the other bytes may be written back.)  The
// requests bound it: 16 prompts x 8 tokens x 256 units of hd = 128, 17 MB of
// tokens, 11.5 us; with a byte at a time 16.5 (64 prompts: 39 and 72).
template <int HD>
__global__ __launch_bounds__(64) void kvq_keep_kernel(KvqView c, long long layer_bytes, const int* lens,
                                                      const int* path, const int* n_path, int n, int* new_lens) {
  constexpr int CH = 8;
  constexpr int KL = HD / 8, TK = 64 / KL < CH ? 64 / KL : CH;   // lanes of a token's keys, tokens at once
  constexpr int VL = HD / 2, TV = 64 / VL;                       // the same for values
  const int b = blockIdx.y, h = blockIdx.x % c.Hkv, layer = blockIdx.x / c.Hkv;
  const int lane = threadIdx.x;
  c.pool += layer * layer_bytes;
  const int L = max(lens[b], 0);
  const int m = min(max(n_path[b], 0), n);
  if (new_lens && blockIdx.x == 0 && lane == 0) new_lens[b] = (int)min((long long)L + m, 0x7fffffffll);
  // a lane's 16 bytes of values in the group of four slots that holds `slot`
  auto values_at = [&](int slot) __attribute__((always_inline)) {
    const int x = lane % VL;
    return kPage * HD + x / 16 * 1024 + slot % 16 / 4 * 256 + x % 16 * 16;
  };
  for (int i0 = 0; i0 < m; i0 += CH) {
    // lanes 0..7: an entry's source and destination units (null: not moved);
    // lanes 8..10: the units of the groups of four that the entries go to
    const long long first = (long long)L + i0;
    const int off = (int)(first & 3);
    const uint8_t* src = nullptr;
    uint8_t* dst = nullptr;
    int ss = 0, ds = 0;
    if (lane < CH && i0 + lane < m) {
      const int i = i0 + lane, from = path[(long long)b * n + i];
      if (from > i && from < kTreeMax) {
        const long long sp = (long long)L + from, dp = (long long)L + i;
        src = kvq_unit_of(c, b, sp / kPage, h);
        dst = kvq_unit_of(c, b, dp / kPage, h);
        if (!src || !dst) src = dst = nullptr;
        ss = (int)(sp % kPage);
        ds = (int)(dp % kPage);
      }
    } else if (lane >= CH && lane < CH + 3) {
      const long long dp = first - off + 4 * (lane - CH);
      dst = kvq_unit_of(c, b, dp / kPage, h);
      ds = (int)(dp % kPage);
    }
    const unsigned moved = (unsigned)__ballot(src != nullptr);
    if (!moved) continue;

    uint2 kr[CH / TK];
#pragma unroll
    for (int j = 0; j < CH / TK; ++j) {
      const int e = j * TK + lane / KL;   // (past the eighth: null)
      const uint8_t* s = ptr_of_lane(src, e);
      const int slot = __shfl(ss, e, 64);
      if (s) kr[j] = *(const uint2*)(s + kvq_key_at(slot, lane % KL * 8));
    }
    float sc = 0.f;
    {
      const uint8_t* s = ptr_of_lane(src, lane / 2);
      const int slot = __shfl(ss, lane / 2, 64);
      if (s) sc = *(const float*)(s + (lane & 1 ? kvq_value_scale_at(HD, slot) : kvq_key_scale_at(HD, slot)));
    }
    u32x4 vr[CH / TV];
#pragma unroll
    for (int j = 0; j < CH / TV; ++j) {
      const int e = j * TV + lane / VL;
      const uint8_t* s = ptr_of_lane(src, e);
      const int slot = __shfl(ss, e, 64);
      vr[j] = s ? *(const u32x4*)(s + values_at(slot)) : (u32x4){0u, 0u, 0u, 0u};
    }
    // byte e: entry e's value, of dims x and x + 16
    unsigned long long got[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < CH / TV; ++j) {
      const int e = j * TV + lane / VL;
      const int slot = __shfl(ss, e, 64);
      got[0] |= (unsigned long long)((slot & 16 ? vr[j].y : vr[j].x) >> (8 * (slot & 3)) & 255u) << (8 * e);
      got[1] |= (unsigned long long)((slot & 16 ? vr[j].w : vr[j].z) >> (8 * (slot & 3)) & 255u) << (8 * e);
    }
#pragma unroll
    for (int o = VL; o < 64; o <<= 1)
#pragma unroll
      for (int k = 0; k < 2; ++k) got[k] |= (unsigned long long)__shfl_xor((long long)got[k], o, 64);
    // the moved entries' bytes
    unsigned long long mask = 0;
#pragma unroll
    for (int e = 0; e < CH; ++e) mask |= moved >> e & 1u ? 255ull << (8 * e) : 0ull;
    // their word in group k of four slots: bytes 4 k - off .. + 3
    auto group = [&](unsigned long long w, int k) __attribute__((always_inline)) {
      return k == 0 ? (unsigned)w << (8 * off) : k == 1 ? (unsigned)(w >> (32 - 8 * off))
                                                        : off ? (unsigned)(w >> (64 - 8 * off)) : 0u;
    };
    u32x4 old[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const uint8_t* d = ptr_of_lane(dst, CH + k);
      const int slot = __shfl(ds, CH + k, 64);
      if (lane < VL && group(mask, k)) old[k] = *(const u32x4*)(d + values_at(slot));
    }

#pragma unroll
    for (int j = 0; j < CH / TK; ++j) {
      const int e = j * TK + lane / KL;
      const bool live = ptr_of_lane(src, e) != nullptr;
      uint8_t* d = ptr_of_lane(dst, e);
      const int slot = __shfl(ds, e, 64);
      if (live) *(uint2*)(d + kvq_key_at(slot, lane % KL * 8)) = kr[j];
    }
    {
      const bool live = ptr_of_lane(src, lane / 2) != nullptr;
      uint8_t* d = ptr_of_lane(dst, lane / 2);
      const int slot = __shfl(ds, lane / 2, 64);
      if (live) *(float*)(d + (lane & 1 ? kvq_value_scale_at(HD, slot) : kvq_key_scale_at(HD, slot))) = sc;
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      uint8_t* d = ptr_of_lane(dst, CH + k);
      const int slot = __shfl(ds, CH + k, 64);
      const unsigned on = group(mask, k);
      if (lane < VL && on) {
        u32x4 w = old[k];
        const unsigned x0 = group(got[0], k), x1 = group(got[1], k);
        if (slot & 16) {
          w.y = (w.y & ~on) | (x0 & on);
          w.w = (w.w & ~on) | (x1 & on);
        } else {
          w.x = (w.x & ~on) | (x0 & on);
          w.z = (w.z & ~on) | (x1 & on);
        }
        *(u32x4*)(d + values_at(slot)) = w;
      }
    }
  }
}

template <int HD, int FMT>
hipError_t rows_launch(const KvqView& c, const KvqRows& r, bool write, hipStream_t st) {
  const dim3 grid((unsigned)(kvq_run_pages(r.T) * c.Hkv), (unsigned)c.B);
  const int nt = kvq_threads<HD>();
  if (write) {
    if (r.dtype == 1) kvq_write_kernel<HD, FMT, bf16><<<grid, nt, 0, st>>>(c, r);
    else kvq_write_kernel<HD, FMT, float><<<grid, nt, 0, st>>>(c, r);
  } else {
    if (r.dtype == 1) kvq_read_kernel<HD, FMT, bf16><<<grid, nt, 0, st>>>(c, r);
    else kvq_read_kernel<HD, FMT, float><<<grid, nt, 0, st>>>(c, r);
  }
  return hipGetLastError();
}

template <int HD>
hipError_t rows_format(const KvqView& c, const KvqRows& r, bool write, hipStream_t st) {
  return c.format == kE4M3 ? rows_launch<HD, kE4M3>(c, r, write, st) : rows_launch<HD, kInt8>(c, r, write, st);
}

hipError_t rows_any(const KvqView& c, const KvqRows& r, bool write, hipStream_t st) {
  if (c.B == 0 || r.T == 0) return hipSuccess;
  switch (c.hd) {
    case 32: return rows_format<32>(c, r, write, st);
    case 64: return rows_format<64>(c, r, write, st);
    case 128: return rows_format<128>(c, r, write, st);
  }
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t kvq_write_launch(const KvqView& c, const KvqRows& r, hipStream_t st) { return rows_any(c, r, true, st); }
hipError_t kvq_read_launch(const KvqView& c, const KvqRows& r, hipStream_t st) { return rows_any(c, r, false, st); }

hipError_t kvq_keep_launch(const KvqView& c, int n_layers, long long layer_bytes, const int* lens, const int* path,
                           const int* n_path, int n, int* new_lens, hipStream_t st) {
  if (c.B == 0) return hipSuccess;
  const dim3 grid((unsigned)(n_layers * c.Hkv), (unsigned)c.B);
  switch (c.hd) {
    case 32: kvq_keep_kernel<32><<<grid, 64, 0, st>>>(c, layer_bytes, lens, path, n_path, n, new_lens); break;
    case 64: kvq_keep_kernel<64><<<grid, 64, 0, st>>>(c, layer_bytes, lens, path, n_path, n, new_lens); break;
    case 128: kvq_keep_kernel<128><<<grid, 64, 0, st>>>(c, layer_bytes, lens, path, n_path, n, new_lens); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace cdsl

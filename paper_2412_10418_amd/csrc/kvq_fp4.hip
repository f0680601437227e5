// The 4-bit paged cache: rows quantised as they are written, read back, and the
// kept path of a tree moved to the front of the tree's slots.
//
// One scale per block x of 32 dims of a (token, KV head) row, a = max |x|:
//   s = the smallest power of two with a <= 6 s, at least 2^-125 and at most
//   2^125; code = x / s (exact) to the nearest of 0, 1/2, 1, 3/2, 2, 3, 4 and 6,
//   ties to the even code; what lies beyond 6 s becomes 6 s
// The bounds keep every value that is read back (down to s / 2) a normal number
// of fp32 and bf16, so that the attention's products lose none of it.  A scale is
// a byte, the biased exponent of s.  A row that holds a NaN or an infinity has
// scales of 255 in all its blocks and codes 0: it reads back as NaN.
#include <type_traits>

#include "kvq_rows.h"
#include "tree.h"

namespace cdsl {

namespace {

constexpr unsigned kNoValue = 255;   // the scale of a row that is NaN

// Eight values of a row, which is read once: past the caches, so that the codes stay
// there (24 prompts of up to 2047 x 8 heads in bf16, written and read back: 55 -> 45 us;
// 16 of 256 x 32 in fp32: 62 -> 59).
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const bf16x8 t = __builtin_nontemporal_load((const bf16x8*)p);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)t[e];
  } else {
    const f32x4 t0 = __builtin_nontemporal_load((const f32x4*)p), t1 = __builtin_nontemporal_load((const f32x4*)(p + 4));
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = e < 4 ? t0[e & 3] : t1[e & 3];
  }
}

// The biased exponent of a block's scale, from the bits of its largest |x|: 6 =
// 1.5 * 2^2.
__device__ __forceinline__ unsigned fp4_scale(unsigned top) {
  const int e = (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x400000u ? 1 : 0);
  return (unsigned)min(max(e, 2), 252);
}

// Codes of eight values, the first in the lowest four bits.  The instruction
// divides by the scale, rounds to nearest even and saturates.
__device__ __forceinline__ unsigned encode8(const float (&x)[8], unsigned e) {
  const float s = __uint_as_float(e << 23);
  unsigned w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
}

// Eight values from their codes and scale (255: NaN, as the instruction has it).
template <typename T>
__device__ __forceinline__ void store8(T* o, unsigned w, unsigned e) {
  const float s = __uint_as_float(e << 23);
  if constexpr (sizeof(T) == 2) {
    union {
      bf16x2v p[4];
      u32x4 u;
    } y;
    y.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0);
    y.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1);
    y.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2);
    y.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3);
    *(u32x4*)o = y.u;
  } else {
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1);
    const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3);
    *(f32x4*)o = (f32x4){a[0], a[1], b[0], b[1]};
    *(f32x4*)(o + 4) = (f32x4){c[0], c[1], d[0], d[1]};
  }
}

// Threads of a workgroup: a task is four slots x eight dims of the keys or of the
// values, one a thread, so that its codes are whole words in both orders, a
// block of 32 dims is a quad of lanes and a row 4, 8 or 16 lanes.
template <int HD>
constexpr int fp4_threads() { return 2 * HD; }

// Workgroup = (page of the prompt's run, KV head, prompt).  The bytes bound it: 24
// prompts of up to 2047 x 8 heads of 128 in bf16 23 us for 101 MB in, half of them in
// the last cache when it is repeated, and 27 out.
template <int HD, typename T>
__global__ __launch_bounds__(fp4_threads<HD>()) void fp4_write_kernel(KvqView c, KvqRows r) {
  constexpr int NT = fp4_threads<HD>();
  constexpr int LQ = HD / 8;                 // lanes per quad of slots
  constexpr int CODES = 32 * HD, BYTES = fp4_unit_bytes(HD);
  __shared__ __attribute__((aligned(16))) uint8_t lds[BYTES];
  const int b = blockIdx.y, h = blockIdx.x % c.Hkv;
  const KvqRun run = kvq_run(r.start, r.count, r.T, b);
  const long long beg = run.beg, end = run.end;
  const long long page = kvq_first_page(run) + blockIdx.x / c.Hkv;
  const long long base = page * kPage;
  if (base >= end || base + kPage <= beg) return;
  uint8_t* unit = kvq_unit_of(c, b, page, h);
  if (!unit) return;
  const int isv = threadIdx.x / HD, slot = threadIdx.x % HD / LQ * 4, d = threadIdx.x % LQ * 8;
  const T* src = (const T*)(isv ? r.V : r.K) + (isv ? r.vsb : r.ksb) * b + h * HD + d;
  const long long ts = isv ? r.vst : r.kst;
  // whole pages go through LDS, so that their lines leave whole; of the others
  // only the run's bytes are written
  auto page_rows = [&](auto all) __attribute__((always_inline)) {
    constexpr bool WHOLE = decltype(all)::value;
    float x[4][8];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const long long pos = base + slot + t;
      if (WHOLE || (pos >= beg && pos < end)) load8<T>(src + (pos - beg) * ts, x[t]);
      else
#pragma unroll
        for (int e = 0; e < 8; ++e) x[t][e] = 0.f;
    }
    unsigned w[4], s[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      // the largest bit pattern of |x|: NaN and infinity stay on top
      unsigned a = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) a = max(a, __float_as_uint(x[t][e]) & 0x7fffffffu);
      a = max_moved<0xB1>(a);                              // quad_perm 1 0 3 2
      a = max_moved<0x4E>(a);                              // quad_perm 2 3 0 1
      s[t] = fp4_scale(a);
      if constexpr (LQ > 4) a = max_moved<0x141>(a);       // row_half_mirror
      if constexpr (LQ > 8) a = max_moved<0x140>(a);       // row_mirror
      w[t] = encode8(x[t], s[t]);
      const bool bad = a >= 0x7f800000u;
      s[t] = bad ? kNoValue : s[t];
      w[t] = bad ? 0u : w[t];
    }
    if constexpr (WHOLE) {
      unsigned o[4];
      if (isv) transpose4(w, o);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        if (isv) ((unsigned*)lds)[banked(fp4_value_at(HD, slot, d + 2 * t) / 4)] = o[t];
        else ((unsigned*)lds)[banked(fp4_key_at(HD, slot + t, d) / 4)] = w[t];
      }
      if (d % 32 == 0) {
        if (isv) *(unsigned*)(lds + fp4_value_scale_at(HD, slot, d)) = s[0] | s[1] << 8 | s[2] << 16 | s[3] << 24;
        else
#pragma unroll
          for (int t = 0; t < 4; ++t) lds[fp4_key_scale_at(HD, slot + t, d)] = (uint8_t)s[t];
      }
    } else {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        if (base + slot + t < beg || base + slot + t >= end) continue;
        if (!isv) *(unsigned*)(unit + fp4_key_at(HD, slot + t, d)) = w[t];
        else
#pragma unroll
          for (int e = 0; e < 4; ++e) unit[fp4_value_at(HD, slot + t, d + 2 * e)] = (uint8_t)(w[t] >> (8 * e));
        if (d % 32 == 0)
          unit[isv ? fp4_value_scale_at(HD, slot + t, d) : fp4_key_scale_at(HD, slot + t, d)] = (uint8_t)s[t];
      }
    }
  };
  if (base < beg || base + kPage > end) {   // uniform over the workgroup
    page_rows(std::false_type{});
    return;
  }
  page_rows(std::true_type{});
  __syncthreads();
  static_assert(CODES / 16 == NT, "a piece a thread");
  const int i = threadIdx.x;
  *((u32x4*)unit + i) = *(const u32x4*)&((const unsigned*)lds)[banked(4 * i)];
  if (i < (BYTES - CODES) / 16) *((u32x4*)(unit + CODES) + i) = *((const u32x4*)(lds + CODES) + i);
}

// Workgroup = (page of the prompt's run, KV head, prompt): the unit comes in as
// 16-byte pieces, the rows leave as whole lines.  Rows of a page outside the
// pool are NaN.  The same 24 prompts: 17 us for 98 MB out; the codes that come in are
// mostly in the last cache.
template <int HD, typename T>
__global__ __launch_bounds__(fp4_threads<HD>()) void fp4_read_kernel(KvqView c, KvqRows r) {
  constexpr int LQ = HD / 8;
  constexpr int CODES = 32 * HD, BYTES = fp4_unit_bytes(HD);
  __shared__ __attribute__((aligned(16))) uint8_t lds[BYTES];
  const int b = blockIdx.y, h = blockIdx.x % c.Hkv;
  const KvqRun run = kvq_run(r.start, r.count, r.T, b);
  const long long beg = run.beg, end = run.end;
  const long long page = kvq_first_page(run) + blockIdx.x / c.Hkv;
  const long long base = page * kPage;
  if (base >= end || base + kPage <= beg) return;
  const uint8_t* unit = kvq_unit_of(c, b, page, h);
  if (unit) {
    const int i = threadIdx.x;
    *(u32x4*)&((unsigned*)lds)[banked(4 * i)] = *((const u32x4*)unit + i);
    if (i < (BYTES - CODES) / 16) *((u32x4*)(lds + CODES) + i) = *((const u32x4*)(unit + CODES) + i);
  }
  __syncthreads();
  const int isv = threadIdx.x / HD, slot = threadIdx.x % HD / LQ * 4, d = threadIdx.x % LQ * 8;
  unsigned w[4] = {0u, 0u, 0u, 0u}, s[4] = {kNoValue, kNoValue, kNoValue, kNoValue};
  if (unit) {
    unsigned o[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      o[t] = ((const unsigned*)lds)[banked((isv ? fp4_value_at(HD, slot, d + 2 * t) : fp4_key_at(HD, slot + t, d)) / 4)];
      s[t] = lds[isv ? fp4_value_scale_at(HD, slot + t, d) : fp4_key_scale_at(HD, slot + t, d)];
    }
    if (isv) transpose4(o, w);
    else
#pragma unroll
      for (int t = 0; t < 4; ++t) w[t] = o[t];
  }
  T* dst = (T*)(isv ? r.Vo : r.Ko) + h * HD + d;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const long long pos = base + slot + t;
    if (pos >= beg && pos < end) store8<T>(dst + ((long long)b * r.T + (pos - beg)) * c.Hkv * HD, w[t], s[t]);
  }
}

// Moves of single tokens, as in the 8-bit cache: one wave per (layer, KV head,
// prompt), entry i of the path from slot L + path[i] to L + i, eight at a time
// read before any of them is written (path ascending: path[i] >= i, so no later
// entry's source has been written by then).  A token's keys are HD / 8 words; its
// values one byte in four, so that a lane reads the words around its dims and
// the eight entries' bytes go to at most three aligned groups of four slots.  (The
// page is the prompt's own from lens on, so the other bytes may be written back.)
template <int HD>
__global__ __launch_bounds__(64) void fp4_keep_kernel(KvqView c, long long layer_bytes, const int* lens,
                                                      const int* path, const int* n_path, int n, int* new_lens) {
  constexpr int CH = 8, W = fp4_pair(HD);
  constexpr int KL = HD / 8, TK = 64 / KL < CH ? 64 / KL : CH;   // lanes of a token's keys, tokens at once
  constexpr int VL = HD / (2 * W), TV = 64 / VL;                 // the same for values: a lane has W dim pairs
  constexpr int SL = HD / 16, TS = 64 / SL < CH ? 64 / SL : CH;  // and for scales, a byte a lane
  typedef unsigned Chunk __attribute__((ext_vector_type(2 * W)));   // [dim pair][half of the page]
  const int b = blockIdx.y, h = blockIdx.x % c.Hkv, layer = blockIdx.x / c.Hkv;
  const int lane = threadIdx.x;
  c.pool += layer * layer_bytes;
  const int L = max(lens[b], 0);
  const int m = min(max(n_path[b], 0), n);
  if (new_lens && blockIdx.x == 0 && lane == 0) new_lens[b] = (int)min((long long)L + m, 0x7fffffffll);
  // a lane's values in the group of four slots that holds `slot`
  auto values_at = [&](int slot) __attribute__((always_inline)) {
    const int x = lane % VL;
    return 16 * HD + x / 16 * 1024 + (slot % 16 / 4 * 16 + x % 16) * 8 * W;
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

    unsigned kr[CH / TK];
#pragma unroll
    for (int j = 0; j < CH / TK; ++j) {
      const int e = j * TK + lane / KL;   // (past the eighth: null)
      const uint8_t* s = ptr_of_lane(src, e);
      const int slot = __shfl(ss, e, 64);
      if (s) kr[j] = *(const unsigned*)(s + fp4_key_at(HD, slot, lane % KL * 8));
    }
    // a token's scales: of the keys' blocks, then of the values'
    auto scale_at = [&](int slot) __attribute__((always_inline)) {
      const int x = lane % SL;
      return x < SL / 2 ? fp4_key_scale_at(HD, slot, 32 * x) : fp4_value_scale_at(HD, slot, 32 * (x - SL / 2));
    };
    uint8_t sc[CH / TS];
#pragma unroll
    for (int j = 0; j < CH / TS; ++j) {
      const int e = j * TS + lane / SL;
      const uint8_t* s = ptr_of_lane(src, e);
      const int slot = __shfl(ss, e, 64);
      if (s) sc[j] = s[scale_at(slot)];
    }
    Chunk vr[CH / TV];
#pragma unroll
    for (int j = 0; j < CH / TV; ++j) {
      const int e = j * TV + lane / VL;
      const uint8_t* s = ptr_of_lane(src, e);
      const int slot = __shfl(ss, e, 64);
      vr[j] = s ? *(const Chunk*)(s + values_at(slot)) : (Chunk)0u;
    }
    // byte e: entry e's value, of each dim pair
    unsigned long long got[W] = {};
#pragma unroll
    for (int j = 0; j < CH / TV; ++j) {
      const int e = j * TV + lane / VL;
      const int slot = __shfl(ss, e, 64);
#pragma unroll
      for (int k = 0; k < W; ++k)
        got[k] |= (unsigned long long)((slot & 16 ? vr[j][2 * k + 1] : vr[j][2 * k]) >> (8 * (slot & 3)) & 255u) << (8 * e);
    }
#pragma unroll
    for (int o = VL; o < 64; o <<= 1)
#pragma unroll
      for (int k = 0; k < W; ++k) got[k] |= (unsigned long long)__shfl_xor((long long)got[k], o, 64);
    // the moved entries' bytes
    unsigned long long mask = 0;
#pragma unroll
    for (int e = 0; e < CH; ++e) mask |= moved >> e & 1u ? 255ull << (8 * e) : 0ull;
    // their word in group k of four slots: bytes 4 k - off .. + 3
    auto group = [&](unsigned long long w, int k) __attribute__((always_inline)) {
      return k == 0 ? (unsigned)w << (8 * off) : k == 1 ? (unsigned)(w >> (32 - 8 * off))
                                                        : off ? (unsigned)(w >> (64 - 8 * off)) : 0u;
    };
    Chunk old[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const uint8_t* d = ptr_of_lane(dst, CH + k);
      const int slot = __shfl(ds, CH + k, 64);
      if (lane < VL && group(mask, k)) old[k] = *(const Chunk*)(d + values_at(slot));
    }

#pragma unroll
    for (int j = 0; j < CH / TK; ++j) {
      const int e = j * TK + lane / KL;
      const bool live = ptr_of_lane(src, e) != nullptr;
      uint8_t* d = ptr_of_lane(dst, e);
      const int slot = __shfl(ds, e, 64);
      if (live) *(unsigned*)(d + fp4_key_at(HD, slot, lane % KL * 8)) = kr[j];
    }
#pragma unroll
    for (int j = 0; j < CH / TS; ++j) {
      const int e = j * TS + lane / SL;
      const bool live = ptr_of_lane(src, e) != nullptr;
      uint8_t* d = ptr_of_lane(dst, e);
      const int slot = __shfl(ds, e, 64);
      if (live) d[scale_at(slot)] = sc[j];
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      uint8_t* d = ptr_of_lane(dst, CH + k);
      const int slot = __shfl(ds, CH + k, 64);
      const unsigned on = group(mask, k);
      if (lane < VL && on) {
        Chunk w = old[k];
#pragma unroll
        for (int u = 0; u < W; ++u) {
          const unsigned x = group(got[u], k);
          if (slot & 16) w[2 * u + 1] = (w[2 * u + 1] & ~on) | (x & on);
          else w[2 * u] = (w[2 * u] & ~on) | (x & on);
        }
        *(Chunk*)(d + values_at(slot)) = w;
      }
    }
  }
}

template <int HD>
hipError_t fp4_rows(const KvqView& c, const KvqRows& r, bool write, hipStream_t st) {
  const dim3 grid((unsigned)(kvq_run_pages(r.T) * c.Hkv), (unsigned)c.B);
  constexpr int NT = fp4_threads<HD>();
  if (write) {
    if (r.dtype == 1) fp4_write_kernel<HD, bf16><<<grid, NT, 0, st>>>(c, r);
    else fp4_write_kernel<HD, float><<<grid, NT, 0, st>>>(c, r);
  } else {
    if (r.dtype == 1) fp4_read_kernel<HD, bf16><<<grid, NT, 0, st>>>(c, r);
    else fp4_read_kernel<HD, float><<<grid, NT, 0, st>>>(c, r);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t fp4_rows_launch(const KvqView& c, const KvqRows& r, bool write, hipStream_t st) {
  switch (c.hd) {
    case 32: return fp4_rows<32>(c, r, write, st);
    case 64: return fp4_rows<64>(c, r, write, st);
    case 128: return fp4_rows<128>(c, r, write, st);
  }
  return hipErrorInvalidValue;
}

hipError_t fp4_keep_launch(const KvqView& c, int n_layers, long long layer_bytes, const int* lens, const int* path,
                           const int* n_path, int n, int* new_lens, hipStream_t st) {
  const dim3 grid((unsigned)(n_layers * c.Hkv), (unsigned)c.B);
  switch (c.hd) {
    case 32: fp4_keep_kernel<32><<<grid, 64, 0, st>>>(c, layer_bytes, lens, path, n_path, n, new_lens); break;
    case 64: fp4_keep_kernel<64><<<grid, 64, 0, st>>>(c, layer_bytes, lens, path, n_path, n, new_lens); break;
    case 128: fp4_keep_kernel<128><<<grid, 64, 0, st>>>(c, layer_bytes, lens, path, n_path, n, new_lens); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace cdsl

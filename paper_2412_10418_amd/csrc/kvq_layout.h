// The 8-bit and 4-bit paged cache: where its bytes stand, which page a position
// lies on, and which slots of a page a node sees.  Plain C++ without HIP headers,
// so that it also builds as host-only code for unit tests under the address
// and undefined-behaviour sanitizers.
//
// A unit is one (layer, page, KV head) of the cache: the codes of 32 keys,
// the codes of 32 values, 32 key scales and 32 value scales.  Codes stand in
// the order in which a wave's lanes take them as MFMA operands, so that the
// attention reads 1 KB runs, 16 bytes a lane, and moves nothing between
// lanes:
//   keys    [dim / 32][(dim % 32) / 8][slot % 16][slot / 16][dim % 8]
//   values  [dim / 32][(slot % 16) / 4][dim % 16][(dim % 32) / 16][slot / 16][slot % 4]
// In 4 bits a unit holds the codes of 32 keys, those of 32 values, a byte of
// scale for every 32 dims of a key, and the same of the values.  A byte of codes
// is two dims of one token (the even one in the lower half), so that no two
// tokens share a byte, and 64 dims fill a lane's 16 bytes (heads of 32 dims: its
// 8).  With lane = (dim % 32) / 8 * 16 + slot % 16 for keys, and (slot % 16) / 4 *
// 16 + dim % 32 / 2 for values:
//   keys          [dim / 64][lane][dim / 32 % 2][slot / 16][dim % 8 / 2]
//   values        [dim / 64][lane][dim / 32 % 2][slot / 16][slot % 4]
//   key scales    [dim / 64][slot % 16][dim / 32 % 2][slot / 16]
//   value scales  [dim / 64][(slot % 16) / 4][dim / 32 % 2][slot / 16][slot % 4]
#pragma once

#include <stdint.h>

#if defined(__HIPCC__)
#define CDSL_KVQ_HD __host__ __device__ inline
#else
#define CDSL_KVQ_HD inline
#endif

namespace cdsl {

constexpr int kPage = 32;
enum KvqFormat { kInt8 = 0, kE4M3 = 1, kMxfp4 = 4 };

CDSL_KVQ_HD constexpr int kvq_unit_bytes(int hd) { return 2 * kPage * hd + 8 * kPage; }   // 8-bit formats
CDSL_KVQ_HD constexpr int fp4_unit_bytes(int hd) { return 34 * hd; }
CDSL_KVQ_HD constexpr int kvq_unit_bytes(int hd, int format) {
  return format == kMxfp4 ? fp4_unit_bytes(hd) : kvq_unit_bytes(hd);
}
CDSL_KVQ_HD constexpr int kvq_key_at(int slot, int dim) {
  return dim / 32 * 1024 + dim % 32 / 8 * 256 + slot % 16 * 16 + slot / 16 * 8 + dim % 8;
}
CDSL_KVQ_HD constexpr int kvq_value_at(int hd, int slot, int dim) {
  return kPage * hd + dim / 32 * 1024 + slot % 16 / 4 * 256 + dim % 16 * 16 + dim % 32 / 16 * 8 + slot / 16 * 4 +
         slot % 4;
}
CDSL_KVQ_HD constexpr int kvq_key_scale_at(int hd, int slot) { return 2 * kPage * hd + 4 * slot; }
CDSL_KVQ_HD constexpr int kvq_value_scale_at(int hd, int slot) { return 2 * kPage * hd + 4 * kPage + 4 * slot; }

// 4 bits.  Blocks of 32 dims that share a lane's bytes: two, one in heads of 32.
CDSL_KVQ_HD constexpr int fp4_pair(int hd) { return hd > 32 ? 2 : 1; }
// The byte of dims dim (even) and dim + 1 of a key or a value, and the scale of
// its block.
CDSL_KVQ_HD constexpr int fp4_key_at(int hd, int slot, int dim) {
  return dim / 64 * 1024 + (dim % 32 / 8 * 16 + slot % 16) * 8 * fp4_pair(hd) + dim / 32 % 2 * 8 + slot / 16 * 4 +
         dim % 8 / 2;
}
CDSL_KVQ_HD constexpr int fp4_value_at(int hd, int slot, int dim) {
  return 16 * hd + dim / 64 * 1024 + (slot % 16 / 4 * 16 + dim % 32 / 2) * 8 * fp4_pair(hd) + dim / 32 % 2 * 8 +
         slot / 16 * 4 + slot % 4;
}
CDSL_KVQ_HD constexpr int fp4_key_scale_at(int hd, int slot, int dim) {
  return 32 * hd + dim / 64 * 64 + slot % 16 * 2 * fp4_pair(hd) + dim / 32 % 2 * 2 + slot / 16;
}
CDSL_KVQ_HD constexpr int fp4_value_scale_at(int hd, int slot, int dim) {
  return 33 * hd + dim / 64 * 64 + slot % 16 / 4 * 8 * fp4_pair(hd) + dim / 32 % 2 * 8 + slot / 16 * 4 + slot % 4;
}

struct KvqView {
  uint8_t* pool;           // base of the layer (keep: of layer 0)
  const int* table;        // [B][table_stride] page ids
  int B, table_stride, pages, Hkv, hd, format;
};

// Unit of logical page p of prompt b and KV head h; null for a page beyond
// the table or an id outside the pool.
CDSL_KVQ_HD uint8_t* kvq_unit_of(const KvqView& c, int b, long long p, int h) {
  if (p < 0 || p >= c.table_stride) return nullptr;
  const int id = c.table[(long long)b * c.table_stride + p];
  if (id < 0 || id >= c.pages) return nullptr;
  return c.pool + ((long long)id * c.Hkv + h) * kvq_unit_bytes(c.hd, c.format);
}

// Positions [beg, end) of prompt b's run of T rows (null: from 0, all T).
struct KvqRun {
  long long beg, end;
};
CDSL_KVQ_HD KvqRun kvq_run(const int* start, const int* count, int T, int b) {
  KvqRun r;
  r.beg = start ? start[b] : 0;
  const int n = count ? count[b] : T;
  r.end = r.beg + (n < 0 ? 0 : n < T ? n : T);
  return r;
}
// First page of a run, and how many pages a run of T rows touches at most.
CDSL_KVQ_HD long long kvq_first_page(const KvqRun& r) { return (r.beg >= 0 ? r.beg : r.beg - (kPage - 1)) / kPage; }
CDSL_KVQ_HD int kvq_run_pages(int T) { return T / kPage + (T % kPage ? 1 : 0) + 1; }

// Bit s of the result: whether slot s of a page is visible to a node.  i0 =
// page * 32 - L is the node in the page's slot 0 (negative: so many prompt
// tokens come first).  Chain: the nodes up to `node`.  Tree: the nodes
// whose bit is set in `mask`, kTreeMax bits and a word of zeros behind.
constexpr int kTreeMax = 512;            // nodes of a tree with parents
constexpr int kTreeWords = kTreeMax / 32 + 1;
CDSL_KVQ_HD uint32_t slots_of_chain(int i0, int node) {
  const int last = node - i0;   // the node's slot
  return last >= 31 ? ~0u : last < 0 ? 0u : (2u << last) - 1u;
}
CDSL_KVQ_HD uint32_t slots_of_tree(int i0, const uint32_t* mask) {
  if (i0 <= -kPage) return ~0u;
  if (i0 < 0) return (mask[0] << -i0) | ((1u << -i0) - 1u);
  const uint64_t w = (uint64_t)mask[(i0 >> 5) + 1] << 32 | mask[i0 >> 5];
  return (uint32_t)(w >> (i0 & 31));
}

}  // namespace cdsl

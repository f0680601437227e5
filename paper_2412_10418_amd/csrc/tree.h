// Internal interface of the 8-bit paged cache (kvq.hip), the attention of a
// token tree over it (tree_attention.h, an instance file per head dimension) and
// the tree's verification (tree_accept.hip).
#pragma once
#include "common.h"
#include "kvq_layout.h"
#include "tree_plan.h"

namespace cdsl {

struct KvqRows {
  const void* K;           // write: [B][T][Hkv][hd] with the strides below
  const void* V;
  void* Ko;                // read: contiguous
  void* Vo;
  int dtype, T;
  long long ksb, kst, vsb, vst;
  const int* start;        // null: 0
  const int* count;        // null: T
};

hipError_t kvq_write_launch(const KvqView& c, const KvqRows& r, hipStream_t st);
hipError_t kvq_read_launch(const KvqView& c, const KvqRows& r, hipStream_t st);
hipError_t kvq_keep_launch(const KvqView& c, int n_layers, long long layer_bytes, const int* lens, const int* path,
                           const int* n_path, int n, int* new_lens, hipStream_t st);

struct TreeAttnArgs {
  KvqView c;
  const void* q;
  long long qsb, qst;
  void* out;               // [B][n][H][hd]
  const int* lens;
  const int* n_nodes;      // null: n
  const int* parents;      // null: causal
  int n, H, G;
  float scale_log2;        // softmax scale * log2(e)
  float* part_o;           // [slots][n * H][hd]
  float* part_ml;          // [slots][n * H][2]
  int slots, row_groups;   // key splits of all prompts (B: no splits)
  int split_pages;         // pages per key split, at least
  int wg_tiles;            // row tiles (of 16) per workgroup
};

hipError_t tree_attn_launch(TreeAttnArgs a, const TreeAttnPlan& p, int dtype, void* workspace, hipStream_t st);

constexpr int kAcceptMaxVocab = 1 << 20;

size_t tree_accept_workspace(int B, int n, int V);
hipError_t tree_accept_launch(const float* p, const float* q, int B, int n, int V, const int* tokens,
                              const int* parents, const int* n_nodes, const float* u, const float* v, int replace,
                              int* path, int* n_path, int* next_token, void* workspace, hipStream_t st);

}  // namespace cdsl

/*
 * cdsl_ops.h -- kernel-level entry points of the CDSL library.
 *
 * The first part exports single kernels of the step: exactly those that
 * cdsl_rollout / cdsl_verify launch, on caller buffers.  The second part
 * (from cdsl_kvq on) serves callers that hold their own paged cache and draft
 * trees of tokens rather than chains: an 8-bit cache, the attention of a tree
 * over it, the tree's verification and the move of its accepted path.
 * All pointers are device pointers owned by the caller; calls are
 * asynchronous on `stream` (a hipStream_t, NULL = default stream) and return
 * CDSL_OK or a negative CDSL_E* code (see cdsl.h).  No call allocates.
 */
#ifndef CDSL_OPS_H
#define CDSL_OPS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
  CDSL_EPI_STORE = 0,     /* C[M,N] (fp32)  = A * B^T                 */
  CDSL_EPI_RESIDUAL = 1   /* C[M,N] (fp32) += A * B^T  (residual add)   */
};

/* Bytes of workspace cdsl_op_gemm needs for this shape: for bf16 weights
 * the hi / lo planes of A, then the fp32 partial planes of a split K; 0 if
 * none. */
size_t cdsl_op_gemm_workspace(int32_t M, int32_t N, int32_t K, int32_t dtype);

/* Dense projection C = A[M,K] * B[N,K]^T with fp32 accumulation: the
 * contraction of every linear layer of the decoders (q/k/v/o, gate/up/down,
 * LM head).  A (activations) is fp32; B (weights) is bf16 (dtype
 * CDSL_BF16: A is split into bf16 hi + lo halves, two MFMA products, so the
 * result keeps fp32-level accuracy) or fp32 (CDSL_F32); C is fp32.  K must
 * be a multiple of 32 for bf16 (16 for fp32).  The workspace must hold
 * cdsl_op_gemm_workspace(M, N, K, dtype) bytes; every call writes what it
 * reads there, so it needs no initial contents.  Errors: EINVAL. */
int cdsl_op_gemm(const void* A, const void* B, float* C, int32_t M, int32_t N,
                 int32_t K, int32_t dtype, int32_t epilogue, void* workspace,
                 size_t workspace_bytes, void* stream);

/* cdsl_op_gemm for callers that cannot allocate device memory (code under
 * HIP graph capture, serving loops, harnesses that forbid allocation): the
 * same kernels, with the workspace taken from a scratch array the library
 * holds in device memory, CDSL_OP_GEMM_STATIC_BYTES (64 MiB) on each GPU it
 * runs on, until the process ends.  No allocation happens in the call.
 * Shapes whose hi / lo planes of A (4 M K bytes, bf16 weights only) exceed
 * that size are refused with ERANGE.  The planes of a K split get what is
 * left: results are cdsl_op_gemm's, bit for bit, where cdsl_op_gemm_workspace
 * fits (e.g. M = 500, N = 22016, K = 4096: 8 MB), and otherwise those of a
 * smaller split, as accurate (e.g. 716 x 2830 x 12000, whose own split needs
 * 87 MB).  Every call on one GPU shares that GPU's array: calls that overlap
 * on one GPU (two streams, two threads) race and must be serialised by the
 * caller.  The first call on a device looks up that device's copy of the
 * array.  Errors: EINVAL, ERANGE, EDEVICE. */
#define CDSL_OP_GEMM_STATIC_BYTES (64u << 20)
int cdsl_op_gemm_static(const void* A, const void* B, float* C, int32_t M,
                        int32_t N, int32_t K, int32_t dtype, int32_t epilogue,
                        void* stream);

/* Row statistics of logits[M, V] (fp32), one pass per row, never writing
 * probabilities: for row m,
 *   lp[m]        = logits[m, gather[m]] - logsumexp(logits[m, :])
 *                  (skipped, lp untouched, if gather is NULL)
 *   amax[m]      = argmax (lowest id on ties)
 *   topk_ids[m, 0..kk), topk_lp[m, 0..kk): the kk largest entries, value
 *                  descending then id ascending, as log-probs
 *                  (skipped if kk == 0; kk <= 16)
 * This is the log-softmax + gather + argmax + top-k step of verification.
 * Errors: EINVAL. */
int cdsl_op_logit_rows(const float* logits, int32_t M, int32_t V,
                       const int32_t* gather, int32_t kk, float* lp,
                       int32_t* amax, int32_t* topk_ids, float* topk_lp,
                       void* stream);

/* The LM head with its row statistics fused into the GEMM epilogue: the
 * same outputs as cdsl_op_logit_rows on logits = A[M,K] * B[V,K]^T
 * (cdsl_op_gemm's operands and dtypes; argmax and top-k ids identical, the
 * log-probs equal up to the summation order of the logsumexp), without the
 * logits ever reaching memory.  Each column tile of the GEMM reduces its
 * rows to (max, sum of exp, argmax, its kk best, the gathered value); one
 * workgroup per row folds the tiles.  amax may be NULL.  The workspace must
 * hold cdsl_op_lm_head_rows_workspace(M, V, K, dtype, kk) bytes (0 means
 * the shape is not covered).  Errors: EINVAL. */
size_t cdsl_op_lm_head_rows_workspace(int32_t M, int32_t V, int32_t K,
                                      int32_t dtype, int32_t kk);
int cdsl_op_lm_head_rows(const float* A, const void* B, int32_t M, int32_t V,
                         int32_t K, int32_t dtype, const int32_t* gather,
                         int32_t kk, float* lp, int32_t* amax,
                         int32_t* topk_ids, float* topk_lp, void* workspace,
                         size_t workspace_bytes, void* stream);

/* Speculative sampling rows (Sec. 3.2.2) over target_logits[M, V] (p) and
 * draft_logits[M, V] (q), fp32, rows ordered (row group g, position j) with
 * M = G * d; the row's draft token is x = lookaheads[g, j + 1] (an int32
 * [G, d + 1] array, as cdsl_rollout writes it).  For row m = g * d + j:
 *   draft_lp[m] = log q(x)
 *   res_ids[m]  = the draw at v[m] in [0, 1) from w = max(0, p - q) / Z:
 *                 the smallest token t with w_0 + ... + w_t > v[m] * Z
 *                 (argmax p, lowest id, when Z = 0)
 *   res_lp[m]   = log p(res_ids[m]).
 * This is the kernel cdsl_verify_soft runs after the verification pass.
 * Errors: EINVAL (null pointers, M not a multiple of d). */
int cdsl_op_soft_rows(const float* target_logits, const float* draft_logits,
                      int32_t M, int32_t V, int32_t d, const int32_t* lookaheads,
                      const float* v, float* draft_lp, int32_t* res_ids,
                      float* res_lp, void* stream);

/* ---- A drafted tree served from an 8-bit paged cache ----
 *
 * The cache holds keys and values in 8 bits, a scale per token and KV head
 * (fp32): 2 * head_dim + 8 bytes a token and head, where the step's own cache
 * (fp32 values) takes 8 * head_dim.  Pages hold CDSL_KVQ_PAGE tokens; token
 * position x of prompt b lies on page table[b][x / 32], slot x % 32.  One
 * step over trees of drafted tokens is
 *   cdsl_op_kvq_write       the nodes' keys and values, per layer
 *   cdsl_op_tree_attention  the nodes' attention, per layer
 *   cdsl_op_tree_accept     which nodes the target keeps, and the next token
 *   cdsl_op_kvq_keep        the kept nodes to the front, all layers
 * A single token is a tree of one node (decoding); without parents the nodes
 * are a chain, the causal chunk of a prompt.  Keys carry their rotary
 * embedding already; node m stands at cache position lens[b] + m whatever its
 * depth.
 *
 * Scales and codes of a row x of head_dim values with a = max |x|:
 *   CDSL_KVQ_INT8   s = max(a / 127, 2^-126); code = x / s to the nearest
 *                   integer, ties to even
 *   CDSL_KVQ_E4M3   s = the smallest power of two with a <= 448 s, at least
 *                   2^-126; code = x / s to the nearest e4m3, ties to even
 * and the value is code * s.  A row with a NaN or an infinity has s = NaN: it
 * reads back as NaN, and rows that see it attend to NaN.
 *
 * Page ids are not checked on the host.  A position beyond the table, below
 * 0, or on a page id outside [0, pages) is never accessed: it is not written,
 * reads as NaN, makes the attention rows that see it NaN, and is not moved.
 * Prompts may share pages that they only read.  Pointers and the strides of
 * rows (in bytes) must be multiples of 16.  Calls check their arguments on
 * the host before they launch; they allocate nothing, keep nothing between
 * calls, and may be captured into a graph.  Calls may run at once on several
 * streams if none writes what another uses (workspaces included). */
#define CDSL_KVQ_PAGE 32
#define CDSL_TREE_MAX 512          /* nodes of a tree that has parents */
#define CDSL_ACCEPT_MAX_VOCAB (1 << 20)
enum { CDSL_KVQ_INT8 = 0, CDSL_KVQ_E4M3 = 1 };

typedef struct cdsl_kvq {
  void* pool;            /* device, cdsl_op_kvq_pool_bytes; needs no initial contents */
  const int32_t* table;  /* device [batch][table_stride] page ids */
  int32_t n_layers;
  int32_t pages;         /* pages per layer */
  int32_t n_kv_heads;
  int32_t head_dim;      /* 32, 64 or 128 */
  int32_t batch;         /* prompts (<= 65535) */
  int32_t table_stride;  /* pages per prompt (< 2^26) */
  int32_t format;        /* CDSL_KVQ_INT8 or CDSL_KVQ_E4M3 */
} cdsl_kvq;

/* Bytes of the pool: n_layers * pages * n_kv_heads units of
 * 64 * head_dim + 256 bytes, laid out [layer][page][head].  0 for arguments
 * out of range and pools of 2^62 bytes or more. */
size_t cdsl_op_kvq_pool_bytes(int32_t n_layers, int32_t pages,
                              int32_t n_kv_heads, int32_t head_dim);

/* Quantises rows into a layer of the cache.  K and V are
 * [batch][T][n_kv_heads][head_dim] of dtype CDSL_F32 or CDSL_BF16, heads and
 * dims contiguous, prompts and tokens k_stride_b / k_stride_t (v_...)
 * elements apart.  Token t of prompt b, t < count[b] (NULL: T; clamped to
 * 0..T), goes to position start[b] + t (NULL: 0 + t).  All other slots keep
 * their contents, also those of the same page.  Two rows of one call must
 * not go to the same slot of the same page.  Errors: EINVAL, ERANGE,
 * EDEVICE. */
int cdsl_op_kvq_write(const cdsl_kvq* cache, int32_t layer, const void* K,
                      const void* V, int32_t dtype, int32_t T,
                      int64_t k_stride_b, int64_t k_stride_t,
                      int64_t v_stride_b, int64_t v_stride_t,
                      const int32_t* start, const int32_t* count,
                      void* stream);

/* Reads rows back: K and V ([batch][T][n_kv_heads][head_dim], contiguous,
 * dtype CDSL_F32 or CDSL_BF16) receive position start[b] + t for t <
 * count[b]; the rows behind are left as they were.  Errors: EINVAL, ERANGE,
 * EDEVICE. */
int cdsl_op_kvq_read(const cdsl_kvq* cache, int32_t layer, void* K, void* V,
                     int32_t dtype, int32_t T, const int32_t* start,
                     const int32_t* count, void* stream);

/* Attention of n nodes per prompt over a layer of the cache.  Q is
 * [batch][n][H][head_dim] (CDSL_F32 or CDSL_BF16, heads and dims contiguous,
 * prompts and nodes q_stride_b / q_stride_t elements apart), out the same
 * shape and type, contiguous, not overlapping Q.  Node m < n_nodes[b] (NULL:
 * n; clamped to 0..n) of prompt b sees positions [0, lens[b]), itself (at
 * lens[b] + m) and, with parents [batch][n], the nodes above it: parents[b][m]
 * in [0, m), anything else ends the way up.  parents NULL: all nodes up to m.
 * A length below 0 counts as 0.  Query head h reads KV head h / (H /
 * n_kv_heads).  scale multiplies q . k before the softmax.  Rows of nodes from
 * n_nodes[b] on are left as they were.  A prompt whose lens[b] + n_nodes[b] its
 * table cannot hold gets NaN rows.
 * Products, sums and softmax statistics are those of fp32, but for the
 * probabilities of a bf16 call, which are rounded to bf16 (to twice its bits
 * where n * H / n_kv_heads is 16 or less), and for entries of Q below 2^-15
 * (bf16: 2^-31) of their row's largest, which are off by up to 2^-39 of that.
 * They overflow as in fp32, before the division by the sum of the probabilities
 * (the largest of which counts 1 to 2^8) and with rows of Q scaled to entries
 * below 2: keys, and values times the number of keys, stay below 2^119.
 * max_len: a bound on lens, known to the host; it only decides how the keys
 * are split over the chip (0: not known, as for short prompts).  The
 * workspace must hold cdsl_op_tree_attention_workspace bytes for the same
 * arguments (0: none needed, or arguments that the call refuses); it needs no
 * initial contents.  Results do not depend on other calls, and the same
 * arguments give the same bits.  Errors: EINVAL, ERANGE (n beyond
 * CDSL_TREE_MAX with parents, batch * n * H of 2^24 or more), EDEVICE. */
size_t cdsl_op_tree_attention_workspace(int32_t batch, int32_t n, int32_t H,
                                        int32_t n_kv_heads, int32_t head_dim,
                                        int32_t max_len);
int cdsl_op_tree_attention(const cdsl_kvq* cache, int32_t layer, const void* Q,
                           int32_t dtype, int32_t n, int32_t H,
                           int64_t q_stride_b, int64_t q_stride_t,
                           const int32_t* lens, const int32_t* n_nodes,
                           const int32_t* parents, float scale,
                           int32_t max_len, void* out, void* workspace,
                           size_t workspace_bytes, void* stream);

/* Verification of drafted trees (speculative sampling, Sec. 3.2.2, over a
 * tree).  Node 0 of a prompt is its last committed token; nodes j >= 1 are
 * drafted tokens, tokens[b][j], under parents[b][j] in [0, j).  target_probs
 * and draft_probs [batch][n][V] (fp32, contiguous; temperature and
 * truncation are the caller's) hold in row j the target's and the draft's
 * distribution after node j; both rows are read at the tokens of all their
 * children, and whole where the walk ends (the target's) and where a child of
 * their node is rejected.  From the node reached (0 at first) with rows p and q,
 * its children are tested in index order: child j with token x is kept when
 *   u[b][j] * q_r(x) <= P_r(x) and P_r(x) > 0
 * and becomes the node reached; otherwise P_{r+1} = max(0, P_r - q_r)
 * divided by its sum.  P_0 = p.  q_r = q when the children are independent
 * draws (replace != 0), or q without the tokens rejected so far, divided by
 * what is left of 1 (replace = 0: drawn without replacement; children are
 * passed over once nothing is left).  When no child is left, next_token[b]
 * is the smallest token t with P_r(0) + ... + P_r(t) > v[b] * (sum of P_r), or
 * -1 if p has no mass.  If a rejection leaves no mass, no further child is
 * tested and next_token[b] is argmax p, the lowest id of the largest: 0 where p
 * has no mass itself but a child was there to be rejected.  For a sum that is
 * not finite it is -1.  Sums and tests are in fp64.  path[b][0..n_path[b]) are
 * the nodes reached from 0 on (path[b][0] = 0), the rest of path [batch][n] is
 * -1.  n_nodes (NULL: n) is clamped to 1..n.  A child whose token is outside
 * [0, V), or whose parent is outside [0, j), is passed over.  u [batch][n] and
 * v [batch] are uniforms in [0, 1).  The workspace must hold cdsl_op_tree_accept_workspace bytes (0:
 * none needed); it needs no initial contents.  Errors: EINVAL, ERANGE (batch
 * beyond 65535, n beyond CDSL_TREE_MAX, V beyond CDSL_ACCEPT_MAX_VOCAB),
 * EDEVICE. */
size_t cdsl_op_tree_accept_workspace(int32_t batch, int32_t n, int32_t V);
int cdsl_op_tree_accept(const float* target_probs, const float* draft_probs,
                        int32_t batch, int32_t n, int32_t V,
                        const int32_t* tokens, const int32_t* parents,
                        const int32_t* n_nodes, const float* u, const float* v,
                        int32_t replace, int32_t* path, int32_t* n_path,
                        int32_t* next_token, void* workspace,
                        size_t workspace_bytes, void* stream);

/* Keeps a path of each prompt's tree: in every layer, the entry at position
 * lens[b] + path[b][i] moves to lens[b] + i, i < n_path[b] (clamped to
 * 0..n).  path [batch][n] holds ascending nodes in [0, CDSL_TREE_MAX), as
 * cdsl_op_tree_accept writes it (or only its first n columns).  new_lens[b]
 * (NULL: not wanted; no part of lens, n_path or path) receives lens[b] +
 * n_path[b], or 2^31 - 1 if that is more.  A length below 0 counts as 0.  The
 * prompts' pages from the one with position lens[b] on must be their own.
 * Errors: EINVAL, ERANGE, EDEVICE. */
int cdsl_op_kvq_keep(const cdsl_kvq* cache, const int32_t* lens,
                     const int32_t* path, const int32_t* n_path, int32_t n,
                     int32_t* new_lens, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* CDSL_OPS_H */

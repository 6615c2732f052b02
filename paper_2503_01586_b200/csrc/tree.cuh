// What the kernels of elitekv_attend_tree share.
#pragma once

#include "common.cuh"

// Lengths of a sequence as every kernel of the call sees them: n cached tokens (clamped to what the cache holds and to
// 0), the last `nodes` of them the tree's.
struct TreeLens {
  int n, nodes;
  bool bad;
};
__device__ __forceinline__ TreeLens tree_lens(const int32_t* seq_lens, const int32_t* n_nodes, int b, int m, long long max_len) {
  TreeLens t;
  const long long n = seq_lens[b], k = n_nodes ? n_nodes[b] : m;
  t.n = (int)(n < 0 ? 0 : n > max_len ? max_len : n);
  t.nodes = (int)(k < 0 ? 0 : k > m ? m : k);
  if (t.nodes > t.n) t.nodes = t.n;
  t.bad = t.n != n || t.nodes != k;
  return t;
}

struct TreeCall {
  const void *q_rope, *q_abs;
  const int32_t *seq_lens, *n_nodes;
  const uint64_t* mask;
  int B, m;
  void* workspace;
  void* out;
};

// Items (partial results) of the combine that follows: seq_first [B+1], part_ml, part_acc [item][m][n_h][vw]
size_t ekv_tree_generic_bytes(const elitekv_layer* L, int B, int m);
int ekv_launch_tree_generic(const elitekv_layer* L, const elitekv_cache* cache, const CacheView& cv, const TreeCall& c, cudaStream_t st);

size_t ekv_tree_tc_bytes(const elitekv_layer* L, int B, int m);
int ekv_tree_tc_supported(const elitekv_layer* L, int B, int m, const CacheView* cv);      // cv may be null: shape alone
int ekv_launch_tree_tc(const elitekv_layer* L, const elitekv_cache* cache, const CacheView& cv, const TreeCall& c, cudaStream_t st);

// A node is a query row of the two-pass decode kernel (csrc/decode_tc.cu): small calls of few nodes
size_t ekv_tree_rows_bytes(const elitekv_layer* L, int B, int m);      // 0: never
int ekv_launch_tree_rows(const elitekv_layer* L, const elitekv_cache* cache, const TreeCall& c, size_t workspace_bytes, cudaStream_t st);

// Greedy acceptance of a tree of drafted tokens, and the cache rows of the accepted branch.
//
// With parent(i) < i (-1: the node follows the committed tokens), draft[i] the drafted token, chosen[i] the
// model's choice after node i and first the choice after the committed tokens, the accepted branch is
//   i_0 = lowest i with parent(i) = -1 and draft[i] = first,   i_k+1 = lowest i with parent(i) = i_k and
//   draft[i] = chosen[i_k]
// Node i_k lies in cache row held + i_k, was rotated at position held + k (its depth), and from now on is the
// sequence's token held + k: its row moves there, bit for bit.  The paper has no counterpart.
//
// Bound: latency (a walk of up to 64 steps in one warp's registers, then a few KB to move).  Block per sequence; a
// thread owns columns of the rows and moves them in the order of the branch, eight rows in flight: i_k >= k, so that
// a row is read before anything lands in its place, and no other thread touches the column.
#include "common.cuh"

namespace {

constexpr int kAccThreads = 256;
constexpr int kAccAhead = 8;

struct AccArgs {
  const int32_t *held, *n_nodes, *parent, *draft, *first, *chosen;
  int32_t *n_accepted, *path, *token, *held_out;
  unsigned char *rope, *latent;
  CacheView cv;
  int m;
  long long rope_bytes, lat_bytes;
  int32_t* status;
};

// columns of one plane, in units of V
template <class V>
__device__ __forceinline__ void move_rows(unsigned char* plane, long long row_bytes, const long long* src, const long long* dst, int n) {
  const int units = (int)(row_bytes / (long long)sizeof(V));
  for (int u = threadIdx.x; u < units; u += kAccThreads) {
    for (int k0 = 0; k0 < n; k0 += kAccAhead) {
      V v[kAccAhead];
#pragma unroll
      for (int e = 0; e < kAccAhead; ++e)
        if (k0 + e < n) v[e] = ((const V*)(plane + src[k0 + e] * row_bytes))[u];
#pragma unroll
      for (int e = 0; e < kAccAhead; ++e)
        if (k0 + e < n) ((V*)(plane + dst[k0 + e] * row_bytes))[u] = v[e];
    }
  }
}

__global__ void __launch_bounds__(kAccThreads)
accept_tree_kernel(const AccArgs a) {
  __shared__ long long s_src[ELITEKV_MAX_TREE_NODES], s_dst[ELITEKV_MAX_TREE_NODES];
  __shared__ int s_path[ELITEKV_MAX_TREE_NODES];
  __shared__ int s_moves;
  const int b = blockIdx.x, lane = threadIdx.x & 31;
  ekv_pdl_wait();
  ekv_pdl_trigger();
  if (threadIdx.x < 32) {
    const int held = a.held[b];
    const int n = min(max(a.n_nodes ? a.n_nodes[b] : a.m, 0), a.m);
    int up[2], tok[2], next[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int i = lane + 32 * e;
      up[e] = -2;                       // matches nothing
      tok[e] = next[e] = 0;
      if (i < n) {
        const long long x = (long long)b * a.m + i;
        const int p = a.parent ? a.parent[x] : i - 1;
        up[e] = p >= 0 && p < i ? p : -1;
        tok[e] = a.draft[x];
        next[e] = a.chosen[x];
      }
    }
    int at = -1, want = a.first[b], count = 0;
    for (int k = 0; k < n; ++k) {
      const unsigned lo = __ballot_sync(0xffffffffu, up[0] == at && tok[0] == want);
      const unsigned hi = __ballot_sync(0xffffffffu, up[1] == at && tok[1] == want);
      if ((lo | hi) == 0) break;
      at = lo ? __ffs(lo) - 1 : 31 + __ffs(hi);
      const int w0 = __shfl_sync(0xffffffffu, next[0], at & 31), w1 = __shfl_sync(0xffffffffu, next[1], at & 31);
      want = at < 32 ? w0 : w1;
      if (lane == 0) s_path[count] = at;
      ++count;
    }
    __syncwarp();
    // the moves: accepted nodes that are not in place already
    int moves = 0;
    for (int k0 = 0; k0 < a.m; k0 += 32) {
      const int k = k0 + lane;
      const int i = k < count ? s_path[k] : -1;
      long long src = -1, dst = -1;
      if (k < count && i != k) {
        int code, detail;
        src = ekv_token_row(a.cv, b, held + i, &code, &detail);
        if (src >= 0) dst = ekv_token_row(a.cv, b, held + k, &code, &detail);
        if (dst < 0) ekv_record(a.status, code, b, detail);
      }
      const unsigned on = __ballot_sync(0xffffffffu, dst >= 0);
      if (dst >= 0) {
        const int at2 = moves + __popc(on & ((1u << lane) - 1u));
        s_src[at2] = src;
        s_dst[at2] = dst;
      }
      moves += __popc(on);
      if (k < a.m) a.path[(long long)b * a.m + k] = i;
    }
    if (lane == 0) {
      s_moves = moves;
      a.n_accepted[b] = count;
      a.token[b] = want;
      a.held_out[b] = held + count;
    }
  }
  __syncthreads();
  const int n = s_moves;
  if (n == 0) return;
  move_rows<uint4>(a.latent, a.lat_bytes, s_src, s_dst, n);
  if ((a.rope_bytes & 15) == 0)
    move_rows<uint4>(a.rope, a.rope_bytes, s_src, s_dst, n);
  else
    move_rows<uint32_t>(a.rope, a.rope_bytes, s_src, s_dst, n);
}

}  // namespace

extern "C" int elitekv_accept_tree(const elitekv_layer* L, const elitekv_cache* cache, const int32_t* held, const int32_t* n_nodes,
                                   const int32_t* parent, const int32_t* draft, const int32_t* first, const int32_t* chosen,
                                   int32_t B, int32_t m, int32_t* n_accepted, int32_t* path, int32_t* token, int32_t* held_out,
                                   elitekv_stream_t stream) {
  if (!L || !cache || B <= 0 || B > cache->n_seqs || m < 1 || m > ELITEKV_MAX_TREE_NODES) return ELITEKV_ERR_INVALID_ARG;
  if (!held || !draft || !first || !chosen || !n_accepted || !path || !token || !held_out) return ELITEKV_ERR_INVALID_ARG;
  if (!ekv_on_device(L)) return ELITEKV_ERR_INVALID_ARG;
  AccArgs a;
  int rc = ekv_make_view(cache, &a.cv);
  if (rc != ELITEKV_OK) return rc;
  a.held = held;
  a.n_nodes = n_nodes;
  a.parent = parent;
  a.draft = draft;
  a.first = first;
  a.chosen = chosen;
  a.n_accepted = n_accepted;
  a.path = path;
  a.token = token;
  a.held_out = held_out;
  a.rope = (unsigned char*)cache->rope;
  a.latent = (unsigned char*)cache->latent;
  a.m = m;
  a.rope_bytes = (long long)L->n_h * L->r * 4;
  a.lat_bytes = (long long)L->d_c * 2;
  a.status = L->d_status;
  EKV_CUDA_OK(ekv_launch_pdl(accept_tree_kernel, dim3((unsigned)B), dim3(kAccThreads), 0, (cudaStream_t)stream, a));
  EKV_CUDA_OK(cudaGetLastError());
  return ELITEKV_OK;
}

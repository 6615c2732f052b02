// Attention of a tree of drafted tokens over the cache: entry points and the kernel for any shape.
//
//   s[i,h,t] = scale (q_rope[i,h] . k_rope[t,h] + q_abs[i,h] . c[t]),   p = softmax over the tokens that node i sees,
//   acc[i,h] = sum_t p c[t]   (W_uv follows in the combine, csrc/combine.cu)
//
// Node i sees every committed token (t < n - nodes) and the nodes j of its mask (t = n - nodes + j).
//
// tree_generic_kernel: a warp per (sequence, node, head) and split of the tokens.  Lanes hold the latent axis, eight
// coordinates at a time, of four tokens; queries and the running sum (fp32) lie in shared memory.  Tokens that the row does
// not see are skipped: nothing of theirs is read.  Bound: the trips to L2 of four tokens in turn, a row's own read of the
// whole cache.  It serves what the tensor-core form does not cover, and calls so small that that form's start costs more.
#include "tree.cuh"

namespace {

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

constexpr int kDecodeGeneric = 1;     // elitekv_decode_plan_info
constexpr int kAhead = 4;             // tokens of a warp in flight
constexpr int kSplits = 32;           // partial results of a row, at most

struct GenArgs {
  const bf16 *q_rope, *q_abs, *rope, *latent;
  const int32_t *seq_lens, *n_nodes;
  const uint64_t* mask;
  CacheView cv;
  int B, m, n_h, r2, d_c, kw, voff, vw, splits;
  long long max_len;
  float scale_log2e;
  float *part_acc, *part_ml;
  int32_t *seq_first, *counters, *status;
  int n_counters;
};

// the items of the combine and its counters; lengths that do not fit are recorded once
__global__ void tree_generic_prep_kernel(const GenArgs a) {
  ekv_pdl_wait();
  ekv_pdl_trigger();
  const long long t = (long long)blockIdx.x * blockDim.x + threadIdx.x, step = (long long)gridDim.x * blockDim.x;
  for (long long b = t; b <= a.B; b += step) {
    a.seq_first[b] = (int)b * a.splits;
    if (b < a.B && tree_lens(a.seq_lens, a.n_nodes, (int)b, a.m, a.max_len).bad)
      ekv_record(a.status, ELITEKV_ERR_BAD_POSITION, (int)b, a.seq_lens[b]);
  }
  for (long long k = t; k < a.n_counters; k += step) a.counters[k] = 0;
}

__global__ void tree_generic_kernel(const GenArgs a) {
  extern __shared__ float s_row[];
  const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float* const s_q = s_row + (size_t)warp * (a.kw + a.vw);      // scaled by nothing: bf16 values as floats
  float* const s_acc = s_q + a.kw;
  const long long rows = (long long)a.B * a.m * a.n_h, row = (long long)blockIdx.x * warps + warp;
  const int split = blockIdx.y;
  ekv_pdl_wait();
  ekv_pdl_trigger();
  if (row >= rows) return;
  const int h = (int)(row % a.n_h), i = (int)(row / a.n_h % a.m), b = (int)(row / a.n_h / a.m);
  const TreeLens len = tree_lens(a.seq_lens, a.n_nodes, b, a.m, a.max_len);
  const int per = (len.n + a.splits - 1) / a.splits;
  const int t0 = min(split * per, len.n), t1 = i < len.nodes ? min(t0 + per, len.n) : t0;
  const int prefix = len.n - len.nodes;
  const unsigned long long mask = i < len.nodes ? a.mask[(long long)b * a.m + i] : 0ull;
  for (int k = lane; k < a.kw; k += 32) s_q[k] = __bfloat162float(a.q_abs[row * a.kw + k]);
  for (int k = lane; k < a.vw; k += 32) s_acc[k] = 0.f;
  __syncwarp();
  float m_run = -1e30f, l_run = 0.f;
  auto unpack = [](const uint4& x, float* f) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 y = __bfloat1622float2(*(const bf162*)&w[e]);
      f[2 * e] = y.x;
      f[2 * e + 1] = y.y;
    }
  };
  for (int t = t0; t < t1; t += kAhead) {
    bool seen[kAhead];
    const bf16* c[kAhead];
    const bf16* kr[kAhead];
    float s[kAhead];
#pragma unroll
    for (int g = 0; g < kAhead; ++g) {
      const int tg = t + g;
      seen[g] = tg < t1 && (tg < prefix || (mask >> (tg - prefix) & 1));
      s[g] = 0.f;
      long long at = 0;
      if (seen[g]) {
        int code, detail;
        at = ekv_token_row(a.cv, b, tg, &code, &detail);
        if (at < 0) {
          if (lane == 0) ekv_record(a.status, code, b, detail);
          at = 0;                                  // page 0, as in the other attention kernels
        }
      }
      c[g] = a.latent + at * a.d_c;
      kr[g] = a.rope + (at * a.n_h + h) * a.r2;
    }
    for (int k = lane * 8; k < a.kw; k += 256) {
      uint4 x[kAhead];
#pragma unroll
      for (int g = 0; g < kAhead; ++g) x[g] = seen[g] ? __ldg((const uint4*)(c[g] + k)) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int g = 0; g < kAhead; ++g) {
        float f[8];
        unpack(x[g], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[g] = fmaf(f[e], s_q[k + e], s[g]);
      }
    }
    for (int k = lane; k < a.r2; k += 32) {
      const float q = __bfloat162float(a.q_rope[row * a.r2 + k]);
#pragma unroll
      for (int g = 0; g < kAhead; ++g)
        if (seen[g]) s[g] = fmaf(q, __bfloat162float(kr[g][k]), s[g]);
    }
    float m_new = m_run;
#pragma unroll
    for (int g = 0; g < kAhead; ++g) {
      s[g] = warp_sum(s[g]) * a.scale_log2e;
      if (seen[g]) m_new = fmaxf(m_new, s[g]);
    }
    const float corr = exp2f(m_run - m_new);
    m_run = m_new;
    l_run *= corr;
    float p[kAhead];
#pragma unroll
    for (int g = 0; g < kAhead; ++g) {
      p[g] = seen[g] ? exp2f(s[g] - m_new) : 0.f;
      l_run += p[g];
    }
    for (int k = lane * 8; k < a.vw; k += 256) {
      uint4 x[kAhead];
#pragma unroll
      for (int g = 0; g < kAhead; ++g) x[g] = seen[g] ? __ldg((const uint4*)(c[g] + a.voff + k)) : make_uint4(0, 0, 0, 0);
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = s_acc[k + e] * corr;
#pragma unroll
      for (int g = 0; g < kAhead; ++g) {
        float f[8];
        unpack(x[g], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = fmaf(p[g], f[e], y[e]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) s_acc[k + e] = y[e];
    }
  }
  __syncwarp();
  const long long item = (long long)b * a.splits + split, at = (item * a.m + i) * a.n_h + h;
  for (int k = lane; k < a.vw; k += 32) a.part_acc[at * a.vw + k] = s_acc[k];
  if (lane == 0) {
    a.part_ml[at * 2] = m_run;
    a.part_ml[at * 2 + 1] = l_run;
  }
}

// How many tokens a single node sees: they are the first ones of its sequence.
__global__ void tree_single_kernel(const int32_t* seq_lens, const int32_t* n_nodes, const uint64_t* mask, int B, long long max_len, int32_t* lens,
                                   int32_t* status) {
  ekv_pdl_wait();
  ekv_pdl_trigger();
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b >= B) return;
  const TreeLens t = tree_lens(seq_lens, n_nodes, b, 1, max_len);
  if (t.bad) ekv_record(status, ELITEKV_ERR_BAD_POSITION, b, seq_lens[b]);
  lens[b] = t.nodes == 0 ? 0 : t.n - 1 + (int)(mask[b] & 1);
}
inline size_t lens_bytes(int B) { return align256(sizeof(int32_t) * (size_t)B); }

// Splits: enough warps for the device
int generic_splits(const elitekv_layer* L, int B, int m) {
  const long long rows = (long long)B * m * L->n_h, want = 16ll * L->sm_count;
  const long long s = (want + rows - 1) / rows;
  return (int)(s > kSplits ? kSplits : s);
}

// Whether a call is so small that the generic kernel is the quicker one.  Its time is the groups of kAhead tokens that
// a warp takes in turn, each a few trips to L2 and shuffles (about 2 us) and its share of the row; that of the
// tensor-core form hardly depends on so little work (30 to 52 us).  Measured, generic and tensor-core in us, by groups:
// rows of 64 latents 1: 15/32, 3: 24/32, 5: 25 to 30/32 to 35, 7: 25 to 31/30, 10: 46/36; of 768, 1: 20/43, 3: 40/48;
// of 1536, 1: 27 to 30/50, 2: 46/52, 3: 53/52.  The tokens are the capacity of the cache, since the lengths are on the device.
// Where nodes can be query rows of the decode kernel (tree_rows_fit; 33, 25 us), a second group is too many.
bool tree_is_small(const elitekv_layer* L, int B, int m, long long max_len, bool rows_fit) {
  if ((long long)B * m * L->n_h > 16ll * L->sm_count) return false;
  const int splits = generic_splits(L, B, m);
  const long long groups = ((max_len + splits - 1) / splits + kAhead - 1) / kAhead;
  return groups * (2048 + L->kw + L->vw) <= (rows_fit ? 6144 : 12288);
}

// Whether few enough nodes and tokens for the decode kernel, in which every node reads the cache for itself: 20 us less
// to begin with, and then a time that grows with nodes x tokens and, by 0.3 us, with nodes x sequences.  Measured, that kernel
// and the tree's own in us, by the sum below in millions: 7B, two nodes over 40 tokens (6) 33/51, 4 x 1000, 4 nodes (66) 45/60,
// 8 x 2000, 2 (115) 63/78, 4 x 1000, 8 (131) 61/62, 1 x 6000, 8 (155) 61/72, 1 x 3000, 16 (164) 62/59, 2 x 8000, 4 (205)
// 78/82, 16 x 256, 8 (235) 93/72; 13B, 4 x 1000, 4 (157) 60/69, 1 x 8000, 4 (254) 86/74; 87.5 %, 1 x 6000, 8 (82) 41/78,
// 32 x 100, 8 (307) 73/69; S-LRD, 32 x 512, 2 (117) 57/70, 1 x 4000, 16 (115) 56/52, 16 x 256, 8 (184) 69/57.
bool tree_rows_fit(const elitekv_layer* L, const elitekv_cache* cache, const CacheView& cv, int B, int m) {
  if (ekv_tree_rows_bytes(L, B, m) == 0 || !ekv_tc_supported(L, cache)) return false;
  long long tokens = cv.max_ctx;
  if (tokens > 1 << 20 || B > 1 << 10) return false;
  tokens *= B;
  if (cv.page_table && ((long long)cv.num_pages << cv.page_shift) < tokens) tokens = (long long)cv.num_pages << cv.page_shift;
  const int blocks = m * (L->sm_count / ekv_tc_workers(L, 1));          // that read the cache
  return blocks * (tokens * (L->kw + L->vw) + ((long long)B << 20)) <= 170000000;
}

struct GenCarve {
  size_t first, ml, acc, slice, cnt, total;
};
GenCarve generic_carve(const elitekv_layer* L, int B, int m) {
  // (rows x splits is at most this, which grows with B and m as the splits, rounded, do not)
  const size_t rows = (size_t)B * m * L->n_h, most = rows + 16 * (size_t)L->sm_count, parts = rows * kSplits < most ? rows * kSplits : most;
  GenCarve c;
  size_t o = 0;
  c.first = o; o = align256(o + sizeof(int32_t) * ((size_t)B + 1));
  c.ml = o;    o = align256(o + sizeof(float) * 2 * parts);
  c.acc = o;   o = align256(o + sizeof(float) * parts * L->vw);
  c.slice = o; o = align256(o + ekv_combine_scratch_bytes(L, B) * m);
  c.cnt = o;   o = align256(o + sizeof(int32_t) * (size_t)ekv_combine_counters(L, B) * m);
  c.total = o;
  return c;
}

}  // namespace

size_t ekv_tree_generic_bytes(const elitekv_layer* L, int B, int m) { return generic_carve(L, B, m).total; }

int ekv_launch_tree_generic(const elitekv_layer* L, const elitekv_cache* cache, const CacheView& cv, const TreeCall& c, cudaStream_t st) {
  const GenCarve w = generic_carve(L, c.B, c.m);
  unsigned char* const base = (unsigned char*)c.workspace;
  const size_t per_warp = sizeof(float) * ((size_t)L->kw + L->vw);
  int warps = 8;
  while (warps > 1 && per_warp * warps > (size_t)L->smem_optin) warps >>= 1;
  if (per_warp * warps > (size_t)L->smem_optin) return ELITEKV_ERR_UNSUPPORTED_SHAPE;
  GenArgs a;
  a.q_rope = (const bf16*)c.q_rope;
  a.q_abs = (const bf16*)c.q_abs;
  a.rope = (const bf16*)cache->rope;
  a.latent = (const bf16*)cache->latent;
  a.seq_lens = c.seq_lens;
  a.n_nodes = c.n_nodes;
  a.mask = c.mask;
  a.cv = cv;
  a.B = c.B;
  a.m = c.m;
  a.n_h = L->n_h;
  a.r2 = 2 * L->r;
  a.d_c = L->d_c;
  a.kw = L->kw;
  a.voff = L->voff;
  a.vw = L->vw;
  a.splits = generic_splits(L, c.B, c.m);
  a.max_len = cv.max_ctx;
  a.scale_log2e = L->scale * 1.4426950408889634f;
  a.part_acc = (float*)(base + w.acc);
  a.part_ml = (float*)(base + w.ml);
  a.seq_first = (int32_t*)(base + w.first);
  a.counters = (int32_t*)(base + w.cnt);
  a.n_counters = ekv_combine_counters(L, c.B) * c.m;
  a.status = L->d_status;
  const int n_prep = c.B + 1 > a.n_counters ? c.B + 1 : a.n_counters;
  const int prep_blocks = (n_prep + 255) / 256;
  EKV_CUDA_OK(ekv_launch_pdl(tree_generic_prep_kernel, dim3(prep_blocks < 64 ? prep_blocks : 64), dim3(256), 0, st, a));
  const long long rows = (long long)c.B * c.m * L->n_h, blocks = (rows + warps - 1) / warps;
  if (blocks > 0x7fffffffll) return ELITEKV_ERR_UNSUPPORTED_SHAPE;
  EKV_CUDA_OK(ekv_allow_smem(tree_generic_kernel, per_warp * warps));
  EKV_CUDA_OK(ekv_launch_pdl(tree_generic_kernel, dim3((unsigned)blocks, (unsigned)a.splits), dim3(32 * warps), per_warp * warps, st, a));
  DecodeScratch ws = {};
  ws.rows = c.m;
  ws.seq_first = a.seq_first;
  ws.part_ml = a.part_ml;
  ws.part_acc = a.part_acc;
  ws.slice_out = (float*)(base + w.slice);
  ws.counters = a.counters;
  return ekv_launch_combine(L, c.B, ws, c.out, st);
}

namespace {

// What a call of this size uses, whatever kernel the cache's layout leads to
size_t tree_need(const elitekv_layer* L, int B, int m) {
  const size_t g = ekv_tree_generic_bytes(L, B, m), t = ekv_tree_tc_supported(L, B, m, nullptr) ? ekv_tree_tc_bytes(L, B, m) : 0;
  const size_t r = ekv_tree_rows_bytes(L, B, m);
  size_t most = g > t ? g : t, d = 0;
  if (r > most) most = r;
  if (m == 1 && elitekv_decode_workspace_size(L, B, &d) == ELITEKV_OK && d + lens_bytes(B) > most) most = d + lens_bytes(B);
  return most;
}

}  // namespace

// Fewer nodes may need more (fewer row blocks are cut into more runs, another kernel serves them): the size is that of the
// largest tree and of all smaller ones.
extern "C" int elitekv_attend_tree_workspace_size(const elitekv_layer* L, int32_t B, int32_t m, size_t* bytes) {
  if (!L || !bytes || B <= 0 || m < 1 || m > ELITEKV_MAX_TREE_NODES) return ELITEKV_ERR_INVALID_ARG;
  *bytes = 0;
  for (int k = 1; k <= m; ++k) {
    const size_t n = tree_need(L, B, k);
    if (n > *bytes) *bytes = n;
  }
  return ELITEKV_OK;
}

extern "C" int elitekv_attend_tree(const elitekv_layer* L, const elitekv_cache* cache, const void* q_rope, const void* q_abs,
                                   const int32_t* seq_lens, const int32_t* n_nodes, const uint64_t* tree_mask, int32_t B, int32_t m,
                                   void* workspace, size_t workspace_bytes, void* out, elitekv_stream_t stream) {
  if (!L || !cache || !q_abs || !seq_lens || !tree_mask || !workspace || !out || (L->r > 0 && !q_rope)) return ELITEKV_ERR_INVALID_ARG;
  if (B <= 0 || B > cache->n_seqs || m < 1 || m > ELITEKV_MAX_TREE_NODES) return ELITEKV_ERR_INVALID_ARG;
  if (((uintptr_t)q_abs & 15) || ((uintptr_t)q_rope & 15) || ((uintptr_t)out & 3) || ((uintptr_t)tree_mask & 7) || !ekv_on_device(L))
    return ELITEKV_ERR_INVALID_ARG;
  CacheView cv;
  int rc = ekv_make_view(cache, &cv);
  if (rc != ELITEKV_OK) return rc;
  if (((uintptr_t)workspace & 255) || workspace_bytes < tree_need(L, B, m)) return ELITEKV_ERR_WORKSPACE_TOO_SMALL;
  const TreeCall c{q_rope, q_abs, seq_lens, n_nodes, tree_mask, B, m, workspace, out};
  const bool dense = ekv_tree_tc_supported(L, B, m, &cv) != 0;
  int32_t plan[5];
  if (m == 1 && elitekv_decode_plan_info(L, cache, B, plan) == ELITEKV_OK && (plan[0] != kDecodeGeneric || !dense)) {
    // One node: decoding over the tokens that it sees, which are the first ones.  (Not where decoding would be on its kernel for
    // any shape, which reads the cache head by head: pages of 32 tokens, 11 x 14418 of 13B: 9157 us, 301 here.)
    int32_t* const lens = (int32_t*)workspace;
    EKV_CUDA_OK(ekv_launch_pdl(tree_single_kernel, dim3((unsigned)((B + 255) / 256)), dim3(256), 0, (cudaStream_t)stream, seq_lens, n_nodes, tree_mask, B,
                               cv.max_ctx, lens, L->d_status));
    rc = elitekv_decode(L, cache, q_rope, q_abs, lens, B, (unsigned char*)workspace + lens_bytes(B), workspace_bytes - lens_bytes(B), out, stream);
    if (rc != ELITEKV_ERR_UNSUPPORTED_SHAPE) return rc;
  }
  const bool rows_fit = tree_rows_fit(L, cache, cv, B, m), small = tree_is_small(L, B, m, cv.max_ctx, rows_fit);
  if (rows_fit && !small) {
    rc = ekv_launch_tree_rows(L, cache, c, workspace_bytes, (cudaStream_t)stream);
    if (rc != ELITEKV_ERR_UNSUPPORTED_SHAPE) return rc;
  }
  if (dense && !small) return ekv_launch_tree_tc(L, cache, cv, c, (cudaStream_t)stream);
  return ekv_launch_tree_generic(L, cache, cv, c, (cudaStream_t)stream);
}

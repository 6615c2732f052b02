// Tables of a serving step, built on the device: page table, slot map, rotary positions, tree masks.
//
// From held[b] cached and fresh[b] new tokens per sequence (ps tokens a page):
//   need_b  = max(0, ceil((held_b + fresh_b) / ps) - pages_held_b)     pages taken off the free stack's top, in
//                                                                      order of sequences
//   slot    = page(held_b + i) ps + (held_b + i) mod ps                cache row of new token i
//   pos     = held_b + i, in a tree held_b + depth(i)                  siblings share a position, not a slot
//   mask_i  = bit i | mask_parent(i)                                   what a node sees of its tree
// The paper has no counterpart (it leaves the serving loop to the engine).
//
// Bound: latency; a few KB to 2 MB move.  One launch, no workspace and no order between blocks: every block sums
// the lengths of ALL sequences itself (B integers out of L2) instead of waiting for another block's sums, checks
// them, and fills its share of the outputs.  So all blocks agree on whether the step fits, and nothing is written
// to the page table when it does not.
#include "common.cuh"

namespace {

constexpr int kTabThreads = 256;
constexpr int kTabWarps = kTabThreads / 32;

struct TabArgs {
  elitekv_tables t;
  CacheView cv;
  int B, m;
  long long n_slots;
};

// the last index b with first[b] <= x (first[0] = 0, first[B] > x)
__device__ __forceinline__ int tab_find(const int* first, int B, int x) {
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// Masks of the nodes `lane` and `lane + 32` of a tree, by doubling: after k steps a mask holds the node's nearest
// 2^k - 1 ancestors beside itself, and `up` names the next one (-1: none).
__device__ __forceinline__ void tree_masks(int up0, int up1, int lane, unsigned long long* mask) {
  unsigned long long m0 = 1ull << lane, m1 = 1ull << (lane + 32);
#pragma unroll
  for (int k = 0; k < 6; ++k) {
    int nu[2];
    unsigned long long nm[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int up = e ? up1 : up0, src = up & 31;
      const unsigned long long a = __shfl_sync(0xffffffffu, m0, src), b = __shfl_sync(0xffffffffu, m1, src);
      const int ua = __shfl_sync(0xffffffffu, up0, src), ub = __shfl_sync(0xffffffffu, up1, src);
      nm[e] = up < 0 ? 0ull : up < 32 ? a : b;
      nu[e] = up < 0 ? -1 : up < 32 ? ua : ub;
    }
    m0 |= nm[0];
    m1 |= nm[1];
    up0 = nu[0];
    up1 = nu[1];
  }
  mask[0] = m0;
  mask[1] = m1;
}

__global__ void __launch_bounds__(kTabThreads)
step_tables_kernel(const TabArgs a) {
  extern __shared__ int s_tab[];               // first token [B+1], first new page [B+1]
  __shared__ long long s_sum[2][kTabWarps];
  __shared__ int s_bad;
  __shared__ unsigned s_page;                  // the smallest bad page id among those that new tokens go to, plus 1 (0: a negative one)
  int* const s_tok = s_tab;
  int* const s_pg = s_tab + a.B + 1;
  const elitekv_tables& t = a.t;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const bool paged = a.cv.page_table != nullptr;
  const int shift = a.cv.page_shift;
  const long long max_len = paged ? (long long)a.cv.max_pages_per_seq << shift : a.cv.max_ctx;
  constexpr int kNone = 0x7fffffff;             // no sequence
  constexpr unsigned kNoPage = 0xffffffffu;     // (any int32 may be a bad id, the largest as well)
  if (tid == 0) {
    s_bad = kNone;
    s_page = kNoPage;
  }
  ekv_pdl_wait();
  ekv_pdl_trigger();
  __syncthreads();

  // ---- sums over the sequences (64 bits: what does not fit 32 is refused below)
  long long tok0 = 0, pg0 = 0;
  for (int b0 = 0; b0 < a.B; b0 += kTabThreads) {
    const int b = b0 + tid;
    long long nt = 0, np = 0;
    if (b < a.B) {
      const long long held = t.held[b], fresh = t.fresh[b];
      const bool bad = held < 0 || fresh < 0 || held + fresh > max_len || held + fresh > 0x7fffffffll || (a.m > 0 && fresh > a.m);
      const long long ph = paged ? t.pages_held[b] : 0;
      if (bad || (paged && (ph < (held + a.cv.page_mask) >> shift || ph > a.cv.max_pages_per_seq))) {
        atomicMin(&s_bad, b);
      } else {
        nt = fresh;
        if (paged) {
          const long long end = (held + fresh + a.cv.page_mask) >> shift;
          np = end > ph ? end - ph : 0;
          // pages of the sequence's own that new tokens go to
          for (long long p = held >> shift; p < (end < ph ? end : ph) && fresh > 0; ++p) {
            const int id = t.page_table[(long long)b * a.cv.max_pages_per_seq + p];
            if (id < 0 || id >= a.cv.num_pages) atomicMin(&s_page, id < 0 ? 0u : (unsigned)id + 1u);
          }
        }
      }
    }
    // inclusive sums over the warp, then over the warps
    long long it = nt, ip = np;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long x = __shfl_up_sync(0xffffffffu, it, o), y = __shfl_up_sync(0xffffffffu, ip, o);
      if (lane >= o) { it += x; ip += y; }
    }
    if (lane == 31) { s_sum[0][warp] = it; s_sum[1][warp] = ip; }
    __syncthreads();
    long long bt = tok0, bp = pg0;
    for (int w = 0; w < kTabWarps; ++w) {
      if (w < warp) { bt += s_sum[0][w]; bp += s_sum[1][w]; }
      tok0 += s_sum[0][w];
      pg0 += s_sum[1][w];
    }
    if (b < a.B) { s_tok[b] = (int)(bt + it - nt); s_pg[b] = (int)(bp + ip - np); }
    __syncthreads();
  }
  if (tid == 0) { s_tok[a.B] = (int)tok0; s_pg[a.B] = (int)pg0; }

  // ---- does the step fit?  The same answer in every block.
  const int n_free = paged ? *t.n_free : 0;
  int status = ELITEKV_OK, detail = 0;
  if (s_bad != kNone) {
    status = ELITEKV_ERR_BAD_POSITION;
    detail = s_bad;
  } else if (tok0 > 0x7fffffffll || (a.m == 0 && tok0 > a.n_slots)) {
    status = ELITEKV_ERR_BAD_POSITION;
    detail = -1;
  } else if (paged && (n_free < 0 || n_free > a.cv.num_pages)) {
    status = ELITEKV_ERR_BAD_PAGE;
    detail = n_free;
  } else if (pg0 > n_free) {
    status = ELITEKV_ERR_NO_PAGES;
    detail = (int)(pg0 - n_free);
  } else {
    for (int k = tid; k < (int)pg0; k += kTabThreads) {
      const int id = t.free_pages[n_free - 1 - k];
      if (id < 0 || id >= a.cv.num_pages) atomicMin(&s_page, id < 0 ? 0u : (unsigned)id + 1u);
    }
  }
  __syncthreads();
  if (status == ELITEKV_OK && s_page != kNoPage) {
    status = ELITEKV_ERR_BAD_PAGE;
    detail = (int)(s_page - 1u);
  }
  const bool ok = status == ELITEKV_OK;

  const long long g0 = (long long)blockIdx.x * kTabThreads + tid, gs = (long long)gridDim.x * kTabThreads;
  // ---- per sequence and per new page
  for (long long b = g0; b < a.B; b += gs) {
    const int held = t.held[b];
    const int fresh = ok ? s_tok[b + 1] - s_tok[b] : 0;
    t.seq_lens[b] = held + fresh;
    t.first[b] = ok ? s_tok[b] : 0;
    if (t.granted) t.granted[b] = fresh;
    if (paged) t.pages_held_out[b] = t.pages_held[b] + (ok ? s_pg[b + 1] - s_pg[b] : 0);
  }
  if (g0 == 0) {
    t.first[a.B] = ok ? (int)tok0 : 0;
    if (paged) *t.n_free_out = ok ? n_free - (int)pg0 : n_free;
    t.result[0] = status;
    t.result[1] = ok ? (int)tok0 : 0;
    t.result[2] = ok ? (int)pg0 : 0;
    t.result[3] = detail;
  }
  if (ok)
    for (long long k = g0; k < pg0; k += gs) {
      const int b = tab_find(s_pg, a.B, (int)k);
      t.page_table[(long long)b * a.cv.max_pages_per_seq + t.pages_held[b] + ((int)k - s_pg[b])] = t.free_pages[n_free - 1 - (int)k];
    }

  // ---- per token
  auto slot_of = [&](int b, int held, int i) -> long long {
    const int p = held + i;
    if (!paged) return (long long)b * a.cv.max_ctx + p;
    const int pi = p >> shift, ph = t.pages_held[b];
    const int page = pi < ph ? t.page_table[(long long)b * a.cv.max_pages_per_seq + pi] : t.free_pages[n_free - 1 - (s_pg[b] + pi - ph)];
    return ((long long)page << shift) + (p & a.cv.page_mask);
  };
  if (a.m == 0) {
    for (long long x = g0; x < a.n_slots; x += gs) {
      int b = -1, p = 0;
      long long slot = -1;
      if (ok && x < tok0) {
        b = tab_find(s_tok, a.B, (int)x);
        const int held = t.held[b], i = (int)x - s_tok[b];
        p = held + i;
        slot = slot_of(b, held, i);
      }
      t.seq_id[x] = b;
      t.pos[x] = p;
      t.slot[x] = slot;
    }
    return;
  }
  // a warp per tree: nodes `lane` and `lane + 32`
  for (long long bb = (long long)blockIdx.x * kTabWarps + warp; bb < a.B; bb += (long long)gridDim.x * kTabWarps) {
    const int b = (int)bb, held = t.held[b], fresh = ok ? t.fresh[b] : 0;
    int up[2];
    unsigned long long mask[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int i = lane + 32 * e;
      int p = -1;
      if (i < fresh) p = t.parent ? t.parent[bb * a.m + i] : i - 1;
      up[e] = p >= 0 && p < i ? p : -1;
    }
    tree_masks(up[0], up[1], lane, mask);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int i = lane + 32 * e;
      if (i >= a.m) continue;
      const bool on = i < fresh;
      const long long x = bb * a.m + i;
      t.seq_id[x] = on ? b : -1;
      t.pos[x] = on ? held + __popcll(mask[e]) - 1 : 0;
      t.slot[x] = on ? slot_of(b, held, i) : -1;
      t.tree_mask[x] = on ? mask[e] : 0;
    }
  }
}

}  // namespace

extern "C" int elitekv_step_tables(const elitekv_cache* cache, const elitekv_tables* tables, int32_t B, int32_t m,
                                   int64_t n_slots, elitekv_stream_t stream) {
  if (!cache || !tables || B <= 0 || B > cache->n_seqs || m < 0 || m > ELITEKV_MAX_TREE_NODES || n_slots < 0)
    return ELITEKV_ERR_INVALID_ARG;
  if (B > ELITEKV_MAX_TABLE_SEQS) return ELITEKV_ERR_UNSUPPORTED_SHAPE;
  const elitekv_tables& t = *tables;
  if (!t.held || !t.fresh || !t.seq_lens || !t.first || !t.result) return ELITEKV_ERR_INVALID_ARG;
  if (n_slots > 0 && (!t.seq_id || !t.pos || !t.slot)) return ELITEKV_ERR_INVALID_ARG;
  if (m > 0 ? n_slots != (int64_t)B * m || !t.tree_mask : t.parent != nullptr) return ELITEKV_ERR_INVALID_ARG;
  if (((uintptr_t)t.slot & 7) || ((uintptr_t)t.tree_mask & 7)) return ELITEKV_ERR_INVALID_ARG;
  // inputs that every block reads are not written by any
  if (t.seq_lens == t.held || t.seq_lens == t.fresh || (t.granted && (t.granted == t.held || t.granted == t.fresh))) return ELITEKV_ERR_INVALID_ARG;
  TabArgs a;
  a.t = t;
  int rc = ekv_make_view(cache, &a.cv);
  if (rc != ELITEKV_OK) return rc;
  if (cache->page_table) {
    if (!t.page_table || t.page_table != cache->page_table || !t.pages_held || !t.free_pages || !t.n_free || !t.pages_held_out ||
        !t.n_free_out || t.pages_held_out == t.pages_held || t.n_free_out == t.n_free)
      return ELITEKV_ERR_INVALID_ARG;
  }
  a.B = B;
  a.m = m;
  a.n_slots = n_slots;
  // a thread per packed token and a warp per tree, up to a fixed cap (no layer here to ask for the device's SMs; 148 on B200):
  // every block reads all lengths
  const long long want = m > 0 ? (B + kTabWarps - 1) / kTabWarps : (n_slots + kTabThreads - 1) / kTabThreads;
  const unsigned blocks = (unsigned)(want < 1 ? 1 : want > 222 ? 222 : want);
  const size_t smem = sizeof(int) * 2 * ((size_t)B + 1);
  EKV_CUDA_OK(ekv_allow_smem(step_tables_kernel, smem));
  EKV_CUDA_OK(ekv_launch_pdl(step_tables_kernel, dim3(blocks), dim3(kTabThreads), smem, (cudaStream_t)stream, a));
  EKV_CUDA_OK(cudaGetLastError());
  return ELITEKV_OK;
}

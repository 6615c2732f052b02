// Attention of a tree of drafted tokens on the tensor cores (sm_100a: tcgen05, TMEM, TMA).
//
// All heads and nodes of a sequence read the same latent rows, so that one sequence is two dense products over its
// cached tokens:
//     S [rows x tokens]  = [Q_abs | Q_rope] [rows x (kw + rope)] . [C_k | K_rope]^T
//     O [rows x vw]      = P [rows x tokens] . C_v            P = 2^(S - ref), bf16
// with rows = heads x nodes, head by head.  The rope columns of a block's heads join the score product with zeros where
// row and column belong to different heads (the prep kernel lays the queries out so): 16 nodes of a 7B layer add 4 steps
// of 64 to 24 that way; on FP32 lanes in the epilogue they took 30 us a tile.
// From about five nodes on (7B, 75 %) they are bound by the tensor cores and by what L2 hands to the SMs, below that by
// the cache's bytes.  An O of 128 rows has 1536 columns, three times what TMEM holds, so the products are not fused in
// one block: P goes through L2, 2 bytes per row and token, which costs less than exchanging partial scores between
// blocks that split the latent axis, and both products are plain streams of operands.
//
// Work units, taken by persistent workers (a pair of blocks on 256 rows, or one block where 128 rows are enough) from
// ONE ordered list, by an atomic counter:
//     score unit  (piece, 256 tokens)           S tile over the whole kw, softmax terms, P tile to the ring in L2
//     value unit  (piece, 256 latent columns)   O tile over the piece's tokens, to the partial result
// A piece is (row block, up to kPiece tokens of a sequence).  The list interleaves the score units of piece j with the
// value units of piece j - D, so that P and the piece's cache rows are read again while L2 holds them.  A unit waits only
// for units before it in the list, and a worker that is not resident has claimed nothing: some resident worker can always
// go on, whatever else runs on the device.
//
// Softmax reference.  P is bf16 and O fp32: both have 8 exponent bits, so the reference of 2^(S - ref) only has to keep
// the exponents in range.  It is 0 while the largest score of (row, 256 tokens) is within 2^+-64, else a multiple of
// 64 near it (sums over n tokens then stay finite for latents below 2^64 / n).  All tiles of a row agree on it unless scores are extreme; the block that finishes a piece's last
// score unit looks, and brings P of rows that do not agree to the largest reference: a factor of a power of two, exact.
// The sums are of the rounded P, so that their rounding cancels where one token dominates.
//
// Pieces of one run add into the run's partial result in order (fp32, read and written by the owner of the value unit):
// results do not depend on scheduling, and the partial results' number does not grow with the context.  Runs are cut by the
// prep kernel, on the device, where the lengths are.
//
// A rope value that is not finite is its head's matter alone, but in the score product it meets the zeros of the other heads in its
// row block, and 0 times it is NaN.  So a block whose scores hold NaN looks at them one by one, and those of tokens with
// such values among the row block's rope columns are computed again on FP32 lanes from the row's own head.  A call without
// such values pays a look at the sums (0 to 0.6 %); 13B, 8 x 8192 tokens that all hold them, 32 nodes: 71 ms.
//
// Tokens that a row does not see: their scores are dropped by a select, P = 0.  In the value product 0 times a value that
// is not finite would spread it to every row, so the drafted tokens' rows (and the rest of the last 64 tokens) pass a
// warp that clears such values before the tensor core reads them, and notes the nodes: rows that see one become NaN.
//
// Every wait is bounded; when one runs out the block records ELITEKV_ERR_TIMEOUT and leaves.
#include "tc_ptx.cuh"
#include "tree.cuh"
#include "tree_steps.cuh"

namespace {

constexpr int kRows = 128;              // rows per block
constexpr int kTile = 256;              // tokens of a score unit, latent columns of a value unit
constexpr int kPiece = 2048;            // most tokens of a piece
constexpr int kTiles = kPiece / kTile;
constexpr int kSlots = 64;              // pieces in the ring
constexpr int kMostAhead = kSlots - 8;  // D at most
constexpr int kTreeThreads = 416;       // warp 0 loads queries and P, 1 MMA, 2 loads cache rows, 3 clears drafted rows, 4-11 epilogue, 12 claims units
constexpr int kEpiThreads = 128;         // a group of four epilogue warps
constexpr int kQueue = 4;               // two units with the epilogue groups, two ahead (more would be late for those that wait for them)
constexpr int kLead = 16;                // steps before a unit's last load at which the next unit is claimed
constexpr int kMaxStages = 5;
constexpr int kABytes = kRows * 128;
constexpr int kOutBytes = 8192;         // rows on their way out, per epilogue warp: two boxes of 32 rows x 128 bytes

enum { kScore = 0, kValue = 1, kStop = 2 };

struct TreeUnit {
  int kind, b, rb, tok0, len, idx, slot, gen, n, nodes, run, k, pad[4];      // 48 bytes are published; kind: type | layout << 8
};

// Trees of one call differ in size, and rows of padding nodes cost as much as others.  So row blocks come in layouts: heads of
// `m` nodes each, `hb` heads a block, `n_rb` row blocks, with n_rb at least a fifth smaller from one to the next.  A sequence
// has the last that holds its nodes.  (32 ragged sequences of 7B, trees of 7 to 13 nodes: 1035 -> 891 us; 16 of S-LRD, 34 to
// 64 nodes: 345 -> 316; where all are full, 0.1 to 0.5 us more.)
constexpr int kLayouts = 8;
struct TreeLayout {
  int m, hb, n_rb, n_rc;      // n_rc: 64-column steps that hold the rope columns of any row block
};
struct TreeLayouts {
  int n, tiles;               // tiles: [block][n_rc] of a sequence's spread queries, at most
  TreeLayout of[kLayouts];
};
__device__ __forceinline__ int tree_layout(const TreeLayouts& l, int nodes) {
  int k = 0;
  while (k + 1 < l.n && l.of[k + 1].m >= nodes) ++k;
  return k;
}
struct TreeQueryMaps {
  CUtensorMap of[kLayouts];
};

struct TreeTcArgs {
  CacheView cv;
  const bf16 *q_rope, *q_abs, *rope, *latent;      // (for scores that are computed again)
  const uint64_t* mask;
  TreeLayouts lay;
  int m, n_h, r2, kw, vw, d_c, n_rb, n_ct, box_s, box_v, v3;       // n_rb: of the first layout
  float scale_log2e;
  bf16* P;                    // [slot][CG][kPiece / 64][128][64]: what a step loads is one piece (4 KB from row to row: 655 clocks a
                              // step instead of 530)
  float2* stats;              // [slot][CG][tiles][128]: (reference, sum) of a row's tile
  float2* pref;               // [slot][CG][128]: the same of the piece
  float2* cstate;             // [run][rb][ct][CG][128]: of the run so far
  int *s_cnt, *ready, *v_done, *chain;
  float* part_acc;            // [run][rb][CG][vw / 64][128][64]
  float2* part_ml;            // [run][rb][CG][128]
  const int* hdr;             // [0] claim counter, [1] runs, [2] pieces (row blocks included), [3] D
  const int4* runs;           // [run][2], by pieces: (b, first token, tokens, pieces), (n, nodes, run, layout)
  int32_t* status;
};

struct __align__(16) TreeBars {        // (units behind it are written 16 bytes at a time)
  uint64_t full[kMaxStages], empty[kMaxStages], spec[kMaxStages], fixed[kMaxStages];
  uint64_t acc_full[2], acc_empty[2];
  uint64_t q_full[kQueue], q_empty[kQueue], go;
};

template <int CG>
struct TreeSmem {
  static constexpr int b_bytes = kTile / CG * 128;            // 256 (128) token rows, or 64 tokens of 256 (128) columns
  static constexpr int stage = kABytes + b_bytes;
  static constexpr int n_stages = CG == 2 ? 5 : 3;            // (one more: 0.5 % and 3 % with the epilogue's boxes at half their size)
  static constexpr int out = 8 * kOutBytes;
  static constexpr int misc = sizeof(TreeBars) + kQueue * sizeof(TreeUnit) + kQueue * 16 + 64;
  static constexpr int total = n_stages * stage + out + misc + 1024;
};

__device__ __forceinline__ int ld_acquire(const int* p) {
  int v;
  asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void add_release(int* p, int v) {
  asm volatile("red.release.gpu.global.add.s32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}
// generic and asynchronous accesses of global and shared memory, both ways
__device__ __forceinline__ void fence_proxy_all() { asm volatile("fence.proxy.async;" ::: "memory"); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// until *p has reached target (counters wrap nowhere near: a call's counts start at zero)
__device__ __forceinline__ bool poll_global(const int* p, int target, volatile int* abort_flag, int why) {
  for (unsigned i = 0; i < (1u << 22); ++i) {
    if (ld_acquire(p) >= target) return true;
    if ((i & 63) == 63 && *abort_flag) return false;
  }
  if (*abort_flag == 0) *abort_flag = why;
  return false;
}
// (the limit is some 0.6 s or more: a tile whose scores are all computed again takes milliseconds, and a wait may span several)
__device__ __forceinline__ bool warp_wait_cluster(uint32_t bar, uint32_t parity, volatile int* abort_flag, int why) {
  for (unsigned i = 0; i < kSpinLimit; ++i) {
    if (__any_sync(0xffffffffu, mbar_try_wait_cluster(bar, parity))) return true;
    if ((i & 1023) == 1023 && __any_sync(0xffffffffu, *abort_flag != 0)) return false;
  }
  if (*abort_flag == 0) *abort_flag = why;
  return false;
}
// cache row of token t of sequence b; a page outside the pool counts as page 0 (recorded where `status` is given)
__device__ __forceinline__ long long tree_row(const CacheView& cv, int b, int t, int32_t* status) {
  if (cv.page_table == nullptr) return (long long)b * cv.max_ctx + t;
  int page = cv.page_table[(long long)b * cv.max_pages_per_seq + (t >> cv.page_shift)];
  if (page < 0 || page >= cv.num_pages) {
    if (status) ekv_record(status, ELITEKV_ERR_BAD_PAGE, b, page);
    page = 0;
  }
  return ((long long)page << cv.page_shift) + (t & cv.page_mask);
}

// Whether one of eight bf16 values is not finite, and their product with eight others added to s
__device__ __forceinline__ bool any_not_finite(const uint4& x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  bool bad = false;
#pragma unroll
  for (int e = 0; e < 4; ++e) bad |= (w[e] & 0x7f80u) == 0x7f80u || (w[e] & 0x7f800000u) == 0x7f800000u;
  return bad;
}
__device__ __forceinline__ float dot8(const uint4& x, const uint4& y, float s) {
  const uint32_t v[4] = {x.x, x.y, x.z, x.w}, w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    s = fmaf(__uint_as_float(v[e] << 16), __uint_as_float(w[e] << 16), s);
    s = fmaf(__uint_as_float(v[e] & 0xffff0000u), __uint_as_float(w[e] & 0xffff0000u), s);
  }
  return s;
}

// first rope column that a row block's score product takes: of its first head, on a 16-byte boundary
__host__ __device__ __forceinline__ int tree_rope_col(int h0, int r2) { return h0 * r2 & ~7; }

// The list of units, walked forward: block j of the list holds the score units of piece j and the value units of
// piece j - D.  Pieces are ordered by their place in their run, then by run, then by row block, so that the pieces of a
// run, which add into one partial result in turn, are far apart.  The runs are sorted by their number of pieces: those with
// a k-th piece are the list's first (up to kBins, from where on the list is searched).
constexpr int kBins = 256;
struct PieceWalk {
  int p, at, k, rb;           // piece; run (place in the list), piece of the run, row block
  int4 r, r2;                 // (b, first token, tokens, pieces), (n, nodes, run, layout)
};
__device__ __forceinline__ void walk_load(PieceWalk& w, const TreeTcArgs& a) {
  w.r = a.runs[2 * w.at];
  w.r2 = a.runs[2 * w.at + 1];
}
__device__ __forceinline__ void walk_next(PieceWalk& w, const TreeTcArgs& a, int n_runs, int n_pieces) {
  if (++w.p >= n_pieces) return;
  if (++w.rb < a.lay.of[w.r2.w].n_rb) return;
  w.rb = 0;
  do {
    if (++w.at >= n_runs) { w.at = 0; ++w.k; }
    walk_load(w, a);
    if (w.r.w <= w.k && w.r.w < kBins) { w.at = 0; ++w.k; walk_load(w, a); }
  } while (w.r.w <= w.k);
}
__device__ __forceinline__ int walk_len(const PieceWalk& w) { return min(kPiece, w.r.z - w.k * kPiece); }

// A warp's scores of tokens t0 .. t0 + tokens - 1 that are NaN for another head's rope values (columns [x0, x0 + cols) are
// the row block's): computed again, into the tile.  Whether there was one.  Eight tokens at a time share a lane's read of its query
// (13B, 8 x 8192 tokens that all need it, 32 nodes: 71 ms; one at a time 236).  (A function of its own: inline it cost the kernel 80 bytes of spilled registers.)
__device__ __noinline__ bool mend_scores(const TreeTcArgs& a, uint32_t tm, int b, int h, int i, int t0, int tokens, int prefix,
                                         unsigned long long mask, bool active, int x0, int cols) {
  constexpr int kMend = 8;
  const int lane = threadIdx.x & 31;
  const long long row = ((long long)b * a.m + i) * a.n_h + h;
  bool any = false;
#pragma unroll 1
  for (int t = 0; t < tokens; t += kMend) {
    float v[kMend], s[kMend];
    int at[kMend];                         // cache rows (box coordinates: below 2^31)
    unsigned redo = 0, mine = 0;           // tokens to compute again: of any lane, of this one
    tc_ld8(tm + t, v);
    tc_wait_ld();
#pragma unroll
    for (int e = 0; e < kMend; ++e) {
      const int node = t0 + t + e - prefix;
      const bool want = active && v[e] != v[e] && t + e < tokens && (node < 0 || (mask >> node & 1));
      s[e] = 0.f;
      at[e] = 0;
      if (!__any_sync(0xffffffffu, want)) continue;
      at[e] = (int)tree_row(a.cv, b, t0 + t + e, nullptr);
      bool bad = false;
      for (int k = lane * 8; k < cols; k += 256) bad |= any_not_finite(__ldcg((const uint4*)(a.rope + (long long)at[e] * a.n_h * a.r2 + x0 + k)));
      if (!__any_sync(0xffffffffu, bad)) continue;           // (the latents or the query make them so)
      redo |= 1u << e;
      if (want) mine |= 1u << e;
    }
    if (redo == 0) continue;
    any = true;
    if (mine != 0) {
      const bf16 *const q = a.q_abs + row * a.kw, *const qr = a.q_rope + row * a.r2;
#pragma unroll 2
      for (int k = 0; k < a.kw; k += 8) {
        const uint4 x = __ldcg((const uint4*)(q + k));
        uint4 y[kMend];                    // (tokens that need none take row 0: a branch would make the loads wait for one another)
#pragma unroll
        for (int e = 0; e < kMend; ++e) y[e] = __ldcg((const uint4*)(a.latent + (long long)at[e] * a.d_c + k));
#pragma unroll
        for (int e = 0; e < kMend; ++e) s[e] = dot8(x, y[e], s[e]);
      }
      for (int k = 0; k < a.r2; ++k) {
        const float x = __bfloat162float(qr[k]);
#pragma unroll
        for (int e = 0; e < kMend; ++e) s[e] = fmaf(x, __bfloat162float(a.rope[((long long)at[e] * a.n_h + h) * a.r2 + k]), s[e]);
      }
    }
    __syncwarp();
#pragma unroll
    for (int e = 0; e < kMend; ++e) v[e] = mine >> e & 1 ? s[e] : v[e];
    tc_st8(tm + t, v);
    tc_wait_st();
  }
  return any;
}

template <int CG>
__global__ void __launch_bounds__(kTreeThreads, 1)
tree_tc_kernel(const __grid_constant__ TreeQueryMaps maps_q, const __grid_constant__ CUtensorMap map_k,
               const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_p,
               const __grid_constant__ CUtensorMap map_qr, const __grid_constant__ CUtensorMap map_r,
               const __grid_constant__ CUtensorMap map_ps, const __grid_constant__ CUtensorMap map_o, const __grid_constant__ TreeTcArgs a) {
  using SM = TreeSmem<CG>;
  constexpr int NST = SM::n_stages;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* const base = (unsigned char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  TreeBars* const bars = (TreeBars*)(base + NST * SM::stage + SM::out);
  volatile TreeUnit* const s_unit = (volatile TreeUnit*)(bars + 1);
  // [unit][block of the pair]: nodes with values that are not finite among the columns that the block loads
  volatile unsigned long long* const s_nf = (volatile unsigned long long*)(s_unit + kQueue);
  uint32_t* const s_tmem = (uint32_t*)(s_nf + 2 * kQueue);
  volatile int* const s_abort = (volatile int*)(s_tmem + 1);
  volatile int* const s_verdict = s_abort + 1;      // [2 groups][2]
  volatile int* const s_last = s_verdict + 4;       // [2 groups]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CG == 2 ? cluster_ctarank() : 0;

  if (threadIdx.x == 0) {
    for (int i = 0; i < NST; ++i) {
      mbar_init(smem_u32(&bars->full[i]), 1);
      mbar_init(smem_u32(&bars->empty[i]), 1);
      mbar_init(smem_u32(&bars->spec[i]), 1);
      mbar_init(smem_u32(&bars->fixed[i]), CG);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&bars->acc_full[i]), 1);
      mbar_init(smem_u32(&bars->acc_empty[i]), 4 * CG);
    }
    for (int i = 0; i < kQueue; ++i) {
      mbar_init(smem_u32(&bars->q_full[i]), 1);
      mbar_init(smem_u32(&bars->q_empty[i]), 1 + 7 * CG);
    }
    mbar_init(smem_u32(&bars->go), 1);
    *s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async();
  }
  if (warp == 1) {
    if (CG == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(s_tmem)), "r"(512u) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(s_tmem)), "r"(512u) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  tc_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = *s_tmem;
  ekv_pdl_wait();
  ekv_pdl_trigger();

  const int n_blk = (a.vw + 63) >> 6;                         // 64-column blocks of the partial result
  const int nkl = (a.kw + 63) >> 6;                           // steps of a score unit: latents, then rope columns (n_rc)
  // a published unit: what every role waits for, reads and gives back
  unsigned q_pos = 0;
  auto q_slot = [&]() { return q_pos % kQueue; };
  auto q_parity = [&]() { return (q_pos / kQueue) & 1u; };
  // A unit's words given back (one lane of a warp).  The release orders the warp's reads of them before the other block's warp
  // writes the next unit there (1 % of the long cases; a relaxed arrival would order nothing).
  auto release_unit = [&]() {
    const uint32_t bar = smem_u32(&bars->q_empty[q_slot()]);
    if (rank == 0) mbar_arrive(bar); else mbar_arrive_cluster(map_to_cta(bar, 0));
  };

  if (warp == 0) {
    // ============================================================== queries, P (and the bytes that a step expects)
    bool ok = true;
    unsigned pos = 0;
    for (;; ++q_pos) {
      ok = warp_wait_cluster(smem_u32(&bars->q_full[q_slot()]), q_parity(), s_abort, 1);
      if (!ok) break;
      const volatile TreeUnit* u = s_unit + q_slot();
      const int type = u->kind & 255, lay = u->kind >> 8, b = u->b, rb = u->rb, tok0 = u->tok0, len = u->len, idx = u->idx, slot = u->slot, n = u->n;
      const int prefix = n - u->nodes;
      __syncwarp();
      if (lane == 0) release_unit();
      if (type == kStop) break;
      if (type == kScore) {
        const int all = tree_score_boxes_all(n - (tok0 + idx * kTile), kTile, a.box_s, CG);      // boxes of tokens, both blocks
        const TreeLayout& l = a.lay.of[lay];
        const CUtensorMap* const map_q = &maps_q.of[lay];
        const int h0 = (rb * CG + (int)rank) * l.hb, nkc = nkl + l.n_rc;
        const uint32_t bytes_b = (uint32_t)(all * a.box_s * 128), bytes_l = (uint32_t)(CG * l.m * l.hb * 128) + bytes_b;
        const int yq = (b * a.lay.tiles + (rb * CG + (int)rank) * l.n_rc) * kRows;
        for (int kc = 0; kc < nkc; ++kc, ++pos) {
          const unsigned st = pos % NST;
          ok = warp_wait(smem_u32(&bars->empty[st]), ((pos / NST) & 1) ^ 1, s_abort, 2);
          if (!ok) break;
          const uint32_t fb = smem_u32(&bars->full[st]), dst = smem_u32(base + st * SM::stage);
          const uint32_t cfb = CG == 2 ? map_to_cta(fb, 0) : fb;
          const bool lat = kc < nkl;
          if (kc == max(nkc - kLead, 0) && rank == 0 && lane == 0) mbar_arrive(smem_u32(&bars->go));
          __syncwarp();
          if (elect_one()) {
            if (rank == 0) mbar_expect_tx(fb, lat ? bytes_l : CG * kABytes + bytes_b);
            if (lat) {
              if (CG == 2) tma_load_4d_pair(dst, map_q, kc * 64, 0, h0, b, cfb); else tma_load_4d(dst, map_q, kc * 64, 0, h0, b, cfb);
            } else {
              const int y = yq + (kc - nkl) * kRows;
              if (CG == 2) tma_load_2d_pair(dst, &map_qr, 0, y, cfb); else tma_load_2d(dst, &map_qr, 0, y, cfb);
            }
          }
          __syncwarp();
        }
      } else {
        fence_proxy_all();                  // (P of the piece is complete: the unit was published after that)
        const int bv = a.box_v, per = 64 / bv, ks_n = (len + 63) >> 6;
        const int ch_all = a.v3 ? kTile / 64 : tree_value_chunks_all(min(kTile / 64, (a.vw - idx * kTile + 63) >> 6), CG);      // 64-column chunks loaded, both blocks
        const int y = (slot * CG + (int)rank) * (kPiece / 64) * kRows;
        for (int ks = 0; ks < ks_n; ++ks, ++pos) {
          const int t0 = tok0 + ks * 64, boxes = min(per, (n - t0 + bv - 1) / bv);
          const bool special = t0 + 64 > prefix;
          const unsigned st = pos % NST;
          ok = warp_wait(smem_u32(&bars->empty[st]), ((pos / NST) & 1) ^ 1, s_abort, 4);
          if (!ok) break;
          const uint32_t fb = smem_u32(&bars->full[st]), dst = smem_u32(base + st * SM::stage);
          const uint32_t cfb = CG == 2 ? map_to_cta(fb, 0) : fb;
          if (ks == max(ks_n - kLead, 0) && rank == 0 && lane == 0) mbar_arrive(smem_u32(&bars->go));
          __syncwarp();
          if (elect_one()) {
            if (rank == 0) mbar_expect_tx(fb, (uint32_t)(CG * kABytes + (special ? 0 : ch_all * boxes * bv * 128)));
            if (CG == 2) tma_load_2d_pair(dst, &map_p, 0, y + ks * kRows, cfb); else tma_load_2d(dst, &map_p, 0, y + ks * kRows, cfb);
          }
          __syncwarp();
        }
      }
      if (!ok) break;
    }
  } else if (warp == 2) {
    // ============================================================== cache rows (a box at least in every step: csrc/tree_steps.cuh)
    // Where either product reads a cache row once (one row block), the rows give way in L2 to what is read again: queries, P,
    // partial results (16 x 4096 tokens of 7B, 4 nodes: 134.5 -> 127.7 us, 16 x 2000: 107 -> 95; keeping some of the rows from
    // the score product to the value product by priority was slower, whatever their number)
    const uint64_t pol = a.n_rb == 1 ? make_l2_policy_evict_first() : make_l2_policy_evict_normal();
    bool ok = true;
    unsigned pos = 0;
    for (;; ++q_pos) {
      ok = warp_wait_cluster(smem_u32(&bars->q_full[q_slot()]), q_parity(), s_abort, 17);
      if (!ok) break;
      const volatile TreeUnit* u = s_unit + q_slot();
      const int type = u->kind & 255, lay = u->kind >> 8, b = u->b, rb = u->rb, tok0 = u->tok0, len = u->len, idx = u->idx, n = u->n;
      const int prefix = n - u->nodes;
      __syncwarp();
      if (lane == 0) release_unit();
      if (type == kStop) break;
      if (type == kScore) {
        const int t0 = tok0 + idx * kTile + (int)rank * (kTile / CG);
        const int bs = a.box_s, mine = tree_score_boxes(n - t0, kTile / CG, bs);      // boxes; lane j knows box j's rows
        int row = -bs;                       // (nothing left here: a box before the plane's first row)
        if (lane < mine && t0 < n) row = (int)tree_row(a.cv, b, t0 + lane * bs, a.status);
        const int xr = tree_rope_col(rb * CG * a.lay.of[lay].hb, a.r2), nkc = nkl + a.lay.of[lay].n_rc;
        for (int kc = 0; kc < nkc; ++kc, ++pos) {
          const unsigned st = pos % NST;
          ok = warp_wait(smem_u32(&bars->empty[st]), ((pos / NST) & 1) ^ 1, s_abort, 18);
          if (!ok) break;
          const uint32_t fb = smem_u32(&bars->full[st]), dst = smem_u32(base + st * SM::stage + kABytes);
          const uint32_t cfb = CG == 2 ? map_to_cta(fb, 0) : fb;
          const CUtensorMap* const map_b = kc < nkl ? &map_k : &map_r;
          const int xb = kc < nkl ? kc * 64 : xr + (kc - nkl) * 64;
          for (int j = 0; j < mine; ++j) {
            const int y = __shfl_sync(0xffffffffu, row, j);
            if (elect_one()) {
              if (CG == 2) tma_load_2d_pair_hint(dst + j * bs * 128, map_b, xb, y, cfb, pol);
              else tma_load_2d_hint(dst + j * bs * 128, map_b, xb, y, cfb, pol);
            }
            __syncwarp();
          }
        }
      } else {
        const int bv = a.box_v, per = 64 / bv, ks_n = (len + 63) >> 6;
        // this block's columns: its half of the tile's (a quarter where half of the tile is enough: the product's width is halved)
        const int held = min(kTile / 64, (a.vw - idx * kTile + 63) >> 6), mine = tree_value_share(held, CG);
        const int x0 = idx * kTile + (int)rank * mine * 64, ch = a.v3 ? 4 / CG : tree_value_chunks(held, CG, (int)rank);
        int row = 0;
        for (int ks = 0; ks < ks_n; ++ks, ++pos) {
          const int b0 = ks * per;                    // first box of the step
          if ((b0 & 31) == 0) {
            const int t = tok0 + (b0 + lane) * bv;
            row = t < n && t < tok0 + len ? (int)tree_row(a.cv, b, t, nullptr) : 0;
          }
          const int t0 = tok0 + ks * 64, boxes = min(per, (n - t0 + bv - 1) / bv);
          const bool special = t0 + 64 > prefix;
          const unsigned st = pos % NST;
          ok = warp_wait(smem_u32(&bars->empty[st]), ((pos / NST) & 1) ^ 1, s_abort, 19);
          if (!ok) break;
          const uint32_t fb = smem_u32(&bars->full[st]), sb = smem_u32(&bars->spec[st]), dst = smem_u32(base + st * SM::stage + kABytes);
          const uint32_t cfb = CG == 2 ? map_to_cta(fb, 0) : fb;
          if (special) {
            if (elect_one()) mbar_expect_tx(sb, (uint32_t)(ch * boxes * bv * 128));
            __syncwarp();
          }
          for (int j = 0; j < boxes; ++j) {
            const int y = __shfl_sync(0xffffffffu, row, (b0 + j) & 31);
            if (elect_one()) {
              if (a.v3) {
                if (special || CG == 1) tma_load_3d_hint(dst, &map_v, 0, y, x0 >> 6, special ? sb : fb, pol);
                else tma_load_3d_pair_hint(dst, &map_v, 0, y, x0 >> 6, cfb, pol);
              } else {
                for (int c = 0; c < ch; ++c) {
                  const uint32_t d = dst + c * 8192 + j * bv * 128;
                  if (special || CG == 1) tma_load_2d_hint(d, &map_v, x0 + c * 64, y, special ? sb : fb, pol);
                  else tma_load_2d_pair_hint(d, &map_v, x0 + c * 64, y, cfb, pol);
                }
              }
            }
            __syncwarp();
          }
        }
      }
      if (!ok) break;
    }
  } else if (warp == 1) {
    // ============================================================== products (the first block's warp, for both)
    if (rank == 0) {
      constexpr uint32_t idesc_s = make_idesc(kRows * CG, kTile, 0, 0), idesc_v = make_idesc(kRows * CG, kTile, 0, 1);
      constexpr uint32_t idesc_h = make_idesc(kRows * CG, kTile / 2, 0, 1);       // the last tile, where half of it is enough
      constexpr uint32_t hi_sw = desc_hi(1024, 2);
      const uint32_t base16 = (smem_u32(base) >> 4) & 0x3FFFu;
      bool ok = true;
      unsigned pos = 0, fix_bits = 0;
      for (;; ++q_pos) {
        ok = warp_wait_cluster(smem_u32(&bars->q_full[q_slot()]), q_parity(), s_abort, 5);
        if (!ok) break;
        const volatile TreeUnit* u = s_unit + q_slot();
        const int type = u->kind & 255, lay = u->kind >> 8, tok0 = u->tok0, len = u->len, prefix = u->n - u->nodes;
        const bool half_tile = a.vw - u->idx * kTile <= kTile / 2;
        __syncwarp();
        if (lane == 0) release_unit();
        if (type == kStop) break;
        const unsigned buf = q_pos & 1;
        ok = warp_wait_cluster(smem_u32(&bars->acc_empty[buf]), ((q_pos >> 1) & 1) ^ 1, s_abort, 6);
        if (!ok) break;
        tc_fence_after();
        const uint32_t d = tmem_base + buf * kTile;
        const int steps = type == kScore ? nkl + a.lay.of[lay].n_rc : (len + 63) >> 6;
        for (int ks = 0; ks < steps; ++ks, ++pos) {
          const unsigned st = pos % NST;
          ok = warp_wait(smem_u32(&bars->full[st]), (pos / NST) & 1, s_abort, 7);
          if (ok && type == kValue && tok0 + ks * 64 + 64 > prefix) {
            ok = warp_wait_cluster(smem_u32(&bars->fixed[st]), fix_bits >> st & 1, s_abort, 8);
            fix_bits ^= 1u << st;
          }
          if (!ok) break;
          tc_fence_after();
          const uint32_t la = (base16 + st * (SM::stage >> 4)) | (1u << 16);
          // scores: 64 latents of 256 tokens, K-major; values: 64 tokens of 256 columns, 8 KB from one 64-column chunk to the next
          const uint32_t lb = (base16 + ((st * SM::stage + kABytes) >> 4)) | (type == kScore ? 1u << 16 : (8192u >> 4) << 16);
          const uint32_t step_b = type == kScore ? 2 : 128;
          const uint32_t idesc = type == kScore ? idesc_s : half_tile ? idesc_h : idesc_v;
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              if (CG == 2) tc_mma_pair(d, la + 2 * k, hi_sw, lb + step_b * k, hi_sw, idesc, (ks | k) != 0);
              else tc_mma_w(d, la + 2 * k, hi_sw, lb + step_b * k, hi_sw, idesc, (ks | k) != 0);
            }
            if (CG == 2) tc_commit_pair(smem_u32(&bars->empty[st])); else tc_commit(smem_u32(&bars->empty[st]));
          }
          __syncwarp();
        }
        if (!ok) break;
        if (elect_one()) {
          if (CG == 2) tc_commit_pair(smem_u32(&bars->acc_full[buf])); else tc_commit(smem_u32(&bars->acc_full[buf]));
        }
        __syncwarp();
      }
    }
  } else if (warp == 3) {
    // ============================================================== drafted rows of the value product
    bool ok = true;
    unsigned pos = 0, spec_bits = 0;
    for (;; ++q_pos) {
      ok = warp_wait_cluster(smem_u32(&bars->q_full[q_slot()]), q_parity(), s_abort, 9);
      if (!ok) break;
      const volatile TreeUnit* u = s_unit + q_slot();
      const int type = u->kind & 255, lay = u->kind >> 8, tok0 = u->tok0, len = u->len, idx = u->idx, n = u->n, prefix = n - u->nodes;
      if (type == kStop) break;
      if (type == kScore) {
        pos += nkl + a.lay.of[lay].n_rc;
      } else {
        const int ks_n = (len + 63) >> 6;
        const int held = min(kTile / 64, (a.vw - idx * kTile + 63) >> 6);
        const int ch = max(0, min(tree_value_share(held, CG), held - tree_value_share(held, CG) * (int)rank));      // (chunks past the last column are not stored)
        unsigned nf_lo = 0, nf_hi = 0;
        for (int ks = 0; ks < ks_n; ++ks, ++pos) {
          const int t0 = tok0 + ks * 64;
          if (t0 + 64 <= prefix) continue;
          const unsigned st = pos % NST;
          ok = warp_wait(smem_u32(&bars->spec[st]), spec_bits >> st & 1, s_abort, 10);
          spec_bits ^= 1u << st;
          if (!ok) break;
          const int r0 = max(prefix - t0, 0);
          const int vecs = (64 - r0) * 8;
          for (int c = 0; c < ch; ++c) {
            uint4* const rows = (uint4*)(base + st * SM::stage + kABytes + c * 8192) + r0 * 8;
            for (int e = lane; e < vecs; e += 32) {
              const int t = t0 + r0 + (e >> 3);
              if (t >= n) {
                rows[e] = make_uint4(0, 0, 0, 0);
                continue;
              }
              uint4 x = rows[e];
              uint32_t w[4] = {x.x, x.y, x.z, x.w};
              bool bad = false;
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                if ((w[k] & 0x7f80u) == 0x7f80u) { w[k] &= 0xffff0000u; bad = true; }
                if ((w[k] & 0x7f800000u) == 0x7f800000u) { w[k] &= 0xffffu; bad = true; }
              }
              if (bad) {
                rows[e] = make_uint4(w[0], w[1], w[2], w[3]);
                const int j = t - prefix;
                if (j < 32) nf_lo |= 1u << j; else nf_hi |= 1u << (j - 32);
              }
            }
          }
          if (t0 + 64 >= n || ks == ks_n - 1) {       // the last of the unit: the note goes first
            const unsigned lo = __reduce_or_sync(0xffffffffu, nf_lo), hi = __reduce_or_sync(0xffffffffu, nf_hi);
            // to both blocks: a block's rows meet the columns of both
            if (lane == 0) {
              const uint32_t to = smem_u32((const void*)(s_nf + 2 * q_slot() + rank));
              if (CG == 2) {
#pragma unroll
                for (int c2 = 0; c2 < 2; ++c2) {
                  st_cluster_u32(map_to_cta(to, c2), lo);
                  st_cluster_u32(map_to_cta(to + 4, c2), hi);
                }
              } else {
                s_nf[2 * q_slot()] = (unsigned long long)hi << 32 | lo;
              }
            }
          }
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) {
            if (CG == 2) mbar_arrive_cluster(map_to_cta(smem_u32(&bars->fixed[st]), 0)); else mbar_arrive(smem_u32(&bars->fixed[st]));
          }
        }
        if (!ok) break;
      }
      __syncwarp();
      if (lane == 0) release_unit();
    }
  } else if (warp == 12) {
    // ============================================================== units (the first block's warp, for both)
    if (rank == 0) {
      const int n_runs = __ldcg(a.hdr + 1), n_pieces = __ldcg(a.hdr + 2), ahead = __ldcg(a.hdr + 3);
      // (the list is read over and over: brought into L1 once)
      int warm = 0;
      for (int k = lane * 4; k < n_runs; k += 128) warm |= a.runs[2 * k].x;
      PieceWalk ws{0, 0, 0, 0, make_int4(0, 0, 0, 0), make_int4(0, 0, 0, 0)};
      if (n_runs > 0) walk_load(ws, a);
      PieceWalk wv = ws;
      int first = warm < 0 ? 1 : 0, j = 0;     // first unit of block j (no sequence is negative)
      bool stopped = false;
      for (;; ++q_pos) {
        // claimed late: a unit that waits here while others depend on it holds them up
        if (q_pos > 0 && !stopped && !warp_wait(smem_u32(&bars->go), (q_pos - 1) & 1, s_abort, 20)) break;
        if (!warp_wait_cluster(smem_u32(&bars->q_empty[q_slot()]), q_parity() ^ 1, s_abort, 11)) break;
        int unit = 0;
        if (lane == 0) unit = atomicAdd((int*)a.hdr, 1);
        unit = __shfl_sync(0xffffffffu, unit, 0);
        int n_s = 0, n_v = 0;
        bool stop = false;
        for (;;) {
          n_s = j < n_pieces ? (walk_len(ws) + kTile - 1) / kTile : 0;
          n_v = j >= ahead ? a.n_ct : 0;
          stop = j >= n_pieces + ahead;
          if (stop || unit < first + n_s + n_v) break;
          first += n_s + n_v;
          if (j < n_pieces) walk_next(ws, a, n_runs, n_pieces);
          if (j >= ahead) walk_next(wv, a, n_runs, n_pieces);
          ++j;
        }
        const int at = unit - first;
        const bool score = at < n_s;
        const PieceWalk& w = score ? ws : wv;
        // a value unit is published when P of its piece is complete, in both blocks' rows
        if (!stop && !score && !__all_sync(0xffffffffu, lane != 0 || poll_global(a.ready + w.p % kSlots, (w.p / kSlots + 1) * CG, s_abort, 3))) break;
        int x, y, z, t;                        // 16 bytes of the unit per lane
        if (lane == 0) { x = stop ? kStop : (score ? kScore : kValue) | w.r2.w << 8; y = w.r.x; z = w.rb; t = w.r.y + w.k * kPiece; }
        else if (lane == 1) { x = walk_len(w); y = score ? at : at - n_s; z = w.p % kSlots; t = w.p / kSlots; }
        else { x = w.r2.x; y = w.r2.y; z = w.r2.z; t = w.k; }
        const uint32_t to = smem_u32((const void*)(s_unit + q_slot())) + 16 * lane, bar = smem_u32(&bars->q_full[q_slot()]);
#pragma unroll
        for (int c = 0; c < CG; ++c) {
          const uint32_t cbar = map_to_cta(bar, c);
          if (lane == 0) mbar_expect_tx_cluster_relaxed(cbar, 48);
          if (lane < 3) st_async_v4(map_to_cta(to, c), (uint32_t)x, (uint32_t)y, (uint32_t)z, (uint32_t)t, cbar);
        }
        __syncwarp();
        if (stop && stopped) break;            // once for each epilogue group
        stopped = stop;
      }
    }
  } else {
    // ============================================================== epilogue: thread = row; two groups of four warps
    // Group g has the units at even (odd) places and their accumulator, so that the waits of one group's unit (rows on
    // their way to memory, counters) pass while the other computes.
    const int group_id = (warp - 4) >> 2, quarter = warp & 3, r = quarter * 32 + lane;
    const bool leader = (threadIdx.x & 127) == 0;
    const uint32_t tm = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(group_id * kTile);
    int laid = -1, hl = 0, i = 0;               // the row's head and node in layout `laid`
    volatile int* const verdict = s_verdict + 2 * group_id;
    volatile int* const last = s_last + group_id;
    // rows on their way out: two boxes (128-byte swizzle)
    const uint32_t out_box = smem_u32(base + NST * SM::stage + (warp - 4) * kOutBytes);
    auto put = [&](int box, int j, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {       // 16 bytes of this lane's row
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};"
                   ::"r"(out_box + box * (kOutBytes / 2) + lane * 128 + ((j ^ (lane & 7)) << 4)), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
    };
    auto out_free = [&]() {                     // the box of the store before the last has been read
      if (lane == 0) bulk_wait_group_read<1>();
      __syncwarp();
    };
    unsigned turn = 0;
    // the leader looks, everybody gets its verdict
    auto group = [&](auto probe) -> bool {
      volatile int* const word = verdict + (turn & 1u);
      ++turn;
      if (leader) *word = probe() ? 1 : 0;
      named_bar_sync(2 + group_id, kEpiThreads);
      return *word != 0;
    };
    auto group_bar = [&](uint32_t bar, uint32_t parity, int why) -> bool {
      const bool ok = group([&]() {
        for (unsigned k = 0; k < kSpinLimit; ++k) {
          if (mbar_try_wait_cluster(bar, parity)) return true;
          if ((k & 1023) == 1023 && *s_abort) return false;
        }
        if (*s_abort == 0) *s_abort = why;
        return false;
      });
      if (ok) (void)mbar_try_wait_cluster(bar, parity);
      return ok;
    };
    for (q_pos = group_id;; q_pos += 2) {
      if (!group_bar(smem_u32(&bars->q_full[q_slot()]), q_parity(), 12)) break;
      const volatile TreeUnit* u = s_unit + q_slot();
      const int type = u->kind & 255, lay = u->kind >> 8, b = u->b, rb = u->rb, tok0 = u->tok0, len = u->len, idx = u->idx, slot = u->slot, gen = u->gen, n = u->n;
      const int nodes = u->nodes, run = u->run, k_run = u->k, prefix = n - nodes;
      if (type == kStop) break;
      const uint32_t acc_bar = smem_u32(&bars->acc_full[group_id]), acc_par = (q_pos >> 1) & 1;
      if (lay != laid) {
        laid = lay;
        hl = r / a.lay.of[lay].m;
        i = r - hl * a.lay.of[lay].m;
      }
      const int hb = a.lay.of[lay].hb, h = (rb * CG + (int)rank) * hb + hl;
      const bool real = hl < hb && h < a.n_h, active = real && i < nodes;
      const unsigned long long mask = active ? a.mask[(long long)b * a.m + i] : 0ull;
      const long long half = (long long)slot * CG + rank;        // this block's share of the slot
      auto acc_done = [&]() {
        tc_fence_before();
        __syncwarp();
        // What the arrival stands for is in registers: tcgen05.wait::ld has waited for it.  (With release semantics over the
        // cluster it held the warp that issues the products for 2500 clocks a unit.)
        if (lane == 0) {
          const uint32_t bar = smem_u32(&bars->acc_empty[group_id]);
          if (rank == 0) mbar_arrive(bar); else mbar_arrive_cluster_relaxed(map_to_cta(bar, 0));
        }
      };
      if (type == kScore) {
        const int t0 = tok0 + idx * kTile;
        // the slot's last piece is read to the end
        if (gen > 0 && !group([&]() { return poll_global(a.v_done + slot, gen * a.n_ct * CG, s_abort, 13); })) break;
        if (!group_bar(acc_bar, acc_par, 14)) break;
        tc_fence_after();
        // which of 32 tokens the row sees; tiles of committed tokens alone skip it
        const bool all = t0 + kTile <= prefix;
        auto seen_bits = [&](int t) -> unsigned {                  // tokens t .. t + 31
          if (t + 32 <= prefix) return 0xffffffffu;
          const int d = prefix - t;                                // committed ones in front: d of them
          const unsigned long long v = d >= 0 ? (mask << d) | ((1ull << d) - 1ull) : d > -64 ? mask >> -d : 0ull;
          const int left = n - t;
          return left <= 0 ? 0u : (unsigned)v & (left >= 32 ? 0xffffffffu : (1u << left) - 1u);
        };
        // one pass with the reference 0; another where a row's largest score is out of range
        float ref = 0.f, sum = 0.f;
        for (bool again = false, looked = a.lay.of[lay].n_rc == 0;;) {
          float top = -INFINITY, sum4[4] = {0.f, 0.f, 0.f, 0.f};
          auto chunk = [&](int cc, float* x) {                     // 32 tokens
            if (!all) {
              const unsigned bits = seen_bits(t0 + cc * 32);
#pragma unroll
              for (int e = 0; e < 32; ++e) x[e] = bits >> e & 1 ? x[e] : -INFINITY;
            }
            float t4[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
            for (int e = 4; e < 32; ++e) t4[e & 3] = fmaxf(t4[e & 3], x[e]);
            top = fmaxf(top, fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3])));
            const int box = (cc >> 1) & 1;                         // 64 tokens each
            if ((cc & 1) == 0) out_free();
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              uint32_t w[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const bf162 p = __floats2bfloat162_rn(ex2(fmaf(x[8 * g + 2 * e], a.scale_log2e, -ref)), ex2(fmaf(x[8 * g + 2 * e + 1], a.scale_log2e, -ref)));
                w[e] = *(const uint32_t*)&p;
                sum4[2 * (e & 1)] += __uint_as_float(w[e] << 16);
                sum4[2 * (e & 1) + 1] += __uint_as_float(w[e] & 0xffff0000u);
              }
              put(box, (cc & 1) * 4 + g, w[0], w[1], w[2], w[3]);
            }
            if ((cc & 1) == 0) return;
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) {
              tma_store_2d(&map_ps, 0, ((int)half * (kPiece / 64) + idx * (kTile / 64) + (cc >> 1)) * kRows + quarter * 32, out_box + box * (kOutBytes / 2));
              bulk_commit_group();
            }
          };
          float v0[32], v1[32];
          tc_ld32(tm, v0);
#pragma unroll 1
          for (int cc = 0; cc < kTile / 32; cc += 2) {
            tc_wait_ld();
            tc_ld32(tm + (cc + 1) * 32, v1);
            chunk(cc, v0);
            tc_wait_ld();
            if (cc + 2 < kTile / 32) tc_ld32(tm + (cc + 2) * 32, v0);
            chunk(cc + 1, v1);
          }
          sum = (sum4[0] + sum4[1]) + (sum4[2] + sum4[3]);
          if (again) break;
          if (!looked && __any_sync(0xffffffffu, active && sum != sum)) {
            looked = true;
            const int x0 = tree_rope_col(rb * CG * hb, a.r2), cols = min(a.lay.of[lay].n_rc * 64, a.n_h * a.r2 - x0);
            if (mend_scores(a, tm, b, h, i, t0, min(kTile, n - t0), prefix, active ? mask : 0ull, active, x0, cols)) {
              if (lane == 0) bulk_wait_group_all();
              __syncwarp();
              continue;
            }
          }
          // (rows of padding nodes weigh nothing, whatever their queries hold)
          top *= a.scale_log2e;
          ref = !active || top == -INFINITY || fabsf(top) <= 64.f ? 0.f : 64.f * rintf(top * (1.f / 64.f));
          if (__all_sync(0xffffffffu, ref == 0.f)) break;
          again = true;
          if (lane == 0) bulk_wait_group_all();      // both passes write the same rows
          __syncwarp();
        }
        if (!active) sum = 0.f;
        acc_done();
        a.stats[(half * kTiles + idx) * kRows + r] = make_float2(ref, sum);
        if (lane == 0) {
          bulk_wait_group_all();             // the rows are in memory
          fence_proxy_all();
        }
        __threadfence();
        named_bar_sync(2 + group_id, kEpiThreads);
        const int tiles = (len + kTile - 1) / kTile;
        if (leader) {
          const int before = atomicAdd(a.s_cnt + half, 1);
          __threadfence();
          *last = before == tiles - 1;
        }
        named_bar_sync(2 + group_id, kEpiThreads);
        if (*last) {
          // the piece's rows agree on a reference
          const float2* const st = a.stats + half * kTiles * kRows + r;
          float m_ref = -1e30f, total = 0.f;
          float2 x[kTiles];
#pragma unroll
          for (int t = 0; t < kTiles; ++t) x[t] = t < tiles ? __ldcg(st + t * kRows) : make_float2(0.f, 0.f);
#pragma unroll
          for (int t = 0; t < kTiles; ++t)
            if (x[t].y != 0.f) m_ref = fmaxf(m_ref, x[t].x);
#pragma unroll
          for (int t = 0; t < kTiles; ++t) {
            if (x[t].y == 0.f) continue;
            const float f = x[t].x == m_ref ? 1.f : exp2f(x[t].x - m_ref);
            total = fmaf(x[t].y, f, total);
            if (f != 1.f && real) {
#pragma unroll 1
              for (int e = 0; e < kTile / 2; ++e) {
                uint32_t* const pr = (uint32_t*)(a.P + ((half * (kPiece / 64) + t * (kTile / 64) + (e >> 5)) * kRows + r) * 64) + (e & 31);
                const uint32_t w = __ldcg(pr);
                const bf162 y = __floats2bfloat162_rn(__uint_as_float(w << 16) * f, __uint_as_float(w & 0xffff0000u) * f);
                *pr = *(const uint32_t*)&y;
              }
            }
          }
          a.pref[half * kRows + r] = make_float2(m_ref, total);
          fence_proxy_all();
          __threadfence();
          named_bar_sync(2 + group_id, kEpiThreads);
          if (leader) {
            a.s_cnt[half] = 0;
            add_release(a.ready + slot, 1);
          }
        }
      } else {
        const long long ci = ((long long)run * a.n_rb + rb) * a.n_ct + idx;
        if (!group_bar(acc_bar, acc_par, 16)) break;
        tc_fence_after();
        // the piece before in the run is in the partial result
        if (k_run > 0 && !group([&]() { return poll_global(a.chain + ci, k_run * CG, s_abort, 15); })) break;
        const float2 mine = __ldcg(a.pref + half * kRows + r);
        float2* const state = a.cstate + (ci * CG + rank) * kRows + r;
        const long long tile = ((long long)run * a.n_rb + rb) * CG + rank;      // the block's rows in the partial result
        float2 now = mine;
        float f_old = 1.f, f_new = 1.f;
        if (k_run > 0) {
          const float2 old = __ldcg(state);
          now.x = fmaxf(old.x, mine.x);
          f_old = exp2f(old.x - now.x);
          f_new = exp2f(mine.x - now.x);
          now.y = old.y * f_old + mine.y * f_new;
          if (old.y == 0.f || !real) f_old = 1.f;       // (nothing there to scale, or nobody reads it)
        }
        // (values before the drafted ones are what all rows see; a row that sees nothing adds nothing)
        const bool special = tok0 + ((len + 63) & ~63) > prefix;
        const bool spoiled = special && ((s_nf[2 * q_slot()] | (CG == 2 ? s_nf[2 * q_slot() + 1] : 0ull)) & mask) != 0;
        const bool none = mine.y == 0.f;
        const bool scaled = __any_sync(0xffffffffu, f_old != 1.f);
        *state = now;
        if (idx == 0) a.part_ml[tile * kRows + r] = now;
        auto chunk = [&](int cc, float* x) {              // 32 columns
          const int col = idx * kTile + cc * 32;
          if (col >= a.vw) return;                        // (the same for the whole warp)
          const long long row0 = (tile * n_blk + (col >> 6)) * kRows;
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] = spoiled ? __uint_as_float(0x7fffffffu) : none ? 0.f : x[e] * f_new;
          if (scaled) {                                   // references moved: what is there is scaled by its reader
            const float* const o = a.part_acc + (row0 + r) * 64 + (col & 63);
#pragma unroll
            for (int e = 0; e < 32; e += 4)
              if (col + e < a.vw) {
                const float4 y = __ldcg((const float4*)(o + e));
                x[e] += y.x * f_old; x[e + 1] += y.y * f_old; x[e + 2] += y.z * f_old; x[e + 3] += y.w * f_old;
              }
          }
          const int box = cc & 1;
          out_free();
#pragma unroll
          for (int g = 0; g < 8; ++g)
            put(box, g, __float_as_uint(x[4 * g]), __float_as_uint(x[4 * g + 1]), __float_as_uint(x[4 * g + 2]), __float_as_uint(x[4 * g + 3]));
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) {
            const uint32_t from = out_box + box * (kOutBytes / 2);
            if (k_run == 0 || scaled) tma_store_2d(&map_o, col & 63, (int)row0 + quarter * 32, from);
            else tma_add_2d(&map_o, col & 63, (int)row0 + quarter * 32, from);
            bulk_commit_group();
          }
        };
        float v0[32], v1[32];
        tc_ld32(tm, v0);
#pragma unroll 1
        for (int cc = 0; cc < kTile / 32; cc += 2) {
          tc_wait_ld();
          tc_ld32(tm + (cc + 1) * 32, v1);
          chunk(cc, v0);
          tc_wait_ld();
          if (cc + 2 < kTile / 32) tc_ld32(tm + (cc + 2) * 32, v0);
          chunk(cc + 1, v1);
        }
        acc_done();
        if (lane == 0) {
          bulk_wait_group_all();
          fence_proxy_all();
        }
        __threadfence();
        named_bar_sync(2 + group_id, kEpiThreads);
        if (leader) {
          add_release(a.chain + ci, 1);
          add_release(a.v_done + slot, 1);
        }
      }
      if (lane == 0) release_unit();
    }
  }

  // ============================================================== teardown
  tc_fence_before();
  __syncthreads();
  if (*s_abort) drain_after_abort();
  if (threadIdx.x == 0 && *s_abort) ekv_record(a.status, ELITEKV_ERR_TIMEOUT, (int)blockIdx.x | (*s_abort << 16), 0);
  __syncwarp();
  if (CG == 2) cluster_sync_all();         // the tensor core and the peer's roles are through with this block's memory
  if (warp == 1) {
    tc_fence_after();
    if (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
  }
}

// ------------------------------------------------------------------ runs
struct TreePrepArgs {
  const int32_t *seq_lens, *n_nodes;
  const bf16* q_rope;
  bf16* qr;                   // [B][lay.tiles: row block, block, n_rc][128][64]
  TreeLayouts lay;
  int B, m, n_ct, want, workers, cg, n_h, r2, zero_blocks;
  long long max_len;
  int* hdr;
  int4* runs;
  int32_t *seq_first, *seq_lay;
  int* zero;
  int n_zero;
  int32_t* status;
};

// One block cuts every sequence into runs of equal length (a multiple of 256 tokens): about `want` of them beside one
// per sequence, so that the value units fill the workers a few times over.  Others zero the counters; the rest of the
// grid spreads the queries' rope parts over the columns of their row block's heads.
__global__ void __launch_bounds__(256)
tree_prep_kernel(const TreePrepArgs a) {
  ekv_pdl_wait();
  ekv_pdl_trigger();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (blockIdx.x > a.zero_blocks) {
    // 16 bytes of the spread queries per thread: chunk c's columns [64 c + 8 v, + 8) of a row
    const long long vecs = (long long)a.B * a.lay.tiles * kRows * 8;
    const long long step = (long long)(gridDim.x - 1 - a.zero_blocks) * 256;
    for (long long x = (long long)(blockIdx.x - 1 - a.zero_blocks) * 256 + tid; x < vecs; x += step) {
      const int v = (int)(x & 7), row = (int)(x >> 3) % kRows;
      const long long y = (x >> 3) / kRows;
      const int tile = (int)(y % a.lay.tiles), b = (int)(y / a.lay.tiles);
      const TreeLayout& l = a.lay.of[tree_layout(a.lay, tree_lens(a.seq_lens, a.n_nodes, b, a.m, a.max_len).nodes)];
      const int c = tile % l.n_rc, block = tile / l.n_rc;
      if (block >= l.n_rb * a.cg) continue;
      const int hl = row / l.m, i = row - hl * l.m, h = block * l.hb + hl;
      const int col = tree_rope_col(block / a.cg * a.cg * l.hb, a.r2) + c * 64 + v * 8 - h * a.r2;     // of the head's own 2r
      const bool real = hl < l.hb && h < a.n_h;
      const bf16* const q = a.q_rope + (((long long)b * a.m + i) * a.n_h + (real ? h : 0)) * a.r2;
      __align__(16) unsigned short w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = real && col + e >= 0 && col + e < a.r2 ? ((const unsigned short*)q)[col + e] : (unsigned short)0;
      *(uint4*)(a.qr + x * 8) = *(const uint4*)w;
    }
    return;
  }
  if (blockIdx.x > 0) {
    const int t = (blockIdx.x - 1) * 256 + tid, step = a.zero_blocks * 256;
    for (int k = t; k < a.n_zero; k += step) a.zero[k] = 0;
    return;
  }
  __shared__ long long s_sum[8];
  __shared__ int s_cnt[3][8];
  __shared__ int s_bin[kBins + 1];            // runs of so many pieces (kBins: that many or more), then where they go
  long long total = 0;
  for (int b = tid; b < a.B; b += 256) {
    const TreeLens t = tree_lens(a.seq_lens, a.n_nodes, b, a.m, a.max_len);
    if (t.bad) ekv_record(a.status, ELITEKV_ERR_BAD_POSITION, b, a.seq_lens[b]);
    if (t.nodes > 0) total += t.n;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  if (lane == 0) s_sum[warp] = total;
  __syncthreads();
  total = 0;
  for (int w = 0; w < 8; ++w) total += s_sum[w];
  const long long per = (total + a.want - 1) / a.want;
  const long long up = (per + 255) / 256 * 256;
  const int run_len = (int)(up < 256 ? 256 : up > (1ll << 30) ? 1ll << 30 : up);      // (no sequence is longer than 2^30)
  int run0 = 0, item0 = 0, score0 = 0;
  for (int k = tid; k <= kBins; k += 256) s_bin[k] = 0;
  __syncthreads();
  // runs of a sequence: their length, the pieces of one and of the last
  auto cut = [&](const TreeLens& t, int& runs, int& len, int& pieces, int& pieces_last) {
    runs = pieces = pieces_last = 0;
    len = 256;
    if (t.nodes == 0) return;                 // a sequence without nodes has only padding: zero rows
    runs = (t.n + run_len - 1) / run_len;
    len = ((t.n + runs - 1) / runs + 255) / 256 * 256;
    runs = (t.n + len - 1) / len;
    pieces = (len + kPiece - 1) / kPiece;
    pieces_last = (t.n - (runs - 1) * len + kPiece - 1) / kPiece;
  };
  for (int b = tid; b < a.B; b += 256) {
    int runs, len, pieces, last;
    cut(tree_lens(a.seq_lens, a.n_nodes, b, a.m, a.max_len), runs, len, pieces, last);
    if (runs > 1) atomicAdd(&s_bin[min(pieces, kBins)], runs - 1);
    if (runs > 0) atomicAdd(&s_bin[min(last, kBins)], 1);
  }
  __syncthreads();
  if (warp == 0) {                            // most pieces first: lane l adds up eight bins from the top
    int v[8], sum = 0;
    for (int e = 0; e < 8; ++e) {
      v[e] = sum;
      sum += s_bin[kBins - 8 * lane - e];
    }
    int before = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, before, o);
      if (lane >= o) before += y;
    }
    before -= sum;
    __syncwarp();
    for (int e = 0; e < 8; ++e) s_bin[kBins - 8 * lane - e] = before + v[e];
  }
  __syncthreads();
  for (int b0 = 0; b0 < a.B; b0 += 256) {
    const int b = b0 + tid;
    TreeLens t{0, 0, false};
    int runs = 0, len = 256, pieces = 0, last = 0;
    if (b < a.B) {
      t = tree_lens(a.seq_lens, a.n_nodes, b, a.m, a.max_len);
      cut(t, runs, len, pieces, last);
    }
    const int lay = tree_layout(a.lay, t.nodes), n_rb = a.lay.of[lay].n_rb;
    const int items = runs > 0 ? ((runs - 1) * pieces + last) * n_rb : 0, scores = runs > 0 ? (t.n + kTile - 1) / kTile * n_rb : 0;
    int v[3] = {runs, items, scores}, x[3];
#pragma unroll
    for (int e = 0; e < 3; ++e) {
      x[e] = v[e];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x[e], o);
        if (lane >= o) x[e] += y;
      }
      if (lane == 31) s_cnt[e][warp] = x[e];
    }
    __syncthreads();
    int at = run0 + x[0] - v[0];
    for (int w = 0; w < 8; ++w) {
      if (w < warp) at += s_cnt[0][w];
      run0 += s_cnt[0][w];
      item0 += s_cnt[1][w];
      score0 += s_cnt[2][w];
    }
    if (b < a.B) {
      a.seq_first[b] = at;
      a.seq_lay[b] = lay;
      for (int k = 0; k < runs; ++k) {
        const int tok = k * len, l = min(len, t.n - tok), np = k < runs - 1 ? pieces : last;
        const int to = atomicAdd(&s_bin[min(np, kBins)], 1);      // (the order among equals is nobody's concern)
        a.runs[2 * to] = make_int4(b, tok, l, np);
        a.runs[2 * to + 1] = make_int4(t.n, t.nodes, at + k, lay);
      }
    }
    __syncthreads();
  }
  if (tid == 0) {
    a.seq_first[a.B] = run0;
    const long long pieces = item0, units = score0 + pieces * a.n_ct;
    // how far the score units go ahead of the value units: what the workers hold three and a half times over (1.5 times: 3 to 6 %
    // slower, 2.5: up to 2 %)
    long long d = units > 0 ? (7ll * a.workers * pieces + 2 * units - 1) / (2 * units) : 1;
    d = d < 1 ? 1 : d > kMostAhead ? kMostAhead : d;
    a.hdr[0] = 0;
    a.hdr[1] = run0;
    a.hdr[2] = (int)pieces;
    a.hdr[3] = (int)d;
  }
}

// ------------------------------------------------------------------ runs joined, W_uv
// out[b,i,h,:] = (sum over runs 2^(m_run - M) acc_run / L) . W_uv,h: block = (head, as many whole sequences as 128 rows
// (b, i) hold, a share of the latent axis).  The partial results lie in blocks of 64 latents, in which the m rows of a head
// are one piece: bulk copies bring (64 latents, one run) of all rows into a ring, kUpWarps warps add them up with the runs'
// weights and write a bf16 head plus a bf16 remainder as the A tile of two products with W_uv's [64 x d_h] block.  Blocks
// that share a tile's depth are a cluster; each adds its share of the columns over the others' sums in block order through
// distributed shared memory.
// Bound: the partial results, read once; the ring keeps up to 96 KB of them in flight (32 KB, in registers, took 3 times
// as long).
constexpr int kUpWarps = 16;              // that join and lay out; one more each for partial results, products, W_uv
constexpr int kUpThreads = 32 * (kUpWarps + 3);
constexpr int kUpSlots = 16;              // of the ring, at most
constexpr int kUpRing = 96 * 1024;
constexpr int kUpHeld = 8;                // runs whose weights a row keeps

struct UpArgs {
  const float* part_acc;
  const float2* part_ml;
  const int32_t *seq_first, *seq_lay;
  TreeLayouts lay;
  bf16* out;
  int B, m, n_h, d_h, n_half, vw, spt, n_w, n_slots, slot_bytes, group;
  int32_t* status;
};
template <int N> struct UpRows { static constexpr int value = N; };      // rows of a thread that joins
struct __align__(16) UpBars {
  uint64_t full[kUpSlots], empty[kUpSlots], a_full[2], done[2], w_full[3], w_empty[3];
};
struct UpSmem {
  static constexpr int a_bytes = 2 * 2 * kRows * 128;                 // 2 stages of head and remainder
  static constexpr int misc = sizeof(UpBars) + 16 + kRows * (kUpHeld * 4 + 24);
  __host__ __device__ static constexpr int w_block(int d_h) { return (d_h + 63) / 64 * 8192; }
  __host__ __device__ static constexpr int n_w(int d_h) { return d_h <= 128 ? 3 : 2; }
  __host__ __device__ static constexpr int ring(int d_h) { return d_h <= 128 ? kUpRing : kUpRing - 32 * 1024; }
  __host__ __device__ static constexpr int total(int d_h) { return a_bytes + n_w(d_h) * w_block(d_h) + ring(d_h) + misc + 1024; }
};

template <int KS>
__global__ void __launch_bounds__(kUpThreads, 1)
tree_up_kernel(const __grid_constant__ CUtensorMap map_w, const UpArgs a) {
  extern __shared__ unsigned char smem_raw[];
  unsigned char* const base = (unsigned char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  const int wb = UpSmem::w_block(a.d_h);
  unsigned char* const s_w = base + UpSmem::a_bytes;
  unsigned char* const s_ring = s_w + a.n_w * wb;
  UpBars* const bars = (UpBars*)(s_ring + UpSmem::ring(a.d_h));
  uint32_t* const s_tmem = (uint32_t*)(bars + 1);
  volatile int* const s_abort = (volatile int*)(s_tmem + 1);
  float* const s_wt = (float*)(s_tmem + 4);              // [128][kUpHeld] normalised weights of a row's runs
  float2* const s_ml = (float2*)(s_wt + kRows * kUpHeld);       // [128] (M, 1 / L); M = -inf: the row sees nothing
  int2* const s_run = (int2*)(s_ml + kRows);             // [128] first run, runs
  int2* const s_lay = s_run + kRows;                     // [128] the head's first row in a run's partial results, its rows there
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int h = blockIdx.y, z = KS > 1 ? (int)cluster_ctarank() : 0;
  const int b0 = blockIdx.x * a.spt, n_seq = min(a.spt, a.B - b0), n_rows = n_seq * a.m;       // this block's sequences and rows
  const int chunks = (a.vw + 63) >> 6, c0 = chunks * z / KS, c1 = chunks * (z + 1) / KS;
  const uint32_t cols = a.d_h <= 32 ? 32 : a.d_h <= 64 ? 64 : a.d_h <= 128 ? 128 : 256;

  if (tid == 0) {
    for (int i = 0; i < kUpSlots; ++i) {
      mbar_init(smem_u32(&bars->full[i]), 1);
      mbar_init(smem_u32(&bars->empty[i]), kUpWarps);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&bars->a_full[i]), kUpWarps);
      mbar_init(smem_u32(&bars->done[i]), 1);
    }
    for (int i = 0; i < 3; ++i) {
      mbar_init(smem_u32(&bars->w_full[i]), 1);
      mbar_init(smem_u32(&bars->w_empty[i]), 1);
    }
    *s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async();
  }
  if (warp == kUpWarps + 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(s_tmem)), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *s_tmem;
  // W_uv's block of this block's q-th chunk (the layer's own copy: no kernel writes it)
  auto load_w = [&](int q) {
    const uint32_t fb = smem_u32(&bars->w_full[q % a.n_w]), dst = smem_u32(s_w) + (uint32_t)(q % a.n_w) * wb;
    mbar_expect_tx(fb, (uint32_t)wb);
    for (int j = 0; j < wb / 8192; ++j) tma_load_2d(dst + j * 8192, &map_w, h * a.d_h + j * 64, (c0 + q) * 64, fb);
  };
  const int mine = c1 - c0;
  if (tid == 32 * (kUpWarps + 1))
    for (int q = 0; q < mine && q < a.n_w - 1; ++q) load_w(q);
  ekv_pdl_wait();
  ekv_pdl_trigger();

  // ---- a row's runs, its largest reference and its sum
  if (tid < kRows) {
    int2 run = make_int2(0, 0), lay = make_int2(0, 0);
    float M = -1e30f, L = 0.f;
    float2 held[kUpHeld];
#pragma unroll
    for (int k = 0; k < kUpHeld; ++k) held[k] = make_float2(-1e30f, 0.f);
    const float2* ml = a.part_ml;
    const long long pitch = (long long)a.n_half * kRows;
    int seen = 0;                          // runs that hold the row: none of a node that its sequence's layout leaves out
    if (tid < n_rows) {
      const int b = b0 + tid / a.m, i = tid % a.m;
      run.x = __ldcg(a.seq_first + b);
      run.y = __ldcg(a.seq_first + b + 1) - run.x;
      const TreeLayout& l = a.lay.of[__ldcg(a.seq_lay + b)];
      const int half = h / l.hb;
      lay = make_int2(half * kRows + (h - half * l.hb) * l.m, l.m);
      if (i < l.m) seen = run.y;
      ml += run.x * pitch + lay.x + i;
#pragma unroll
      for (int k = 0; k < kUpHeld; ++k)
        if (k < seen) held[k] = __ldcg(ml + k * pitch);
#pragma unroll
      for (int k = 0; k < kUpHeld; ++k) M = fmaxf(M, held[k].x);
      for (int k = kUpHeld; k < seen; ++k) M = fmaxf(M, __ldcg(ml + k * pitch).x);
#pragma unroll
      for (int k = 0; k < kUpHeld; ++k) L = fmaf(held[k].y, exp2f(held[k].x - M), L);
      for (int k = kUpHeld; k < seen; ++k) {
        const float2 x = __ldcg(ml + k * pitch);
        L = fmaf(x.y, exp2f(x.x - M), L);
      }
    }
    const float inv = L != 0.f ? 1.f / L : 0.f;          // (nothing seen: a zero row)
#pragma unroll
    for (int k = 0; k < kUpHeld; ++k) s_wt[tid * kUpHeld + k] = k < seen ? exp2f(held[k].x - M) * inv : 0.f;
    s_ml[tid] = make_float2(L != 0.f ? M : -INFINITY, inv);
    s_run[tid] = run;
    s_lay[tid] = lay;
  }
  __syncthreads();
  int most = 0;
  for (int k = lane; k < n_rows; k += 32) most = max(most, s_run[k].y);
  most = __reduce_max_sync(0xffffffffu, most);
  const int steps = max((most + a.group - 1) / a.group, 1);     // units of a chunk (no runs at all: a tile of zeros)
  bool ok = true;
  // normalised weight of a row's k-th run (0: there is none)
  auto weight = [&](int row, int k) -> float {
    if (k < kUpHeld) return s_wt[row * kUpHeld + k];
    if (k >= s_run[row].y || s_ml[row].x == -INFINITY) return 0.f;
    return exp2f(__ldcg(a.part_ml + (long long)(s_run[row].x + k) * a.n_half * kRows + s_lay[row].x + row % a.m).x - s_ml[row].x) * s_ml[row].y;
  };

  if (warp == kUpWarps) {
    // ---- partial results: unit (chunk, `group` runs of every sequence).  A lane copies up to four (run, sequence) pairs.
    const float* src[4];
    int left[4], to[4];                    // runs of the sequence from this one on; place in the unit
    unsigned bytes[4];
    const int pairs = a.group * n_seq;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int x = lane + 32 * t, g = x / n_seq, e = x - g * n_seq;
      const int2 run = x < pairs ? s_run[e * a.m] : make_int2(0, 0);
      left[t] = x < pairs ? run.y - g : 0;
      to[t] = (g * n_rows + e * a.m) * 256;
      const int2 lay = x < pairs ? s_lay[e * a.m] : make_int2(0, 0);
      bytes[t] = (unsigned)lay.y * 256;
      src[t] = a.part_acc + (((long long)run.x + g) * a.n_half + lay.x / kRows) * chunks * kRows * 64 + lay.x % kRows * 64;
    }
    const long long run_pitch = (long long)a.n_half * chunks * kRows * 64;
    int slot = 0;
    uint32_t turn = 1;
    for (int q = 0; q < mine && ok; ++q)
      for (int k = 0; k < steps; ++k) {
        ok = warp_wait(smem_u32(&bars->empty[slot]), turn, s_abort, 1);
        if (!ok) break;
        const int k0 = k * a.group;
        unsigned n = 0;
#pragma unroll
        for (int t = 0; t < 4; ++t)
          if (left[t] > k0) n += bytes[t];
        n = __reduce_add_sync(0xffffffffu, n);
        const uint32_t fb = smem_u32(&bars->full[slot]), dst = smem_u32(s_ring) + (uint32_t)slot * a.slot_bytes;
        if (lane == 0) mbar_expect_tx(fb, n);
        __syncwarp();
#pragma unroll
        for (int t = 0; t < 4; ++t)
          if (left[t] > k0) bulk_load(dst + to[t], src[t] + k0 * run_pitch + (long long)(c0 + q) * kRows * 64, bytes[t], fb);
        __syncwarp();
        if (++slot == a.n_slots) { slot = 0; turn ^= 1; }
      }
  } else if (warp == kUpWarps + 1) {
    // ---- products
    const uint32_t idesc = make_idesc(kRows, 16, 0, 1) + ((uint32_t)((a.d_h >> 3) - 2) << 17);
    constexpr uint32_t hi_sw = desc_hi(1024, 2);
    for (int q = 0; q < mine && ok; ++q) {
      const int st = q & 1;
      ok = warp_wait(smem_u32(&bars->a_full[st]), (q >> 1) & 1, s_abort, 2) &&
           warp_wait(smem_u32(&bars->w_full[q % a.n_w]), (q / a.n_w) & 1, s_abort, 3);
      if (!ok) break;
      tc_fence_after();
      if (elect_one()) {
        const uint32_t la = desc_lo(smem_u32(base) + st * 2 * kRows * 128, 16), lb = desc_lo(smem_u32(s_w) + (uint32_t)(q % a.n_w) * wb, 8192);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          tc_mma_w(tmem, la + 2 * k, hi_sw, lb + 128 * k, hi_sw, idesc, q != 0 || k != 0);
          tc_mma_w(tmem, la + (kRows * 128 >> 4) + 2 * k, hi_sw, lb + 128 * k, hi_sw, idesc, 1);
        }
        tc_commit(smem_u32(&bars->done[st]));
        tc_commit(smem_u32(&bars->w_empty[q % a.n_w]));
      }
      __syncwarp();
    }
  } else if (warp == kUpWarps + 2) {
    // ---- W_uv: a block goes where the products n_w chunks before read theirs
    for (int q = a.n_w - 1; q < mine && ok; ++q) {
      if (q >= a.n_w) ok = warp_wait(smem_u32(&bars->w_empty[q % a.n_w]), (q / a.n_w - 1) & 1, s_abort, 4);
      if (ok && lane == 0) load_w(q);
      __syncwarp();
    }
  } else {
    // ---- rows joined and laid out: a thread has 4 of a chunk's columns of the rows row_t + 32 p, p < P
    const int col4 = tid & 15, row_t = tid >> 4;
    constexpr int kStep = 2 * kUpWarps;
    int least = most;                      // runs that every sequence has
    for (int k = lane; k < n_rows; k += 32) least = min(least, s_run[k].y);
    least = __reduce_min_sync(0xffffffffu, least);
    auto join = [&](auto rows_per_thread) {
      constexpr int P = decltype(rows_per_thread)::value, U = 4 / P;      // U runs at a time
      int off[P];                          // of a row in a run's share of a unit
      bool none[P];                        // the row sees nothing (its place may hold anything)
#pragma unroll
      for (int p = 0; p < P; ++p) {
        off[p] = min(row_t + kStep * p, n_rows - 1) * 256 + col4 * 16;
        none[p] = s_ml[row_t + kStep * p].x == -INFINITY;
      }
      const float* const wt = s_wt + row_t * kUpHeld;
      int slot = 0;
      uint32_t turn = 0;
      for (int q = 0; q < mine; ++q) {
        const int st = q & 1;
        const bool in = (c0 + q) * 64 + col4 * 4 < a.vw;
        // all rows of all runs hold values: nothing has to be kept out
        const int plain = (c0 + q) * 64 + 64 <= a.vw ? min(least, kUpHeld) : 0;
        float4 acc[P];
#pragma unroll
        for (int p = 0; p < P; ++p) acc[p] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
        for (int k = 0; k < steps; ++k) {
          ok = ok && mbar_wait(smem_u32(&bars->full[slot]), turn, s_abort, 5);
          const unsigned char* src = s_ring + (size_t)slot * a.slot_bytes;
          const int k0 = k * a.group, n_g = min(a.group, most - k0);
#pragma unroll 1
          for (int g = 0; g < n_g; g += U, src += U * n_rows * 256) {
            if (g + U <= n_g && k0 + g + U <= plain) {
#pragma unroll
              for (int e = 0; e < U; ++e)
#pragma unroll
                for (int p = 0; p < P; ++p) {
                  const float4 y = *(const float4*)(src + e * n_rows * 256 + off[p]);
                  const float v = wt[kStep * p * kUpHeld + k0 + g + e];
                  acc[p].x = fmaf(y.x, v, acc[p].x); acc[p].y = fmaf(y.y, v, acc[p].y);
                  acc[p].z = fmaf(y.z, v, acc[p].z); acc[p].w = fmaf(y.w, v, acc[p].w);
                }
            } else {
#pragma unroll 1
              for (int e = 0; e < U && g + e < n_g; ++e)
#pragma unroll
                for (int p = 0; p < P; ++p) {
                  const float v = in ? weight(row_t + kStep * p, k0 + g + e) : 0.f;
                  if (v != 0.f) {          // (else the place may hold anything)
                    const float4 y = *(const float4*)(src + e * n_rows * 256 + off[p]);
                    acc[p].x = fmaf(y.x, v, acc[p].x); acc[p].y = fmaf(y.y, v, acc[p].y);
                    acc[p].z = fmaf(y.z, v, acc[p].z); acc[p].w = fmaf(y.w, v, acc[p].w);
                  }
                }
            }
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&bars->empty[slot]));
          if (++slot == a.n_slots) { slot = 0; turn ^= 1; }
        }
        // the products of chunk q - 2 have read the stage
        if (q >= 2) ok = ok && mbar_wait(smem_u32(&bars->done[st]), ((q >> 1) - 1) & 1, s_abort, 6);
        unsigned char* const hi = base + st * 2 * kRows * 128;
#pragma unroll
        for (int p = 0; p < P; ++p) {      // (rows of nobody hold anything)
          const int row = row_t + kStep * p;
          const float4 v = none[p] ? make_float4(0.f, 0.f, 0.f, 0.f) : acc[p];
          const bf162 h0 = __floats2bfloat162_rn(v.x, v.y), h1 = __floats2bfloat162_rn(v.z, v.w);
          const float2 f0 = __bfloat1622float2(h0), f1 = __bfloat1622float2(h1);
          const bf162 l0 = __floats2bfloat162_rn(v.x - f0.x, v.y - f0.y), l1 = __floats2bfloat162_rn(v.z - f1.x, v.w - f1.y);
          const int at = row * 128 + (((col4 >> 1) ^ (row & 7)) << 4) + (col4 & 1) * 8;
          *(uint2*)(hi + at) = make_uint2(*(const uint32_t*)&h0, *(const uint32_t*)&h1);
          *(uint2*)(hi + kRows * 128 + at) = make_uint2(*(const uint32_t*)&l0, *(const uint32_t*)&l1);
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars->a_full[st]));
      }
    };
    static_assert(kRows == 4 * kStep, "rows per thread");
    if (n_rows <= kStep) join(UpRows<1>());
    else if (n_rows <= 2 * kStep) join(UpRows<2>());
    else join(UpRows<4>());
    // the last products of both stages
    if (mine >= 2) ok = ok && mbar_wait(smem_u32(&bars->done[mine & 1]), ((mine - 2) >> 1) & 1, s_abort, 7);
    if (mine >= 1) ok = ok && mbar_wait(smem_u32(&bars->done[(mine - 1) & 1]), ((mine - 1) >> 1) & 1, s_abort, 8);
  }
  __syncwarp();
  tc_fence_after();
  ok = __syncthreads_and(ok) != 0;

  const int quarter = warp & 3, part = warp >> 2;        // rows of a warp; kUpWarps / 4 warps share their columns, 8 at a time
  constexpr int kParts = kUpWarps / 4;
  const int row = quarter * 32 + lane;
  bf16* const dst = a.out + (((long long)b0 * a.m + row) * a.n_h + h) * a.d_h;
  const uint32_t tm = tmem + ((uint32_t)(quarter * 32) << 16);
  const bool wide = ((uintptr_t)a.out & 15) == 0;        // (rows are whole 32 bytes; the caller's `out` is on 4)
  auto store8 = [&](bf16* to, const float* v) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bf162 y = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
      w[e] = *(const uint32_t*)&y;
    }
    if (wide) {
      *(uint4*)to = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) ((uint32_t*)to)[e] = w[e];
    }
  };
  if (KS == 1) {
    for (int c = part * 16; c < a.d_h && ok && warp < kUpWarps; c += 16 * kParts) {
      float v[16];
      tc_ld16(tm + c, v);
      tc_wait_ld();
      if (row < n_rows) {
        store8(dst + c, v);
        store8(dst + c + 8, v + 8);
      }
      __syncwarp();
    }
  } else {
    // every block sends its sums of columns [q w, (q + 1) w) to block q
    const int w = a.d_h / KS;
    float* const recv = (float*)base;                    // [source][column][row], over stages and ring
    static_assert(kRows * 256 * 4 <= UpSmem::a_bytes + kUpRing - 32 * 1024, "the sums of a tile fit");
    cluster_sync_all();                                  // all bulk copies have landed and all products are done in every block
    for (int c = part * 8; c < a.d_h && warp < kUpWarps; c += 8 * kParts) {
      float v[8];
      tc_ld8(tm + c, v);
      tc_wait_ld();
      // (w is a multiple of 8: the columns have one owner)
      const int q = c / w;
      const uint32_t to = map_to_cta(smem_u32(recv + ((size_t)z * w + c - q * w) * kRows + row), (uint32_t)q);
#pragma unroll
      for (int e = 0; e < 8; ++e) st_cluster_u32(to + e * kRows * 4, __float_as_uint(v[e]));
    }
    __syncwarp();
    cluster_sync_all();
    if (row < n_rows && ok && warp < kUpWarps) {
      for (int k = part * 8; k < w; k += 8 * kParts) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[e] = recv[(size_t)(k + e) * kRows + row];
#pragma unroll
          for (int q = 1; q < KS; ++q) v[e] += recv[((size_t)q * w + k + e) * kRows + row];
        }
        store8(dst + z * w + k, v);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (*s_abort) drain_after_abort();
  if (tid == 0 && *s_abort) ekv_record(a.status, ELITEKV_ERR_TIMEOUT, (int)blockIdx.x | (*s_abort << 16), (int)blockIdx.y);
  if (warp == kUpWarps + 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
  }
}

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// rows of a block are whole heads; one block where it holds all of them, else pairs
struct TreeShape {
  int cg, n_rb, n_ct, workers, want;
  TreeLayouts lay;
};
TreeShape tree_shape(const elitekv_layer* L, int m) {
  TreeShape s;
  const int most = kRows / m, blocks = (L->n_h + most - 1) / most;
  s.cg = blocks == 1 ? 1 : 2;
  s.n_rb = (blocks + s.cg - 1) / s.cg;
  s.lay.n = s.lay.tiles = 0;
  for (int k = m; k >= 1 && s.lay.n < kLayouts; --k) {
    const int n = (L->n_h + kRows / k - 1) / (kRows / k), n_rb = (n + s.cg - 1) / s.cg;
    if (s.lay.n > 0 && n_rb * 5 > s.lay.of[s.lay.n - 1].n_rb * 4) continue;
    TreeLayout& l = s.lay.of[s.lay.n++];
    l.m = k;
    l.n_rb = n_rb;
    l.hb = (L->n_h + n_rb * s.cg - 1) / (n_rb * s.cg);
    l.n_rc = 0;
    for (int rb = 0; rb < n_rb && L->r > 0; ++rb) {
      const int h0 = rb * s.cg * l.hb, h1 = h0 + s.cg * l.hb < L->n_h ? h0 + s.cg * l.hb : L->n_h;
      const int steps = h1 > h0 ? (h1 * 2 * L->r - tree_rope_col(h0, 2 * L->r) + 63) / 64 : 0;
      l.n_rc = steps > l.n_rc ? steps : l.n_rc;
    }
    if (n_rb * s.cg * l.n_rc > s.lay.tiles) s.lay.tiles = n_rb * s.cg * l.n_rc;
  }
  s.n_ct = (L->vw + kTile - 1) / kTile;
  s.workers = L->sm_count / s.cg;
  s.want = s.workers / (s.n_rb * s.n_ct);
  if (s.want < 1) s.want = 1;
  return s;
}

struct TreeCarve {
  size_t hdr, runs, first, lay, zero, n_zero, stats, pref, cstate, P, qr, ml, acc, total;
  size_t max_runs;
};
TreeCarve tree_carve(const elitekv_layer* L, const TreeShape& s, int B, int m) {
  TreeCarve c;
  c.max_runs = (size_t)B + s.want;
  const size_t chains = c.max_runs * s.n_rb * s.n_ct;
  size_t o = 0;
  c.hdr = o;    o = align256(o + 16);
  c.runs = o;   o = align256(o + c.max_runs * 32);
  c.first = o;  o = align256(o + sizeof(int32_t) * ((size_t)B + 1));
  c.lay = o;    o = align256(o + sizeof(int32_t) * (size_t)B);
  c.n_zero = (size_t)kSlots * (s.cg + 2) + chains;
  c.zero = o;   o = align256(o + sizeof(int) * c.n_zero);
  c.stats = o;  o = align256(o + sizeof(float2) * kSlots * s.cg * kTiles * kRows);
  c.pref = o;   o = align256(o + sizeof(float2) * kSlots * s.cg * kRows);
  c.cstate = o; o = align256(o + sizeof(float2) * chains * s.cg * kRows);
  c.P = o;      o = align256(o + sizeof(bf16) * (size_t)kSlots * s.cg * kRows * kPiece);
  c.qr = o;     o = align256(o + sizeof(bf16) * (size_t)B * s.lay.tiles * kRows * 64);
  const size_t tile_rows = c.max_runs * s.n_rb * s.cg * kRows;
  c.ml = o;     o = align256(o + sizeof(float2) * tile_rows);
  c.acc = o;    o = align256(o + sizeof(float) * tile_rows * ((L->vw + 63) / 64) * 64);
  c.total = o;
  return c;
}

// bf16 [rows][cols] with `pitch` elements from row to row, box [box_rows][64], 128-byte swizzle
int make_map_pitch(CUtensorMap* m, const void* ptr, unsigned long long rows, unsigned long long cols, unsigned long long pitch, unsigned box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return ELITEKV_ERR_CUDA;
  cuuint64_t dims[2] = {cols, rows}, strides[1] = {pitch * sizeof(bf16)};
  cuuint32_t box[2] = {64, box_rows}, estr[2] = {1, 1};
  CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? ELITEKV_OK : ELITEKV_ERR_CUDA;
}
// [rows][cols], box of 32 rows x 128 bytes, 128-byte swizzle: what the epilogue warps write
int make_map_box(CUtensorMap* m, CUtensorMapDataType type, const void* ptr, unsigned long long rows, unsigned long long cols, unsigned size) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return ELITEKV_ERR_CUDA;
  cuuint64_t dims[2] = {cols, rows}, strides[1] = {cols * size};
  cuuint32_t box[2] = {128 / size, 32}, estr[2] = {1, 1};
  CUresult r = fn(m, type, 2, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? ELITEKV_OK : ELITEKV_ERR_CUDA;
}
// bf16 [rows][cols / 64][64] with `pitch` elements from row to row, box [chunks][64 rows][64]: whole chunks of 64 columns
int make_map_chunks(CUtensorMap* m, const void* ptr, unsigned long long rows, unsigned long long cols, unsigned long long pitch, unsigned chunks) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return ELITEKV_ERR_CUDA;
  cuuint64_t dims[3] = {64, rows, cols / 64}, strides[2] = {pitch * sizeof(bf16), 128};
  cuuint32_t box[3] = {64, 64, chunks}, estr[3] = {1, 1, 1};
  CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? ELITEKV_OK : ELITEKV_ERR_CUDA;
}
// queries [B][m][n_h][kw] seen as (sequence, head, node, latent): a box is `hb` heads, the first `nodes` nodes of each
int make_map_queries(CUtensorMap* map, const void* ptr, int B, int m, int n_h, int kw, int hb, int nodes) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return ELITEKV_ERR_CUDA;
  cuuint64_t dims[4] = {(cuuint64_t)kw, (cuuint64_t)m, (cuuint64_t)n_h, (cuuint64_t)B};
  cuuint64_t strides[3] = {(cuuint64_t)n_h * kw * 2, (cuuint64_t)kw * 2, (cuuint64_t)m * n_h * kw * 2};
  cuuint32_t box[4] = {64, (cuuint32_t)nodes, (cuuint32_t)hb, 1}, estr[4] = {1, 1, 1, 1};
  CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? ELITEKV_OK : ELITEKV_ERR_CUDA;
}

unsigned long long plane_rows(const CacheView& cv) {
  return cv.page_table ? (unsigned long long)cv.num_pages << cv.page_shift : (unsigned long long)cv.max_ctx * cv.n_seqs;
}

}  // namespace

size_t ekv_tree_tc_bytes(const elitekv_layer* L, int B, int m) { return tree_carve(L, tree_shape(L, m), B, m).total; }

// Pages of 8 tokens and more: a box of the copy engine is whole 1024-byte groups of the swizzle.  Box coordinates have 32 bits,
// rope rows whole 16 bytes.
int ekv_tree_tc_supported(const elitekv_layer* L, int B, int m, const CacheView* cv) {
  const TreeShape s = tree_shape(L, m);
  if (((unsigned long long)B + s.want) * s.n_rb * s.cg * ((L->vw + 63) / 64) * kRows >= (1ull << 31) ||
      (unsigned long long)B * s.lay.tiles * kRows >= (1ull << 31) || L->n_h > 65535)
    return 0;
  if ((L->n_h * L->r) % 4 != 0) return 0;
  if (L->d_h % 16 != 0 || L->d_h > 256) return 0;          // the last product's width
  if (TreeSmem<1>::total > L->smem_optin || TreeSmem<2>::total > L->smem_optin || UpSmem::total(L->d_h) > L->smem_optin) return 0;
  if (cv && cv->page_table && (1 << cv->page_shift) < 8) return 0;
  if (cv && (plane_rows(*cv) >= (1ull << 31) || cv->max_ctx > (1ll << 30))) return 0;
  return 1;
}

int ekv_launch_tree_tc(const elitekv_layer* L, const elitekv_cache* cache, const CacheView& cv, const TreeCall& c, cudaStream_t st) {
  TreeShape s = tree_shape(L, c.m);
  const TreeCarve w = tree_carve(L, s, c.B, c.m);
  if (c.n_nodes == nullptr) s.lay.n = 1;
  unsigned char* const base = (unsigned char*)c.workspace;
  const int page = cv.page_table ? 1 << cv.page_shift : 1 << 30;
  TreeTcArgs a;
  a.cv = cv;
  a.q_rope = (const bf16*)c.q_rope;
  a.q_abs = (const bf16*)c.q_abs;
  a.rope = (const bf16*)cache->rope;
  a.latent = (const bf16*)cache->latent;
  a.mask = c.mask;
  a.m = c.m;
  a.d_c = L->d_c;
  a.n_h = L->n_h;
  a.r2 = 2 * L->r;
  a.kw = L->kw;
  a.vw = L->vw;
  a.lay = s.lay;
  a.n_rb = s.n_rb;
  a.n_ct = s.n_ct;
  a.box_s = page < 128 ? page : 128;
  a.box_v = page < 64 ? page : 64;
  a.scale_log2e = L->scale * 1.4426950408889634f;
  a.P = (bf16*)(base + w.P);
  a.stats = (float2*)(base + w.stats);
  a.pref = (float2*)(base + w.pref);
  a.cstate = (float2*)(base + w.cstate);
  a.s_cnt = (int*)(base + w.zero);
  a.ready = a.s_cnt + kSlots * s.cg;
  a.v_done = a.ready + kSlots;
  a.chain = a.v_done + kSlots;
  a.part_acc = (float*)(base + w.acc);
  a.part_ml = (float2*)(base + w.ml);
  a.hdr = (const int*)(base + w.hdr);
  a.runs = (const int4*)(base + w.runs);
  a.status = L->d_status;
  TreeQueryMaps m_q;
  CUtensorMap m_k, m_v, m_p, m_qr, m_r, m_ps, m_o, m_w;
  a.v3 = a.box_v == 64 && L->vw % 64 == 0;
  const unsigned long long p_rows = (unsigned long long)kSlots * s.cg * (kPiece / 64) * kRows;
  const unsigned long long blk_rows = (unsigned long long)w.max_runs * s.n_rb * s.cg * ((L->vw + 63) / 64) * kRows;
  const unsigned long long rows = plane_rows(cv);
  int rc = ELITEKV_OK;
  for (int k = 0; k < kLayouts && rc == ELITEKV_OK; ++k) {
    if (k < s.lay.n) rc = make_map_queries(&m_q.of[k], c.q_abs, c.B, c.m, L->n_h, L->kw, s.lay.of[k].hb, s.lay.of[k].m);
    else m_q.of[k] = m_q.of[0];
  }
  if (rc == ELITEKV_OK) rc = make_map_pitch(&m_k, cache->latent, rows, L->kw, L->d_c, a.box_s);
  if (rc == ELITEKV_OK)
    rc = a.v3 ? make_map_chunks(&m_v, (const bf16*)cache->latent + L->voff, rows, L->vw, L->d_c, 4 / s.cg)
              : make_map_pitch(&m_v, (const bf16*)cache->latent + L->voff, rows, L->vw, L->d_c, a.box_v);
  if (rc == ELITEKV_OK) rc = make_map_box(&m_ps, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, a.P, p_rows, 64, 2);
  if (rc == ELITEKV_OK) rc = make_map_box(&m_o, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, a.part_acc, blk_rows, 64, 4);
  if (rc == ELITEKV_OK) rc = make_map_pitch(&m_w, L->d_Wuv, L->vw, (unsigned long long)L->n_h * L->d_h, (unsigned long long)L->n_h * L->d_h, 64);
  if (rc == ELITEKV_OK) rc = make_map_pitch(&m_p, a.P, p_rows, 64, 64, kRows);
  // (a layer without rope has neither; the maps are not used)
  m_qr = m_r = m_p;
  if (rc == ELITEKV_OK && s.lay.tiles > 0) {
    rc = make_map_pitch(&m_qr, base + w.qr, (unsigned long long)c.B * s.lay.tiles * kRows, 64, 64, kRows);
    if (rc == ELITEKV_OK) rc = make_map_pitch(&m_r, cache->rope, rows, (unsigned long long)L->n_h * a.r2, (unsigned long long)L->n_h * a.r2, a.box_s);
  }
  if (rc != ELITEKV_OK) return rc;
  TreePrepArgs p;
  p.q_rope = (const bf16*)c.q_rope;
  p.qr = (bf16*)(base + w.qr);
  p.cg = s.cg;
  p.n_h = L->n_h;
  p.r2 = a.r2;
  p.lay = s.lay;
  p.seq_lens = c.seq_lens;
  p.n_nodes = c.n_nodes;
  p.B = c.B;
  p.m = c.m;
  p.n_ct = s.n_ct;
  p.want = s.want;
  p.workers = s.workers;
  p.max_len = cv.max_ctx;
  p.hdr = (int*)(base + w.hdr);
  p.runs = (int4*)(base + w.runs);
  p.seq_first = (int32_t*)(base + w.first);
  p.seq_lay = (int32_t*)(base + w.lay);
  p.zero = a.s_cnt;
  p.n_zero = (int)w.n_zero;
  p.status = L->d_status;
  const int zero_blocks = (p.n_zero + 1023) / 1024;
  p.zero_blocks = zero_blocks < 32 ? zero_blocks : 32;
  const long long qr_blocks = ((long long)c.B * s.lay.tiles * kRows * 8 + 1023) / 1024;
  EKV_CUDA_OK(ekv_launch_pdl(tree_prep_kernel, dim3((unsigned)(1 + p.zero_blocks + (qr_blocks < 1024 ? qr_blocks : 1024))), dim3(256), 0, st, p));
  const int smem = s.cg == 2 ? TreeSmem<2>::total : TreeSmem<1>::total;
  auto launch = [&](auto kern) -> int {
    EKV_CUDA_OK(ekv_allow_smem(kern, smem));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(s.workers * s.cg));
    cfg.blockDim = dim3(kTreeThreads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)s.cg;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    EKV_CUDA_OK(cudaLaunchKernelEx(&cfg, kern, m_q, m_k, m_v, m_p, m_qr, m_r, m_ps, m_o, a));
    return ELITEKV_OK;
  };
  rc = s.cg == 2 ? launch(tree_tc_kernel<2>) : launch(tree_tc_kernel<1>);
  if (rc != ELITEKV_OK) return rc;
  EKV_CUDA_OK(cudaGetLastError());
  UpArgs u;
  u.part_acc = a.part_acc;
  u.part_ml = a.part_ml;
  u.seq_first = p.seq_first;
  u.out = (bf16*)c.out;
  u.B = c.B;
  u.m = c.m;
  u.n_h = L->n_h;
  u.d_h = L->d_h;
  u.seq_lay = p.seq_lay;
  u.lay = s.lay;
  u.n_half = s.n_rb * s.cg;
  u.vw = L->vw;
  u.status = L->d_status;
  u.n_w = UpSmem::n_w(L->d_h);
  // Sequences per tile and shares of the depth: in steps of a whole tile's 64 latents, a block takes one per 64 latents, less
  // when it has fewer rows, and about four to start and end.
  const int chunks = (L->vw + 63) / 64, most = kRows / c.m;
  int ks = 1;
  float best = 0.f;
  for (int k = 1; k <= 4 && k <= chunks; k *= 2) {
    if (L->d_h % (8 * k) != 0) break;
    for (int spt = most; spt >= 1 && spt * 4 >= most; --spt) {
      const long long tiles = L->n_h * (((long long)c.B + spt - 1) / spt);
      const float t = (float)((tiles * k + L->sm_count - 1) / L->sm_count) * ((float)((chunks + k - 1) / k) * (0.3f + 0.7f * (float)(spt * c.m) / kRows) + 4.f);
      if ((k == 1 && spt == most) || t < best) { best = t; ks = k; u.spt = spt; }
      if (spt > 8) spt = (spt + 1) / 2 + 1;
    }
  }
  const int up_rows = (c.B < u.spt ? c.B : u.spt) * c.m;
  u.group = kRows / up_rows < kUpHeld ? kRows / up_rows : kUpHeld;      // runs that a slot holds
  u.slot_bytes = u.group * up_rows * 256;
  u.n_slots = UpSmem::ring(L->d_h) / u.slot_bytes < kUpSlots ? UpSmem::ring(L->d_h) / u.slot_bytes : kUpSlots;
  const long long groups = ((long long)c.B + u.spt - 1) / u.spt;
  auto launch_up = [&](auto kern) -> int {
    const size_t sm = UpSmem::total(L->d_h);
    EKV_CUDA_OK(ekv_allow_smem(kern, sm));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)groups, (unsigned)L->n_h, (unsigned)ks);
    cfg.blockDim = dim3(kUpThreads);
    cfg.dynamicSmemBytes = sm;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 1;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = (unsigned)ks;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    EKV_CUDA_OK(cudaLaunchKernelEx(&cfg, kern, m_w, u));
    EKV_CUDA_OK(cudaGetLastError());
    return ELITEKV_OK;
  };
  return ks == 4 ? launch_up(tree_up_kernel<4>) : ks == 2 ? launch_up(tree_up_kernel<2>) : launch_up(tree_up_kernel<1>);
}

// What each block of tree attention's tensor-core form loads in a step of a unit (apart from the device code, so that the
// rule can be looked at without one).
//
// A stage of the ring is free again when the products have read it.  The load warps of both blocks wait for that by a phase's
// parity, which tells a phase from the one before only: a warp must never be two phases late.  What holds it is
// that a step's products cannot start without the bytes of EVERY load warp, so each of them loads at least one box in each
// step, also where its block has nothing of the unit (a tile that ends in the first block's half; a last tile of up to 64
// latents): such a box lies outside the tensor, which fills zeros and reads nothing.
#pragma once

#ifdef __CUDACC__
#define EKV_HD __host__ __device__ __forceinline__
#else
#define EKV_HD inline
#endif

// Boxes of `box` tokens that a block loads of a score tile: `half` tokens are its share, `left` tokens of the sequence are left
// from the first of them on (none: 0 or less).
EKV_HD int tree_score_boxes(int left, int half, int box) {
  const int n = left > 0 ? (left + box - 1) / box : 1, most = half / box;
  return n < most ? n : most;
}
// of both blocks (cg = 1: of the one)
EKV_HD int tree_score_boxes_all(int left, int tile, int box, int cg) {
  return cg == 1 ? tree_score_boxes(left, tile, box) : tree_score_boxes(left, tile / 2, box) + tree_score_boxes(left - tile / 2, tile / 2, box);
}

// 64-column chunks of a value tile: `held` of them (up to four) hold columns, and a block of a pair has half of four, or one where two are
// enough.
EKV_HD int tree_value_share(int held, int cg) { return held <= 2 ? 2 / cg : 4 / cg; }
EKV_HD int tree_value_chunks(int held, int cg, int rank) {
  const int share = tree_value_share(held, cg), n = held - share * rank;
  return n < 1 ? 1 : n < share ? n : share;
}
EKV_HD int tree_value_chunks_all(int held, int cg) {
  return cg == 1 ? tree_value_chunks(held, 1, 0) : tree_value_chunks(held, 2, 0) + tree_value_chunks(held, 2, 1);
}

// Attention of packed sequences, forward and backward (gfx950).
//
// Sequences of different lengths lie one behind the other; the plan (packed_plan.hip) has cut them into tiles and put
// these in an order, heaviest first.  A token of a sequence of nq queries and nk keys has the place i + nk - nq among
// the keys (the queries are the last tokens) and sees the keys of chunks up to its own: the first
//   sees(i) = min(nk, (place / L + 1) L), none if place < 0
// of them, so that tiles above the diagonal are skipped and only steps on it are masked.  Rows of a tile are the tokens
// of the query heads that share a key head (attn_rows.h), whose gradients are thereby sums over more rows.
#pragma once

#include "attn_rows.h"

namespace mw {

// What a workgroup does for key head hk; false: nothing (the grid is sized for the most items there can be).
__device__ __forceinline__ bool work_item(const int* list, int bid, int Hkv, int& hk, PackedItem& it) {
  int rank;
  tile_item(bid, Hkv, hk, rank);
  if (rank >= list[0]) return false;
  it = reinterpret_cast<const PackedItem*>(list + 8)[rank];
  return true;
}

// How many keys the token of row r sees.
__device__ __forceinline__ int sees(int r, int G, int nq, int nk, int L) {
  const int place = (G == 1 ? r : (int)((unsigned)r / (unsigned)G)) + nk - nq;
  return place < 0 ? 0 : min(nk, (int)((unsigned)place / (unsigned)L + 1) * L);
}

// Offset of row r of key head hk of a sequence that begins at token q0, in a [total, H, D] view.
__device__ __forceinline__ long long packed_offset(const Strides& s, int hk, int G, int q0, int r) {
  const int t = G == 1 ? r : (int)((unsigned)r / (unsigned)G);
  return (long long)(hk * G + (r - t * G)) * s.h + (long long)(q0 + t) * s.t;
}

// Workgroups of 256 threads, four columns each, that join a tile of n rows.
constexpr int join_blocks(int n, int D) { return (n * (D / 4) + 255) / 256; }
// How many tiles are cut only the device knows: at most that many workgroups take what there is in turns.  (One workgroup
// for each that there could be, 8192 of 19200 prompt tokens, most of them empty: the call 406 for 404 us.)
constexpr int kJoinGrid = 1024;

}  // namespace mw

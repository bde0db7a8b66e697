// packed_order.h -- the backward over packed sequences: which query blocks a KV
// tile's chain visits, their places in the summation order, and the order in
// which the chains are started.  Usable on host and device.
//
// A sequence of nq queries and nk keys (causal: query i sees key j iff j <= i + off,
// off = nk - nq) has ceil(nk / bc) KV tiles.  Tile j's chain visits the 64-row query
// blocks from the last one down to the first that sees it, each block for all query
// heads of the group; a block's dQ is the sum over its tiles in ascending order
// (Descending Q-Tile Iteration, Section 3.3 of the paper).  A chain therefore
// waits only on the chain of the tile before it, which order_of starts earlier.
#pragma once

#if defined(__HIPCC__)
#define DASH_ORDER_HD __host__ __device__ inline
#else
#define DASH_ORDER_HD inline
#endif

namespace dash {

struct SeqGeom {
  int nq, nk;
  bool causal;
  int bc;  // rows of a KV tile
  DASH_ORDER_HD int off() const { return nk - nq; }
  DASH_ORDER_HD int blocks() const { return (nq + 63) / 64; }
  DASH_ORDER_HD int tiles() const { return (nk + bc - 1) / bc; }
  // the first query block that sees a key of tile j (blocks(): none does)
  DASH_ORDER_HD int first_block(int j) const {
    if (!causal) return 0;
    const int row = j * bc - off();  // the first query that sees the tile's first key
    const int b = row > 0 ? row / 64 : 0;
    return row < nq ? b : blocks();
  }
  // blocks that tile j's chain visits; does not rise with j
  DASH_ORDER_HD int chain(int j) const { return blocks() - first_block(j); }
  // the last tile that block pb sees (-1: none); its rank is j, as every tile before j
  // is seen too
  DASH_ORDER_HD int last_tile(int pb) const {
    if (!causal) return tiles() - 1;
    const int row = pb * 64 + 63 < nq ? pb * 64 + 63 : nq - 1;
    return row + off() < 0 ? -1 : (row + off()) / bc;
  }
  // tiles whose chain has at least n blocks
  DASH_ORDER_HD int tiles_from(int n) const {
    if (n <= 0) return tiles();
    if (blocks() < n) return 0;
    if (!causal) return tiles();
    // first_block(j) <= blocks - n, and the tile is seen at all (n >= 1)
    const long end = 64L * (blocks() - n + 1) < nq ? 64L * (blocks() - n + 1) : nq;  // rows below end
    const long key = end - 1 + off();  // the last key that one of them sees
    if (key < 0) return 0;
    const int t = (int)(key / bc) + 1;
    return t < tiles() ? t : tiles();
  }
  // block steps of the sequence's chains per query head, about: visible pairs over a
  // step's, and half a step more for every block and tile that the border cuts
  DASH_ORDER_HD long steps() const {
    const long m = nq, n = nk;
    if (m == 0 || n == 0) return 0;
    if (!causal) return (long)blocks() * tiles();
    const long pairs = n >= m ? m * (n - m) + m * (m + 1) / 2 : n * (n + 1) / 2;
    return pairs / (64L * bc) + (blocks() + tiles()) / 2;
  }
};

// Where a group has several query heads, a long tile's chain is split into one chain
// per query head, whose dK and dV partials a further kernel adds in order of the head:
// a chain of all heads of a long tile would outlast the rest of the call.  A tile is
// long where its chain has more than split_above blocks, i.e. more than a
// kSplitShare-th of a worker's share of all steps.  The constants do not ask the device,
// so that the sums' order depends on the lengths alone.  Long tiles times K/V heads are
// then fewer than kSplitShare kSplitWorkers (each has more than that part of the steps).
constexpr int kSplitWorkers = 256, kSplitShare = 8;
DASH_ORDER_HD long split_above(long steps_per_head, int heads_q, int group) {
  return steps_per_head * heads_q / ((long)kSplitShare * kSplitWorkers) / group;
}
// room for the partials of this many tiles
DASH_ORDER_HD int split_tiles(int slots, int heads_kv) {
  const int most = (kSplitShare * kSplitWorkers + heads_kv - 1) / heads_kv;
  return slots < most ? slots : most;
}

// Chains start in descending order of their length, equal ones by sequence: the
// part of tile (s, j)'s place that sequence `other` (number o) adds.  Within one sequence
// lengths do not rise with j, so its own part is j.
DASH_ORDER_HD int order_part(const SeqGeom& other, int o, int s, int j, int length) {
  return o == s ? j : other.tiles_from(o < s ? length : length + 1);
}

}  // namespace dash

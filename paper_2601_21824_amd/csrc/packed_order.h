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

// Where a group has several query heads, a long tile's chain can be split into chains
// of fewer heads each, whose dK and dV partials a further kernel adds in order: as
// one chain it would outlast the rest of the call.  A split is `parts` chains of up
// to ceil(group / parts) heads for every tile whose chain has more than `above` blocks.
// Which one: the least of split_cost over kSplits choices, in block steps of a worker.
// It asks the lengths and a constant number of workers (the 256 CUs), not the device, so
// that the sums' order depends on the lengths alone.
constexpr int kSplitWorkers = 256;
constexpr int kSplitLimits = 8, kSplitParts = 8, kSplits = kSplitLimits * kSplitParts;
// limit i: a tile is long whose whole chain is over 2^-i of a worker's share
DASH_ORDER_HD long split_above(long share, int group, int i) { return (share >> i) / group; }
DASH_ORDER_HD int split_heads(int group, int i) {  // heads per part, choice i: group / 2^i
  const int h = (group + (1 << i) - 1) >> i;
  return h < 1 ? 1 : h;
}
DASH_ORDER_HD int split_parts(int group, int heads) { return (group + heads - 1) / heads; }
// share: steps of all chains over the workers; longest: blocks of the longest chain;
// n_long: tiles with more than `above` blocks; heads: per part (group: none is split).
// Unsplit chains start last, so that on average half of one stands over at the end;
// writing and reading a part's partials counts as 6 steps (by 3, 12 sequences of 8192 tokens, 32
// heads over 8, took one head a part, 474 us, by 5 to 12 two, 420).
DASH_ORDER_HD long split_cost(long share, long longest, long above, long n_long, int heads, int group, int heads_kv) {
  const bool whole = heads >= group;
  const long tail = (whole || above > longest ? longest : above) * group;
  long t = share + tail / 2;
  t = t > tail ? t : tail;
  if (whole) return t;
  const long part = longest > above ? longest * heads : 0;
  t = t > part ? t : part;
  return t + 6 * n_long * heads_kv * split_parts(group, heads) / kSplitWorkers;
}
// Parts there is room for (a part is its dK and its dV); a choice that needs more is not
// taken: all chains in parts of one head where those are few, else eight for every worker.
DASH_ORDER_HD int split_room(int slots, int heads_q) {
  const long all = (long)slots * heads_q;
  return all < 8 * kSplitWorkers ? (int)all : 8 * kSplitWorkers;
}

// Chains start in descending order of their length, equal ones by sequence: the
// part of tile (s, j)'s place that sequence `other` (number o) adds.  Within one sequence
// lengths do not rise with j, so its own part is j.
DASH_ORDER_HD int order_part(const SeqGeom& other, int o, int s, int j, int length) {
  return o == s ? j : other.tiles_from(o < s ? length : length + 1);
}

}  // namespace dash

// Host check of packed_order.h against enumeration: which blocks a KV tile's chain
// visits, each block's last tile, and the order of the chains (a permutation, longest
// first, each sequence's tiles in ascending order).
#include <algorithm>
#include <cstdio>
#include <random>
#include <vector>

#include "packed_order.h"

static int bad = 0;
#define CHECK(x) \
  if (!(x)) std::printf("line %d: %s\n", __LINE__, #x), ++bad

int main() {
  using namespace dash;
  std::mt19937 rng(1);
  for (int bc : {128, 256})
    for (int causal = 0; causal < 2; ++causal)
      for (int trial = 0; trial < 400; ++trial) {
        const int batch = 1 + (int)(rng() % 6), top = 1 << (rng() % 12);
        std::vector<SeqGeom> q;
        for (int s = 0; s < batch; ++s) q.push_back(SeqGeom{(int)(rng() % top), (int)(rng() % top), causal != 0, bc});
        int total = 0;
        for (const SeqGeom& g : q) {
          total += g.tiles();
          const int T = g.tiles(), B = g.blocks();
          CHECK(T == (g.nk + bc - 1) / bc && B == (g.nq + 63) / 64);
          auto sees = [&](int pb, int j) {  // some query of the block sees some key of the tile
            const int last = std::min(pb * 64 + 63, g.nq - 1);
            return !causal || j * bc <= last + g.off();
          };
          for (int j = 0; j < T; ++j) {
            int n = 0;
            for (int pb = 0; pb < B; ++pb) {
              n += sees(pb, j);
              CHECK(sees(pb, j) == (pb >= g.first_block(j)));
            }
            CHECK(n == g.chain(j) && (j == 0 || n <= g.chain(j - 1)));
          }
          for (int pb = 0; pb < B; ++pb) {
            int last = -1;
            for (int j = 0; j < T; ++j)
              if (sees(pb, j)) {
                CHECK(last == j - 1);  // the rank of tile j is j
                last = j;
              }
            CHECK(g.last_tile(pb) == last);
          }
          for (int n = 0; n <= B + 2; ++n) {
            int m = 0;
            for (int j = 0; j < T; ++j) m += g.chain(j) >= n;
            CHECK(g.tiles_from(n) == m);
          }
        }
        // a chain is split only where few of all tiles can be
        for (int hkv : {1, 3, 8})
          for (int group : {2, 4, 32}) {
            long steps = 0;
            for (const SeqGeom& g : q) {
              steps += g.steps();
              long exact = 0;
              for (int j = 0; j < g.tiles(); ++j) exact += g.chain(j);
              CHECK(g.steps() <= exact + g.blocks() + g.tiles() && exact <= g.steps() + g.blocks() + g.tiles());
            }
            // every choice of a split covers the group's heads once
            for (int i = 0; i < kSplitParts; ++i) {
              const int heads = split_heads(group, i), parts = split_parts(group, heads);
              CHECK(heads >= 1 && heads <= group && (parts - 1) * heads < group && parts * heads >= group);
              CHECK(i > 0 || heads == group);
            }
            const long share = steps * hkv * group / kSplitWorkers;
            for (int i = 0; i < kSplitLimits; ++i) {
              const long above = split_above(share, group, i);
              CHECK(above >= 0 && (i == 0 || above <= split_above(share, group, i - 1)));
              int n_long = 0;
              for (const SeqGeom& g : q) n_long += g.tiles_from((int)above + 1);
              CHECK(n_long <= total);
            }
          }
        std::vector<int> seen(total, 0), length(total, -1), seq(total, -1), tile(total, -1);
        for (int s = 0; s < batch; ++s)
          for (int j = 0; j < q[s].tiles(); ++j) {
            int place = 0;
            for (int o = 0; o < batch; ++o) place += order_part(q[o], o, s, j, q[s].chain(j));
            CHECK(place >= 0 && place < total);
            if (place < 0 || place >= total) continue;
            ++seen[place];
            length[place] = q[s].chain(j), seq[place] = s, tile[place] = j;
          }
        std::vector<int> next(batch, 0);
        for (int i = 0; i < total; ++i) {
          CHECK(seen[i] == 1);
          CHECK(i == 0 || length[i] <= length[i - 1]);
          if (seq[i] >= 0) CHECK(tile[i] == next[seq[i]]++);
        }
      }
  std::printf("%s\n", bad ? "FAILED" : "ok");
  return bad != 0;
}

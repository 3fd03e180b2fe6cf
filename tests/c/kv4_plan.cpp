// Plans of the attention over 4-bit pools, printed for tests/test_kv4_plans.py.
//   DT CAUSAL N_KV GROUP HEAD_DIM CUS B, then T L P PBASE BASE for each sequence
//     ->  for each set: query nodes, L, P, rows of a block, row blocks, tiles per chunk, chunks, tiles of the
//         last row block, slab, parts, shared, part0, items; then blocks, parts
#include <cstdio>
#include <iostream>

#include "internal.h"

using namespace specmemo;

int main() {
  int dt, causal, n_kv, g, d, cus, B, row = 0;
  std::cin >> dt >> causal >> n_kv >> g >> d >> cus >> B;
  std::vector<WalkSeq> seqs;
  for (int b = 0; b < B; ++b) {
    WalkSeq s{};
    std::cin >> s.T >> s.L >> s.P >> s.pbase >> s.base;
    s.row0 = row;
    row += s.T;
    if (s.P == 0) s.pbase = 0;
    if (s.T > 0) seqs.push_back(s);
  }
  WalkPlan p;
  plan_walk(dt, causal != 0, seqs, n_kv, g, d, cus, &p, true);
  for (const WalkSetPacked &q : p.sets) {
    const WalkSet s = walk_expand(q, g);
    std::printf("%d %d %d %d %d %d %d %d %d %d %d %d %d\n", s.T, s.L, s.P, s.rb, s.nrb, s.ct, s.nch, walk_tiles(s, s.nrb - 1, g),
                s.slab, s.parts, s.shared, s.part0, s.items);
  }
  std::printf("%lld %lld\n", (long long)p.blocks, (long long)p.parts);
}

// Host plans of the serving calls, printed for tests/test_serving_plans.py.
//   rules SEG VOCAB B TOTAL MAX_NODES CUS  ->  node rows a block, grid y
//   walk DT CAUSAL N_KV GROUP HEAD_DIM CUS B, then T L P PBASE BASE for each sequence
//     ->  blocks, merge blocks, parts, table (1: in the workspace), sets; then for each set
//         T, rows of a block, row blocks, tiles per chunk, chunks, slab, parts, shared
#include <cstdio>
#include <cstring>
#include <iostream>
#include <string>

#include "internal.h"

using namespace specmemo;

int main() {
  std::string kind;
  while (std::cin >> kind) {
    if (kind == "rules") {
      int seg, vocab, B, total, max_nodes, cus;
      std::cin >> seg >> vocab >> B >> total >> max_nodes >> cus;
      const int rows = rules_rows((vocab + seg - 1) / seg, B, total, max_nodes, cus);
      std::printf("%d %lld\n", rows, (long long)B * ((max_nodes + rows - 1) / rows));
    } else {
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
      plan_walk(dt, causal != 0, seqs, n_kv, g, d, cus, &p);
      std::printf("%lld %lld %lld %d %zu\n", (long long)p.blocks, (long long)p.cblocks, (long long)p.parts,
                  (int)(p.sets.size() > (size_t)kMaxWalkSets), p.sets.size());
      for (const WalkSetPacked &q : p.sets) {
        const WalkSet s = walk_expand(q, g);
        std::printf("%d %d %d %d %d %d %d %d\n", s.T, s.rb, s.nrb, s.ct, s.nch, s.slab, s.parts, s.shared);
      }
    }
  }
}

// Launch planning of the attention over key ranges (range_attn.hip): which
// sequences' rows walk a shared prefix together, how many rows a block takes, how
// the keys are split over blocks, and where every part goes.
#include <algorithm>
#include <numeric>

#include "internal.h"

namespace specmemo {

namespace {

constexpr int kMaxCausalChunks = 64;   // one a lane (decode_walk)

// Rules of the split, in us of a block's time (two blocks share a compute unit): a
// 64-key tile takes a block of 64 rows kTileSmall and one of 128 rows kTileLarge.
// kTileF32, for each 32 columns of an fp32 head, is no such time (32 rows against a tile
// of 128 columns take 7.4 us with two blocks a unit: 4 x 1024 rows x 16 heads, 253 us, the
// same with any weight tried) but the weight that cuts and packs best on the whole.
// 0.9 cuts more: 2 x 500 rows x 8 heads of 64 columns 25.8 us, 17.2 with 0.45; 1024 x 4 of
// 128 39.1, 28.2; 8 trees of 16 nodes over a prefix of 512, 4 KV heads of 128 19.8, 25.0;
// 2 KV heads of 64 17.6, 20.9.  0.22 cuts less: 8 tokens over 2048 keys, 4 KV heads of 64
// 29.4, 23.7, of 128 38.0, 43.2; 8 x 1 to 8 tokens over 512 to 2048, 2 of 96 29.6, 21.2.
constexpr double kTileSmall = 1.05, kTileLarge = 2.0, kTileF32 = 0.45;
// A chunk's start and its share of the merge.  Below about this much work a chunk
// is mostly that: 8 sequences of 1 to 8 tokens over 500 to 4000 keys, 64 query heads,
// 19.1 us in chunks of 8 tiles, 26 in chunks of 3, 42 unsplit.
constexpr double kChunkStart = 5.0;
// Chunks may exceed a block slot's average share by this much where their row blocks
// are full: every part of full row blocks is written and read again (16 KB for 32
// rows).  10 sequences of 512 rows over 2.1k to 3k keys: unsplit (48 tiles) 74.8 us,
// chunks of 19 tiles 76.8, of 12 81.1; 24 sequences of 16 rows over a prefix of 4096
// keys (384 packed rows): 22 tiles 51.6 us, 16 tiles 54.4, unsplit 91.
constexpr double kFullSlack = 0.6;

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// (row block, chunk) pairs of a KV head
int count_items(const WalkSet &s, int g) {
  if (!s.causal || s.nrb == 1) return s.nrb * s.nch;
  int n = 0;
  for (int c = 0; c < s.nch; ++c) n += s.nrb - walk_first_rb(s, c, g);
  return n;
}

// Tiles of all row blocks of a KV head.
int64_t count_tiles(const WalkSet &s, int g) {
  if (!s.causal) return (int64_t)s.nrb * walk_tiles(s, 0, g);
  int64_t n = 0;
  for (int rb = 0; rb < s.nrb; ++rb) n += walk_tiles(s, rb, g);
  return n;
}

}  // namespace

void plan_walk(int dt, bool causal, const std::vector<WalkSeq> &seqs, int n_kv, int g, int head_dim, int cus, WalkPlan *p, bool four) {
  const bool f32 = dt == 0;
  const int nseq = (int)seqs.size();
  auto rows_of = [&](int i) { return (int64_t)seqs[i].T * g; };
  // rows that a block's tile costs are paid for: 128 cost about twice 64
  auto paid = [&](int64_t rows) { return f32 ? ceil_div(rows, 32) * 32 : rows <= 64 ? 64 : ceil_div(rows, 128) * 128; };

  auto tile_of = [&](int rb) { return f32 ? kTileF32 * ceil_div(head_dim, 32) : rb > 64 ? kTileLarge : kTileSmall; };

  // Runs of neighbours over one prefix: their rows are packed for its keys where
  // that pays for at most three quarters of the rows and saves more than the merge of
  // the parts costs, of a block slot's work or of the longest block's chain (2 x 16
  // fp32 rows over 100 keys: no faster packed).
  struct Run {
    int first, last;
  };
  std::vector<Run> runs;
  std::vector<int> run_of(nseq, -1);
  for (int i = 0; i < nseq;) {
    int j = i + 1;
    int64_t rows = rows_of(i), apart = paid(rows);
    while (j < nseq && seqs[j].P == seqs[i].P && seqs[j].pbase == seqs[i].pbase && rows + rows_of(j) <= INT32_MAX / 2) {
      rows += rows_of(j);
      apart += paid(rows_of(j));
      ++j;
    }
    bool pack = seqs[i].P > 0 && j - i > 1 && 4 * (int64_t)paid(rows) <= 3 * apart;
    if (pack) {
      const int np = ceil_div(seqs[i].P, kAttnKeyTile);
      int own = 0;
      for (int k = i; k < j; ++k) own = std::max(own, ceil_div(seqs[k].L + seqs[k].T, kAttnKeyTile));
      const double t = tile_of(64), saved = (double)(apart - paid(rows)) / (f32 ? 32 : 64) * np * t * n_kv / (2.0 * cus);
      pack = std::max(saved, std::min(np, own) * t) > kChunkStart;
    }
    if (pack) {
      for (int k = i; k < j; ++k) run_of[k] = (int)runs.size();
      runs.push_back(Run{i, j});
    }
    i = j;
  }

  std::vector<WalkSet> sets;
  for (const Run &r : runs) {
    WalkSet s{};
    s.pbase = seqs[r.first].pbase;
    s.P = seqs[r.first].P;
    s.row0 = seqs[r.first].row0;
    for (int k = r.first; k < r.last; ++k) s.T += seqs[k].T;
    s.shared = -1;
    s.parts = 1;
    sets.push_back(s);
  }
  for (int i = 0; i < nseq; ++i) {
    const WalkSeq &q = seqs[i];
    WalkSet s{};
    s.base = q.base;
    s.L = q.L;
    s.T = q.T;
    s.row0 = q.row0;
    s.shared = run_of[i];
    s.parts = s.shared >= 0;
    if (s.shared < 0) {
      s.pbase = q.pbase;
      s.P = q.P;
    }
    s.causal = causal;
    s.slab = 1;
    sets.push_back(s);
  }

  // Row blocks of 128 rows, or of 64 with the keys of a tile split over two wave
  // groups (half the chain per tile, but every tile is loaded for half the rows, and
  // a block starts twice as often): where nobody has more rows, where 128-row blocks
  // would not give every compute unit one, and for causal blocks, whose lengths
  // differ, also up to two a unit if the longest takes eight times its start.
  // Causal, 32 heads x 1024 rows (256 blocks of 128): 22.0 us in 64, 25.2 in 128; x
  // 2048 (512, up to 32 tiles) 54.6, 67.3; 8 heads x 8192 rows (512, up to 16 tiles)
  // 35.8, 32.7; 8 heads x 4 x 2048 rows (512, up to 4) 22.3, 17.6.  Trees, 8 heads x
  // 5120 rows (320 blocks of 48 tiles): 81.5, 74.8.
  int64_t large_blocks = 0;
  int longest = 0;
  for (const WalkSet &s : sets) {
    large_blocks += (int64_t)ceil_div((int64_t)s.T * g, 128) * n_kv;
    longest = std::max(longest, ceil_div(s.P, kAttnKeyTile) + (s.slab ? ceil_div(s.L + s.T, kAttnKeyTile) : 0));
  }
  const bool small = large_blocks <= cus || (causal && large_blocks <= 2 * cus && longest * kTileLarge >= 8 * kChunkStart);
  auto tile_us = [&](const WalkSet &s) { return tile_of(s.rb); };
  double work = 0;
  for (WalkSet &s : sets) {
    const int64_t rows = (int64_t)s.T * g;
    s.rb = f32 || (four && rows <= 16) ? 32 : rows <= 64 || small ? 64 : 128;
    s.nrb = ceil_div(rows, s.rb);
    work += (double)count_tiles(s, g) * tile_us(s) * n_kv;
  }
  const double share = work / (2.0 * cus);
  const size_t n = sets.size();
  std::vector<double> size(n);             // the longest item of each set
  for (size_t i = 0; i < n; ++i) {
    WalkSet &s = sets[i];
    const int nt = walk_tiles(s, s.nrb - 1, g);
    const double full = std::min(1.0, (double)s.T * g / s.rb);
    const double limit = share * (1 + kFullSlack * full) + kChunkStart;
    int nch = ceil_div(nt, std::max(1, (int)std::min<double>(nt, limit / tile_us(s))));
    if (s.causal && s.nrb > 1) nch = std::min(nch, kMaxCausalChunks);
    s.ct = ceil_div(nt, nch);              // equal chunks; the count may drop by rounding
    s.nch = ceil_div(nt, s.ct);
    s.items = count_items(s, g);
    size[i] = s.ct * tile_us(s);
  }

  // longest items first
  std::vector<int> order(n), place(n);
  std::iota(order.begin(), order.end(), 0);
  std::stable_sort(order.begin(), order.end(), [&](int x, int y) { return size[x] > size[y]; });
  for (size_t i = 0; i < n; ++i) place[order[i]] = (int)i;
  int64_t block = 0, cblock = 0, part = 0;
  for (int i : order) {
    WalkSet s = sets[i];
    if (s.shared >= 0) s.shared = place[s.shared];
    s.cum = (int)block;
    block += (int64_t)s.items * n_kv;
    s.part0 = -1;
    if (s.nch > 1 || s.parts) {
      s.part0 = (int)part;
      part += (int64_t)s.items * n_kv * (s.rb / 32);
    }
    s.ccum = (int)cblock;
    WalkSetPacked q{};
    q.base_lo = (uint32_t)s.base;
    q.base_hi = (uint8_t)(s.base >> 32);
    q.pbase_lo = (uint32_t)s.pbase;
    q.pbase_hi = (uint8_t)(s.pbase >> 32);
    q.rb32 = (uint8_t)(s.rb / 32);
    q.flags = (uint8_t)(s.causal | s.slab << 1 | s.parts << 2);
    q.L = s.L;
    q.T = s.T;
    q.P = s.P;
    q.row0 = s.row0;
    q.ct = s.ct;
    q.items = s.items;
    q.cum = s.cum;
    q.part0 = s.part0;
    q.ccum = s.ccum;
    q.shared = s.shared;
    p->sets.push_back(q);
    cblock += (int64_t)walk_expand(q, g).citems * n_kv;
  }
  p->blocks = block;
  p->cblocks = cblock;
  p->parts = part;
}

}  // namespace specmemo

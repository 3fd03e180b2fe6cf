// Launch planning of the attention over key ranges (range_attn.hip): which
// sequences' rows walk a shared prefix together, how the keys are split over
// blocks, and where every part goes.
#include <algorithm>
#include <numeric>

#include "internal.h"

namespace specmemo {

namespace {

// Fewest tiles of a chunk.  A chunk costs a start-up of about two tiles' time
// and its share of the merge.
constexpr int kMinTilesBf16 = 3, kMinTilesF32 = 2;
constexpr int kMaxCausalChunks = 64;   // one a lane (decode_walk)

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

int64_t chunk_items(const WalkSet &s, int ct, int RB, int g) {
  if (!s.causal || s.nrb == 1) return (int64_t)s.nrb * ceil_div(walk_tiles(s, 0, RB, g), ct);
  int64_t n = 0;
  WalkSet t = s;
  t.ct = ct;
  for (int c = 0, nch = ceil_div(walk_tiles(s, s.nrb - 1, RB, g), ct); c < nch; ++c) n += s.nrb - walk_first_rb(t, c, RB, g);
  return n;
}

}  // namespace

void plan_walk(int dt, bool causal, const std::vector<WalkSeq> &seqs, int n_kv, int g, int cus, WalkPlan *p) {
  const bool f32 = dt == 0;
  const int nseq = (int)seqs.size();
  auto rows_of = [&](int i) { return (int64_t)seqs[i].T * g; };

  // Row blocks: 128 rows, or 64 rows with the keys of a tile split over two wave
  // groups where nobody has more (fp32: 32 rows).
  int64_t most = 0;
  for (int i = 0; i < nseq; ++i) most = std::max(most, rows_of(i));
  int RB = f32 ? 32 : most <= 64 ? 64 : 128;

  // Runs of neighbours over one prefix: their rows are packed for its keys where
  // that walks them with at most three quarters of the row blocks (the parts of
  // both sides are then written and merged).
  struct Run {
    int first, last;
  };
  std::vector<Run> runs;
  std::vector<int> run_of(nseq, -1);
  int RBp = RB;
  for (int i = 0; i < nseq;) {
    int j = i + 1;
    int64_t rows = rows_of(i), apart = ceil_div(rows_of(i), RB) * (int64_t)RB;
    while (j < nseq && seqs[j].P == seqs[i].P && seqs[j].pbase == seqs[i].pbase && rows + rows_of(j) <= INT32_MAX / 2) {
      rows += rows_of(j);
      apart += ceil_div(rows_of(j), RB) * (int64_t)RB;
      ++j;
    }
    const int rbp = f32 ? 32 : rows <= 64 ? 64 : 128;
    if (seqs[i].P > 0 && j - i > 1 && 4 * ceil_div(rows, rbp) * (int64_t)rbp <= 3 * apart) {
      for (int k = i; k < j; ++k) run_of[k] = (int)runs.size();
      runs.push_back(Run{i, j});
      RBp = std::max(RBp, rbp);
    }
    i = j;
  }
  RB = RBp;
  p->rb = RB;

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

  // The split: where the unsplit items fit one round of resident blocks, the
  // shortest chunk that still does; otherwise no item is longer than a block's
  // average share.
  const int64_t slots = 2 * (int64_t)cus;
  const int min_tiles = f32 ? kMinTilesF32 : kMinTilesBf16;
  int64_t items = 0, work = 0;
  int longest = 1;
  for (WalkSet &s : sets) {
    s.nrb = ceil_div((int64_t)s.T * g, RB);
    items += (int64_t)s.nrb * n_kv;
    const int nt = walk_tiles(s, s.nrb - 1, RB, g);
    longest = std::max(longest, nt);
    if (!s.causal) {
      work += (int64_t)nt * s.nrb * n_kv;
    } else {
      for (int rb = 0; rb < s.nrb; ++rb) work += (int64_t)walk_tiles(s, rb, RB, g) * n_kv;
    }
  }
  int ct = longest;
  if (items < slots) {
    int lo = std::min(std::max(min_tiles, ceil_div(longest, slots)), longest), hi = longest;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      int64_t n = 0;
      for (const WalkSet &s : sets) n += chunk_items(s, mid, RB, g) * n_kv;
      if (n <= slots) hi = mid;
      else lo = mid + 1;
    }
    ct = lo;
  } else {
    ct = std::max<int64_t>(min_tiles, (work + slots - 1) / slots);
  }

  std::vector<int> size(sets.size());
  for (size_t i = 0; i < sets.size(); ++i) {
    WalkSet &s = sets[i];
    const int nt = walk_tiles(s, s.nrb - 1, RB, g);
    int nch = std::max(1, ceil_div(nt, ct));
    if (s.causal && s.nrb > 1) nch = std::min(nch, kMaxCausalChunks);
    s.ct = ceil_div(nt, nch);            // equal chunks; the count may drop by rounding
    s.nch = ceil_div(nt, s.ct);
    s.items = (int)chunk_items(s, s.ct, RB, g);
    size[i] = s.nch == 1 ? nt : s.ct;
  }
  // longest items first
  std::vector<int> order(sets.size()), place(sets.size());
  std::iota(order.begin(), order.end(), 0);
  std::stable_sort(order.begin(), order.end(), [&](int x, int y) { return size[x] > size[y]; });
  for (size_t i = 0; i < order.size(); ++i) place[order[i]] = (int)i;
  const int fan = 8 / std::gcd(n_kv, 8), units = n_kv * fan / 8;
  p->fan = fan;
  p->units = units;
  int64_t slot = 0, cslot = 0, part = 0;
  for (int i : order) {
    WalkSet s = sets[i];
    if (s.shared >= 0) s.shared = place[s.shared];
    s.cum = (int)slot;
    slot += (int64_t)ceil_div(s.items, fan) * units;
    s.part0 = -1;
    if (s.nch > 1 || s.parts) {
      s.part0 = (int)part;
      part += (int64_t)s.items * n_kv;
    }
    s.ccum = (int)cslot;
    if (s.slab && s.part0 >= 0) {
      if (!s.parts && s.causal) s.cunit0 = walk_first_rb(s, 1, RB, g) * (RB / 32);
      s.citems = ceil_div((int64_t)s.T * g, 32) - s.cunit0;
      cslot += (int64_t)ceil_div(s.citems, fan) * units;
    }
    p->sets.push_back(s);
  }
  p->slots = slot;
  p->cslots = cslot;
  p->parts = part;
}

}  // namespace specmemo

// Attention of packed query rows over the KV pool: prompt tokens (causal), and
// candidate trees whose sequences share a prefix.
//
// SpecMemo Sec. 3.1: the preallocated cache holds the prompt's K/V before any
// tree is verified, and is sized to a budget; a prefix that several sequences
// share is kept once.  A set is a range of query nodes (prompt tokens, or tree
// nodes) and the keys that its blocks walk: the prefix's rows, which every node
// sees, then the rows of the sequence's slab, under the causal or the tree mask.
// Its query rows are nodes x the GQA group's query heads (node-major), RB to a
// row block; a work item is (set, KV head, row block, chunk of 64-key tiles).
//
//   out = sum_j 2^(s_j - m) v_j / sum_j 2^(s_j - m),  s = q . k scale log2(e)
//
// with the running maximum m and both sums kept in fp32 over one pass of the
// keys.  Parts of a row's keys walked by several blocks (chunks; a prefix walked
// once for the packed rows of all its sequences) are left in the workspace as
// (m, l, O) in fp32 and merged in a fixed order by walk_combine: no atomics.
//
// bf16: the tile loop of tree_attn_bf16 (K and V tiles in LDS rings filled by
// direct loads, S^T = K Q^T and O^T = V^T P^T on the 32x32x16 matrix product,
// 32 query rows a wave, P never leaves its lane).
// fp32: 32 query rows a block on the 32x32x2 fp32 product, the block's waves
// taking 32-key tiles in turn straight from memory, merged through LDS.
#include <type_traits>

#include "attn_tile.h"
#include "device.h"
#include "internal.h"

namespace specmemo {

namespace {

constexpr int D = kAttnHeadDim;
constexpr int TK = kAttnKeyTile;
constexpr float kRescaleSlack = 8.f;   // log2 units: softmax weights stay <= 256 between rescales

struct WalkItem {
  WalkSet S;
  int kvh, rb, ch;
};

// The kernel arguments where they lie, read by scalar loads (an array of the
// arguments indexed through a pointer that may also point elsewhere would be copied
// to scratch memory as a whole).
typedef __attribute__((address_space(4))) const WalkArgs KernArgs;
__device__ __forceinline__ KernArgs *kern_args() { return (KernArgs *)__builtin_amdgcn_kernarg_segment_ptr(); }

// The set that block k belongs to: the last one with first block <= k.
template <bool COMBINE>
__device__ __forceinline__ int find_set(const WalkArgs &a, int k) {
  const int lane = threadIdx.x & 63;
  int lo = 0, cnt = a.nset;
  while (cnt > 1) {   // 64 ways a round: two rounds for up to 4096 sets
    const int st = (cnt + 63) >> 6, at = lane * st;
    int first = 0;
    if (at < cnt) {
      if (a.tab) first = COMBINE ? a.tab[lo + at].ccum : a.tab[lo + at].cum;
      else first = COMBINE ? a.set[lo + at].ccum : a.set[lo + at].cum;
    }
    const int p = __builtin_popcountll(__builtin_amdgcn_ballot_w64(at < cnt && first <= k)) - 1;
    lo += p * st;
    cnt = min(st, cnt - p * st);
  }
  return lo;
}

// Set s, in SGPRs (the direct loads need their base there): from the arguments by
// scalar loads, from the workspace table one word a lane.
__device__ __forceinline__ WalkSet get_set(const WalkArgs &a, int s) {
  constexpr int N = sizeof(WalkSetPacked) / 4;
  static_assert(sizeof(WalkSetPacked) % 4 == 0 && N <= 64, "copied by words");
  s = __builtin_amdgcn_readfirstlane(s);
  int w[N];
  if (a.tab) {
    const int v = reinterpret_cast<const int *>(a.tab + s)[min((int)(threadIdx.x & 63), N - 1)];
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = __builtin_amdgcn_readlane(v, i);
  } else {
    const auto *p = (__attribute__((address_space(4))) const int *)&kern_args()->set[s];
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = p[i];
  }
  WalkSetPacked P;
  __builtin_memcpy(&P, w, sizeof(P));
  return walk_expand(P, a.group);
}

// A set's blocks are its items times the KV heads, KV head fastest, without gaps.
// Blocks reach the eight XCDs round-robin and every set begins at a multiple of
// n_kv, so a KV head's items run on the XCDs that equal it modulo gcd(n_kv, 8), on
// one where n_kv is a multiple of eight, and read its K/V through those L2s.
// (Empty blocks that even out the XCDs' counts set by set push two of the others to
// one compute unit: one KV head, 40 trees of 64 nodes x 4 heads over a prefix of 4096
// keys 79.4 us, 68.9 without; 256 single tokens over 200 to 1000 keys 42.7, 29.6.)
template <bool COMBINE>
__device__ __forceinline__ void decode_unit(const WalkArgs &a, int bid, WalkSet &S, int &kvh, int &i) {
  S = get_set(a, find_set<COMBINE>(a, bid));
  const int n = bid - (COMBINE ? S.ccum : S.cum);
  kvh = n % a.n_kv;
  i = n / a.n_kv;
}

__device__ __forceinline__ void decode_walk(const WalkArgs &a, int bid, WalkItem &it) {
  int i;
  decode_unit<false>(a, bid, it.S, it.kvh, i);
  const WalkSet &S = it.S;
  if (S.nch == 1) {              // longest row blocks first
    it.ch = 0;
    it.rb = S.nrb - 1 - i;
  } else if (!S.causal || S.nrb == 1) {
    it.ch = i / S.nrb;
    it.rb = i % S.nrb;
  } else {                       // chunk by chunk, the row blocks that reach it: at most 64 chunks, one a lane
    const int lane = threadIdx.x & 63;
    const int r0 = lane < S.nch ? walk_first_rb(S, lane, a.group) : S.nrb;
    int before = S.nrb - r0;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int o = __shfl_up(before, off);
      before += lane >= off ? o : 0;
    }
    const int c = __builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < S.nch && before <= i));
    it.ch = c;
    it.rb = i - (__shfl(before, c) - (S.nrb - __shfl(r0, c))) + __shfl(r0, c);
  }
  it.rb = __builtin_amdgcn_readfirstlane(it.rb);
  it.ch = __builtin_amdgcn_readfirstlane(it.ch);
}

// First 32-row unit of the parts of (row block, chunk).
__device__ __forceinline__ int walk_part(const WalkArgs &a, const WalkSet &S, int kvh, int rb, int ch) {
  int i;   // index among the set's items
  if (S.nch == 1) i = S.nrb - 1 - rb;
  else if (!S.causal || S.nrb == 1) i = ch * S.nrb + rb;
  else {
    i = rb - walk_first_rb(S, ch, a.group);
    for (int c = 0; c < ch; ++c) i += S.nrb - walk_first_rb(S, c, a.group);
  }
  return S.part0 + (kvh * S.items + i) * (S.rb >> 5);
}

// A wave's 32 rows of unnormalised O^T (accumulator order, so that a store of whole
// rows is 1 KB in one piece), m and l; rows that do not exist are left out (64
// sequences of 8 rows: a quarter of the traffic).
template <int DB>
__device__ __forceinline__ void write_part(float *u, const f32x16 (&O)[DB], float m, float l, bool row_ok) {
  const int lane = threadIdx.x & 63;
  if (!row_ok) return;
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<f32x4 *>(u + ((4 * i + q) * 64 + lane) * 4) = f32x4{O[i][4 * q], O[i][4 * q + 1], O[i][4 * q + 2], O[i][4 * q + 3]};
  if (lane < 32) {
    u[DB * 1024 + lane] = m;
    u[DB * 1024 + 32 + lane] = l;
  }
}

constexpr int kBf16Waves = 4;
constexpr int kTileBytes = TK * D * 2;        // one K or V tile (16 KB)

// Four waves per block; K and V each have a two-slot ring of 64-key tiles.
// KSPLIT = 1: 32 rows a wave, every wave takes whole tiles.  KSPLIT = 2: two
// groups of waves over the same rows, one for keys 0-31 of every tile and one
// for keys 32-63, merged through LDS at the end (items of few rows: half the
// chain per tile, two waves on every SIMD).
template <int KSPLIT, bool TREE>
__device__ __forceinline__ void walk_bf16(const WalkArgs &a, const WalkItem &it, uint8_t (*kring)[kTileBytes], uint8_t (*vring)[kTileBytes]) {
  constexpr int WAVES = kBf16Waves, RW = WAVES / KSPLIT, RB = 32 * RW, NSB = 2 / KSPLIT;
  constexpr int TILE = kTileBytes;
  constexpr int IPW = TILE / 1024 / WAVES;    // 1 KB direct loads per wave per tile and operand
  int *const par = reinterpret_cast<int *>(vring[1]);   // filled after the first loop barrier
  static_assert(WAVES * 64 >= kMaxNodes && kMaxNodes * 4 <= TILE, "one thread per tree node");
  static_assert(KSPLIT == 1 || RW * 64 * 64 * 4 <= 2 * TILE, "merge buffer fits the K ring");

  const WalkSet &S = it.S;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int rwave = __builtin_amdgcn_readfirstlane(wave % RW), ksb = __builtin_amdgcn_readfirstlane(wave / RW);
  const int h = lane >> 5, g = a.group, L = S.L, P = S.P;
  const int rows = S.T * g;
  const int np = (P + TK - 1) / TK;                               // prefix tiles
  const int kend = walk_keys(S, it.rb, g);                    // slab keys of this row block
  const int j0 = it.ch * S.ct, j1 = min(np + (kend + TK - 1) / TK, j0 + S.ct);

  const uint8_t *const K0 = static_cast<const uint8_t *>(a.k), *const V0 = static_cast<const uint8_t *>(a.v);
  const int64_t head = (int64_t)it.kvh * a.cap_total;
  const int64_t po = (head + S.pbase) * (D * 2), so = (head + S.base) * (D * 2);

  // Direct loads of a tile, as in tree_attn_bf16: lane l of load i writes LDS
  // bytes [1024 i + 16 l, +16), tile row 4 i + l / 16 at physical chunk l % 16.
  const int lrow0 = 4 * wave * IPW + (lane >> 4);
  const int kx = (lane & 15) ^ (lane >> 4);
  const int voff0 = lrow0 * (D * 2) + 16 * vswz(lrow0, lane & 15);
  auto load_off = [&](bool is_k, int u) {
    const int r = lrow0 + 4 * u;
    return is_k ? r * (D * 2) + 16 * (kx ^ ((4 * (wave * IPW + u)) & 15)) : voff0 + 1024 * u;
  };
  auto issue = [&](bool is_k, uint8_t *dst, int j) __attribute__((always_inline)) {
    const bool pre = j < np;
    const int kt = (pre ? j : j - np) * TK, end = pre ? P : kend;
    const uint8_t *src = uniform_ptr((is_k ? K0 : V0) + (pre ? po : so));
    const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void_t *)(dst + 1024 * wave * IPW));
    if (kt + TK <= end) {
      const uint8_t *sb = uniform_ptr(src + (int64_t)kt * (D * 2));
#pragma unroll
      for (int u = 0; u < IPW; ++u) lds_load16(sb, (uint32_t)load_off(is_k, u), lds + 1024 * u);
    } else {                             // rows past the end repeat the last one (finite values, masked out)
#pragma unroll
      for (int u = 0; u < IPW; ++u) {
        const int r = lrow0 + 4 * u;
        const int t = min(kt + r, end - 1);
        lds_load16(src, (uint32_t)(t * (D * 2) + (load_off(is_k, u) - r * (D * 2))), lds + 1024 * u);
      }
    }
  };

  issue(true, kring[0], j0);
  issue(false, vring[0], j0);
  const bool tree = TREE && S.slab;      // the set's slab rows end in a tree
  const int pn = tree && tid < S.T ? a.parent[S.row0 + tid] : -1;
  const int row0 = it.rb * RB + rwave * 32, my_row = row0 + (lane & 31);
  const bool row_ok = my_row < rows;
  const int node = row_ok ? my_row / g : S.T - 1;
  const int hq = it.kvh * g + (row_ok ? my_row % g : 0);
  bf16x8 qf[D / 16];
  {
    const uint16_t *qbase = static_cast<const uint16_t *>(a.q) + ((int64_t)(S.row0 + node) * a.n_q + hq) * D + 8 * h;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) qf[ks] = __builtin_bit_cast(bf16x8, ld16_or_zero(row_ok, qbase + 16 * ks));
  }
  if (tree && tid < S.T) par[tid] = pn;
  // land the Q loads here: a load pending at loop entry is waited for on every iteration
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) asm volatile("" ::"v"(qf[ks]));
  uint64_t alo = 0, ahi = 0;             // ancestor-or-self bits of this lane's node
  if (TREE) {
    ring_barrier();
    if (tree)
      for (int u = node; u >= 0; u = par[u]) {
        alo |= u < 64 ? 1ull << (u & 63) : 0ull;
        ahi |= u < 64 ? 0ull : 1ull << (u & 63);
      }
  }
  // causal: the last slab key of this lane's row, and of the wave's first and last row
  const int lim = L + node;
  const int lim_lo = L + __builtin_amdgcn_readfirstlane(node);
  const int lim_hi = L + min(rows - 1, row0 + 31) / g;
  const bool wave_rows = row0 < rows;    // a wave without rows only loads and waits

  int kro[D / 16];
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) kro[ks] = (lane & 31) * (D * 2) + 16 * ((2 * ks + h) ^ (lane & 15));
  const int tj = (lane & 15) >> 2, tq = lane & 3;
  const int te = 2 * ((lane >> 4) & 1) + (tq >> 1);
  int vro[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) vro[i] = (4 * h + tj) * (D * 2) + 64 * (i ^ tj) + 16 * te + 8 * (tq & 1);
  const int sb0 = ksb * NSB;

  float m = -INFINITY, lsum = 0.f;
  f32x16 O[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) O[i][r] = 0.f;
  const bf16x2_t ones = __builtin_bit_cast(bf16x2_t, 0x3F803F80u);

  auto work = [&](const uint8_t *ks, const uint8_t *vs, int j) __attribute__((always_inline)) {
    const bool pre = j < np;
    const int kt = (pre ? j : j - np) * TK;
    if (!pre && !TREE && kt + 32 * sb0 > lim_hi) return;   // past every row of the wave
    f32x16 Sc[NSB];
#pragma unroll
    for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
      for (int r2 = 0; r2 < 16; ++r2) Sc[sb][r2] = 0.f;
    const uint8_t *kw = ks + sb0 * 32 * (D * 2);
#pragma unroll
    for (int k8 = 0; k8 < D / 16; ++k8)
#pragma unroll
      for (int sb = 0; sb < NSB; ++sb) {
        const bf16x8 kf = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(kw + sb * 32 * (D * 2) + kro[k8]));
        Sc[sb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[k8], Sc[sb], 0, 0, 0);
      }
    // keep the K fragment reads just ahead of their products
#pragma unroll
    for (int k8 = 0; k8 < D / 16; ++k8) {
      __builtin_amdgcn_sched_group_barrier(0x100, NSB, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, NSB, 0);
    }
    // Accumulator entry r of sub-block sb is key kt + 32 (sb0 + sb) + 8 (r / 4) + 4 h + r % 4.
    if (TREE && !pre) {
      if (kt + TK > L) {
#pragma unroll
        for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
          for (int r2 = 0; r2 < 16; ++r2) {
            const int t = kt + 32 * (sb0 + sb) + 8 * (r2 >> 2) + 4 * h + (r2 & 3);
            const uint32_t rel = (uint32_t)(t - L) & 127u;
            const bool anc = ((rel < 64 ? alo : ahi) >> (rel & 63)) & 1u;
            Sc[sb][r2] = (t < kend) & ((t < L) | anc) ? Sc[sb][r2] : -INFINITY;
          }
      }
    } else if (kt + TK - 1 > (pre ? P - 1 : lim_lo)) {
      const int vis = (pre ? P - 1 : lim) - kt - 32 * sb0 - 4 * h;
#pragma unroll
      for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
        for (int r2 = 0; r2 < 16; ++r2)
          Sc[sb][r2] = 32 * sb + 8 * (r2 >> 2) + (r2 & 3) <= vis ? Sc[sb][r2] : -INFINITY;
    }
    float tm;
    if constexpr (NSB == 2) {
      tm = tile_max32(Sc);
    } else {
      const f32x16 &x = Sc[0];
      const float u0 = fmaxf(fmaxf(x[0], x[1]), x[2]), u1 = fmaxf(fmaxf(x[3], x[4]), x[5]);
      const float u2 = fmaxf(fmaxf(x[6], x[7]), x[8]), u3 = fmaxf(fmaxf(x[9], x[10]), x[11]);
      const float u4 = fmaxf(fmaxf(x[12], x[13]), x[14]);
      tm = fmaxf(fmaxf(fmaxf(u0, u1), fmaxf(u2, u3)), fmaxf(u4, x[15]));
    }
    const float tmax = max_with_other_half(tm) * a.scale_log2;
    // Lazy rescaling: m moves only when a score exceeds it by more than kRescaleSlack.
    const bool need = tmax > m + kRescaleSlack;
    if (__builtin_amdgcn_ballot_w64(need)) {
      const float m_new = need ? tmax : m;
      const float alpha = need ? (m == -INFINITY ? 0.f : fast_exp2(m - m_new)) : 1.f;
      m = m_new;
      lsum *= alpha;
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int r2 = 0; r2 < 16; ++r2) O[i][r2] *= alpha;
    }
    const float m_use = m == -INFINITY ? 0.f : m;
    // Weights are rounded to bf16, the matrix product's operand type (2^-8 of a
    // weight, as the inputs' own type); their sum is taken of the rounded ones.
    uint32_t pk[2 * NSB][4];
#pragma unroll
    for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float p0 = fast_exp2(fmaf(Sc[sb][8 * half + 2 * q], a.scale_log2, -m_use));
          const float p1 = fast_exp2(fmaf(Sc[sb][8 * half + 2 * q + 1], a.scale_log2, -m_use));
          pk[2 * sb + half][q] = pack_bf16x2(p0, p1);
        }
#pragma unroll
    for (int mh = 0; mh < 2 * NSB; ++mh)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        lsum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pk[mh][q]), ones, lsum, false);
#pragma unroll
    for (int mh = 0; mh < 2 * NSB; ++mh) {
      const bf16x8 pf = __builtin_bit_cast(bf16x8, uint4{pk[mh][0], pk[mh][1], pk[mh][2], pk[mh][3]});
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        const uint8_t *p = vs + 16 * (2 * sb0 + mh) * (D * 2) + vro[i];
        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)p);
        const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(p + 8 * (D * 2)));
        const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        O[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf, O[i], 0, 0, 0);
      }
    }
  };

  // Iteration j waits for tile j's loads; after its barrier every wave is done
  // with tile j - 1, whose slots take tile j + 1.
  auto tile = [&](int j, auto slot_c) __attribute__((always_inline)) {
    constexpr int slot = decltype(slot_c)::value;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    ring_barrier();
    if (j + 1 < j1) {
      issue(true, kring[slot ^ 1], j + 1);
      issue(false, vring[slot ^ 1], j + 1);
    }
    if (wave_rows) work(kring[slot], vring[slot], j);
  };
  for (int j = j0; j < j1; j += 2) {
    tile(j, std::integral_constant<int, 0>{});
    if (j + 1 < j1) tile(j + 1, std::integral_constant<int, 1>{});
  }

  float ltot = sum_with_other_half(lsum);
  if constexpr (KSPLIT == 2) {
    // Every wave is past its last read of the rings and no load is in flight:
    // the K ring takes the second group's O, the V ring its m and l.
    ring_barrier();
    float *const mo = reinterpret_cast<float *>(kring[0]);
    float *const ml = reinterpret_cast<float *>(vring[0]);
    if (ksb == 1) {
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int r2 = 0; r2 < 16; ++r2) mo[(rwave * 64 + 16 * i + r2) * 64 + lane] = O[i][r2];
      ml[(rwave * 2) * 64 + lane] = m;
      ml[(rwave * 2 + 1) * 64 + lane] = ltot;
    }
    ring_barrier();
    if (ksb == 1) return;
    const float m1 = ml[(rwave * 2) * 64 + lane], l1 = ml[(rwave * 2 + 1) * 64 + lane];
    const float mn = fmaxf(m, m1);
    const float w0 = m == -INFINITY ? 0.f : fast_exp2(m - mn);
    const float w1 = m1 == -INFINITY ? 0.f : fast_exp2(m1 - mn);
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int r2 = 0; r2 < 16; ++r2) O[i][r2] = O[i][r2] * w0 + mo[(rwave * 64 + 16 * i + r2) * 64 + lane] * w1;
    ltot = ltot * w0 + l1 * w1;
    m = mn;
  }
  if (!wave_rows) return;
  if (walk_direct(S, it.rb, g)) {
    if (!row_ok) return;
    // O^T entry r of d-block i is d = 32 i + 8 (r / 4) + 4 h + r % 4 of this lane's row.
    // The halves of a row trade four columns, so that a lane stores 16 bytes and a row
    // 32 in one piece (13B-shaped prompts of 100 to 700: 32.9 us with 8-byte stores,
    // 31.0; through LDS, for whole rows, 32.5).
    const float inv = 1.f / ltot;
    uint16_t *op = static_cast<uint16_t *>(a.out) + ((int64_t)(S.row0 + node) * a.n_q + hq) * D;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const auto &o = O[i];
        const uint32_t a0 = pack_bf16x2(o[8 * p] * inv, o[8 * p + 1] * inv), a1 = pack_bf16x2(o[8 * p + 2] * inv, o[8 * p + 3] * inv);
        const uint32_t b0 = pack_bf16x2(o[8 * p + 4] * inv, o[8 * p + 5] * inv), b1 = pack_bf16x2(o[8 * p + 6] * inv, o[8 * p + 7] * inv);
        const auto s0 = __builtin_amdgcn_permlane32_swap(a0, b0, false, false), s1 = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
        *reinterpret_cast<uint4 *>(op + 32 * i + 16 * p + 8 * h) = uint4{s0[0], s1[0], s0[1], s1[1]};
      }
  } else {
    write_part<D / 32>(a.part + (int64_t)(walk_part(a, S, it.kvh, it.rb, it.ch) + rwave) * walk_unit_floats(D / 32), O, m, ltot, row_ok);
  }
}

template <bool TREE>
__global__ __launch_bounds__(kBf16Waves * 64, 2) void walk_attn_bf16(WalkArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t kring[2][kTileBytes];
  __shared__ __attribute__((aligned(1024))) uint8_t vring[2][kTileBytes];
  WalkItem it;
  decode_walk(a, blockIdx.x, it);
  if (it.S.rb == 64) walk_bf16<2, TREE>(a, it, kring, vring);
  else walk_bf16<1, TREE>(a, it, kring, vring);
}

// fp32: DB 32-column blocks of the head; the block's 32 rows against 32-key tiles,
// wave w taking tiles w, w + W, ...  The sum over the columns may run in any order
// as long as both operands use it: lane half h holds the column quads h qh + t, so
// a lane reads 16 bytes of its key row at a time.  The weights leave the score
// accumulator as they lie (lane half h, entry r: key 8 (r / 4) + 4 h + r % 4) and
// meet V rows of the same order.
// (Eight waves a block, to take short ranges in one turn, cost more to start and
// merge than they save: 2 x 500 rows x 8 heads of 64 columns 22.4 us, 18.4 with four.)
// Up to 64 columns a tile's K and V rows are loaded as a whole, one memory latency;
// past them two waves to a SIMD hide it better than the registers that would take
// (4 x 1024 rows x 16 heads of 128 columns: 250 us, 271 as a whole).
constexpr int kF32Waves = 4;

template <int DB, bool TREE>
__global__ __launch_bounds__(64 * kF32Waves, 2) void walk_attn_f32(WalkArgs a) {
  constexpr int RB = 32, W = kF32Waves, UF = walk_unit_floats(DB);
  constexpr int KQ = DB <= 2 ? 4 * DB : 4, VR = DB <= 2 ? 16 : 4;   // column quads and key rows loaded together
  __shared__ __attribute__((aligned(16))) float merge[W][UF];
  __shared__ int par[kMaxNodes];
  WalkItem it;
  decode_walk(a, blockIdx.x, it);
  const WalkSet &S = it.S;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5, g = a.group, L = S.L, P = S.P, d = a.head_dim;
  const int rows = S.T * g;
  const int np = (P + TK - 1) / TK;
  const int kend = walk_keys(S, it.rb, g);
  const int j0 = it.ch * S.ct, j1 = min(np + (kend + TK - 1) / TK, j0 + S.ct);
  const int64_t head = (int64_t)it.kvh * a.cap_total;
  const float *const K0 = static_cast<const float *>(a.k), *const V0 = static_cast<const float *>(a.v);

  const bool tree = TREE && S.slab;
  const int my_row = it.rb * RB + (lane & 31);
  const bool row_ok = my_row < rows;
  const int node = row_ok ? my_row / g : S.T - 1;
  const int hq = it.kvh * g + (row_ok ? my_row % g : 0);
  const int quads = d >> 2, qh = (quads + 1) >> 1;
  const int myq = h ? quads - qh : qh;               // quads of this lane's half: qh or qh - 1
  f32x4 qf[4 * DB];
  {
    const float *qp = static_cast<const float *>(a.q) + ((int64_t)(S.row0 + node) * a.n_q + hq) * d + 4 * h * qh;
#pragma unroll
    for (int t = 0; t < 4 * DB; ++t) {
      qf[t] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (row_ok && t < myq) qf[t] = *reinterpret_cast<const f32x4 *>(qp + 4 * t);
    }
  }
  uint64_t alo = 0, ahi = 0;
  if (TREE) {
    if (tree && tid < S.T) par[tid] = a.parent[S.row0 + tid];
    ring_barrier();                                  // (does not wait for the queries)
    if (tree)
      for (int u = node; u >= 0; u = par[u]) {
        alo |= u < 64 ? 1ull << (u & 63) : 0ull;
        ahi |= u < 64 ? 0ull : 1ull << (u & 63);
      }
  }
  const int lim = L + node;

  float m = -INFINITY, l = 0.f;
  f32x16 O[DB];
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) O[i][r] = 0.f;
  for (int t2 = 2 * j0 + wave; t2 < 2 * j1; t2 += W) {
    const bool pre = (t2 >> 1) < np;
    const int kt = (pre ? t2 : t2 - 2 * np) * 32, end = pre ? P : kend;
    if (kt >= end) continue;
    const int64_t base = (head + (pre ? S.pbase : S.base)) * d;
    const float *kp = K0 + base + (int64_t)min(kt + (lane & 31), end - 1) * d + 4 * h * qh;
    const float *vp = V0 + base;
    f32x4 kf[KQ];
    float vf[VR][DB];
    auto load_k = [&](int t0) __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < KQ; ++t) {
        kf[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (t0 + t < myq) kf[t] = *reinterpret_cast<const f32x4 *>(kp + 4 * (t0 + t));
      }
    };
    auto load_v = [&](int r0) __attribute__((always_inline)) {
#pragma unroll
      for (int r = 0; r < VR; ++r) {
        const int t = min(kt + 8 * ((r0 + r) >> 2) + 4 * h + ((r0 + r) & 3), end - 1);
#pragma unroll
        for (int i = 0; i < DB; ++i) vf[r][i] = vp[(int64_t)t * d + min(32 * i + (lane & 31), d - 1)];   // columns past the head are not written
      }
    };
    f32x16 Sc;
#pragma unroll
    for (int r = 0; r < 16; ++r) Sc[r] = 0.f;
    load_k(0);
    if (VR == 16) load_v(0);
#pragma unroll
    for (int t0 = 0; t0 < 4 * DB; t0 += KQ) {
      if (t0 > 0) load_k(t0);
#pragma unroll
      for (int t = 0; t < KQ; ++t)
        if (t0 + t < qh) {
#pragma unroll
          for (int e = 0; e < 4; ++e) Sc = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[t][e], qf[t0 + t][e], Sc, 0, 0, 0);
        }
    }
    float tm = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int t = kt + 8 * (r >> 2) + 4 * h + (r & 3);
      bool vis;
      if (TREE && !pre) {
        const uint32_t rel = (uint32_t)(t - L) & 127u;
        vis = (t < kend) & ((t < L) | (((rel < 64 ? alo : ahi) >> (rel & 63)) & 1u));
      } else {
        vis = t <= (pre ? P - 1 : lim);
      }
      Sc[r] = vis ? Sc[r] : -INFINITY;
      tm = fmaxf(tm, Sc[r]);
    }
    const float mn = fmaxf(m, max_with_other_half(tm) * a.scale_log2);
    const float m_use = mn == -INFINITY ? 0.f : mn;
    const float alpha = m == -INFINITY ? 0.f : fast_exp2(m - m_use);
    m = mn;
    l *= alpha;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      Sc[r] = fast_exp2(fmaf(Sc[r], a.scale_log2, -m_use));
      l += Sc[r];
    }
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) O[i][r] *= alpha;
#pragma unroll
    for (int r0 = 0; r0 < 16; r0 += VR) {
      if (VR < 16) load_v(r0);
#pragma unroll
      for (int r = 0; r < VR; ++r)
#pragma unroll
        for (int i = 0; i < DB; ++i) O[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf[r][i], Sc[r0 + r], O[i], 0, 0, 0);
    }
  }
  write_part<DB>(merge[wave], O, m, sum_with_other_half(l), true);
  __syncthreads();
  // Wave w merges entries 4 DB / W w ... of all waves' parts.
  float mw[W], M = -INFINITY, lt = 0.f;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    mw[w] = merge[w][DB * 1024 + (lane & 31)];
    M = fmaxf(M, mw[w]);
  }
#pragma unroll
  for (int w = 0; w < W; ++w) {
    mw[w] = mw[w] == -INFINITY ? 0.f : fast_exp2(mw[w] - M);
    lt = fmaf(merge[w][DB * 1024 + 32 + (lane & 31)], mw[w], lt);
  }
  const bool direct = walk_direct(S, it.rb, g);
  float *const u = direct ? nullptr : a.part + (int64_t)walk_part(a, S, it.kvh, it.rb, it.ch) * UF;
  const float inv = direct ? 1.f / lt : 1.f;
  for (int iq = wave; iq < 4 * DB; iq += W) {        // d-block iq / 4, entries 4 (iq % 4) .. + 3
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const f32x4 v = *reinterpret_cast<const f32x4 *>(&merge[w][(iq * 64 + lane) * 4]);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = fmaf(v[e], mw[w], o[e]);
    }
    const int col = 32 * (iq >> 2) + 8 * (iq & 3) + 4 * h;
    if (!row_ok) continue;
    if (!direct) *reinterpret_cast<f32x4 *>(u + (iq * 64 + lane) * 4) = o;
    else if (col < d)
      *reinterpret_cast<f32x4 *>(static_cast<float *>(a.out) + ((int64_t)(S.row0 + node) * a.n_q + hq) * d + col) =
          f32x4{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
  }
  if (!direct && wave == 0 && lane < 32) {
    u[DB * 1024 + lane] = M;
    u[DB * 1024 + 32 + lane] = lt;
  }
}

// Merge the parts of 32 query rows of a set: its own chunks, then those of the
// prefix's set, where the rows lie among the packed rows of all its sequences.
// Wave w takes the column entries w DB .. + DB - 1 of the accumulator order, and the
// parts one after another, four a turn: a running maximum, the sums rescaled once a turn.
template <int DB, bool BF16>
__global__ __launch_bounds__(256) void walk_combine(WalkArgs a) {
  constexpr int UF = walk_unit_floats(DB);
  WalkSet S;
  int kvh, i;
  decode_unit<true>(a, blockIdx.x, S, kvh, i);
  i += S.cunit0;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, g = a.group;
  const int upb = S.rb >> 5, rb = __builtin_amdgcn_readfirstlane(i / upb), un = __builtin_amdgcn_readfirstlane(i % upb);
  const int row = 32 * i + (lane & 31);
  const bool row_ok = row < S.T * g;
  const int nown = walk_chunks(S, rb, g);
  WalkSet H{};
  int hr = 0, hsh = 5, parts = nown;
  if (S.shared >= 0) {
    H = get_set(a, S.shared);
    hr = (S.row0 - H.row0) * g + (row_ok ? row : 0);
    hsh = __builtin_ctz(H.rb);
    parts += H.nch;
  }
  const int hl = (hr & 31) | (lane & 32);
  // part p: its 32-row unit (own chunks by row block, the prefix's by lane) and this lane's place in it
  auto unit = [&](int p) {
    if (p < nown) return a.part + (int64_t)(walk_part(a, S, kvh, rb, p) + un) * UF;
    return a.part + (int64_t)(walk_part(a, H, kvh, hr >> hsh, p - nown) + ((hr & (H.rb - 1)) >> 5)) * UF;
  };
  if (!row_ok) return;
  // G parts are read at once, everything of them.
  constexpr int G = 4;
  float M = -INFINITY, l = 0.f;
  f32x4 o[DB];
#pragma unroll
  for (int n = 0; n < DB; ++n) o[n] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0; p0 < parts; p0 += G) {
    f32x4 v[G][DB];
    float mp[G], lp[G];
#pragma unroll
    for (int e = 0; e < G; ++e) {
      mp[e] = -INFINITY;
      lp[e] = 0.f;
#pragma unroll
      for (int n = 0; n < DB; ++n) v[e][n] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (p0 + e < parts) {
        const int p = p0 + e, ln = p < nown ? lane : hl;
        const float *u = unit(p);
        mp[e] = u[DB * 1024 + (ln & 31)];
        lp[e] = u[DB * 1024 + 32 + (ln & 31)];
#pragma unroll
        for (int n = 0; n < DB; ++n) v[e][n] = *reinterpret_cast<const f32x4 *>(u + ((wave * DB + n) * 64 + ln) * 4);
      }
    }
    const float Mn = fmaxf(fmaxf(M, fmaxf(mp[0], mp[1])), fmaxf(mp[2], mp[3]));
    // a part without a visible key of this row (m = -inf) weighs nothing
    const float w0 = M == -INFINITY ? 0.f : fast_exp2(M - Mn);
    M = Mn;
    l *= w0;
#pragma unroll
    for (int n = 0; n < DB; ++n) o[n] *= w0;
#pragma unroll
    for (int e = 0; e < G; ++e) {
      const float w = mp[e] == -INFINITY ? 0.f : fast_exp2(mp[e] - M);
      l = fmaf(lp[e], w, l);
#pragma unroll
      for (int n = 0; n < DB; ++n)
#pragma unroll
        for (int c = 0; c < 4; ++c) o[n][c] = fmaf(v[e][n][c], w, o[n][c]);
    }
  }
  const float inv = 1.f / l;
  const int node = row / g, hq = kvh * g + row % g;
  const int64_t at = ((int64_t)(S.row0 + node) * a.n_q + hq) * a.head_dim;
#pragma unroll
  for (int n = 0; n < DB; ++n) {
    const int iq = wave * DB + n, col = 32 * (iq >> 2) + 8 * (iq & 3) + 4 * h;
    if (BF16)
      *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + at + col) =
          uint2{pack_bf16x2(o[n][0] * inv, o[n][1] * inv), pack_bf16x2(o[n][2] * inv, o[n][3] * inv)};
    else if (col < a.head_dim)
      *reinterpret_cast<f32x4 *>(static_cast<float *>(a.out) + at + col) =
          f32x4{o[n][0] * inv, o[n][1] * inv, o[n][2] * inv, o[n][3] * inv};
  }
}

template <int DB, bool TREE>
void launch_f32(const WalkArgs &a, hipStream_t st) {
  hipLaunchKernelGGL((walk_attn_f32<DB, TREE>), dim3(a.blocks), dim3(64 * kF32Waves), 0, st, a);
  if (a.cblocks) hipLaunchKernelGGL((walk_combine<DB, false>), dim3(a.cblocks), dim3(256), 0, st, a);
}

template <bool TREE>
void launch_f32(const WalkArgs &a, hipStream_t st) {
  switch ((a.head_dim + 31) / 32) {
    case 1: return launch_f32<1, TREE>(a, st);
    case 2: return launch_f32<2, TREE>(a, st);
    case 3: return launch_f32<3, TREE>(a, st);
    default: return launch_f32<4, TREE>(a, st);
  }
}

template <bool TREE>
void launch_bf16(const WalkArgs &a, hipStream_t st) {
  hipLaunchKernelGGL((walk_attn_bf16<TREE>), dim3(a.blocks), dim3(64 * kBf16Waves), 0, st, a);
  if (a.cblocks) hipLaunchKernelGGL((walk_combine<D / 32, true>), dim3(a.cblocks), dim3(256), 0, st, a);
}

}  // namespace

hipError_t launch_walk_attn(int dt, bool tree, const WalkArgs &a, hipStream_t st) {
  if (dt == 0) tree ? launch_f32<true>(a, st) : launch_f32<false>(a, st);
  else tree ? launch_bf16<true>(a, st) : launch_bf16<false>(a, st);
  return hipGetLastError();
}

}  // namespace specmemo

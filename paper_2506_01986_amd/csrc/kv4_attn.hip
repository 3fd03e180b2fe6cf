// Attention over a pool in 4 bits (kv4.h): prompt tokens, chunks of prompts and single
// tokens (causal), and candidate trees, with or without a prefix that sequences share.
//
// SpecMemo Sec. 3.1: the cache is what the memory budget goes to; a row of 128
// columns takes 68 bytes instead of 256.  Work items, masks, the one-pass softmax and
// the merge of parts are those of the attention over key ranges (walk.h,
// walk_tile.h); what differs is how the rows reach the matrix cores.
//
// bf16 queries:
//   S^T = K Q^T   K's codes and scales are operands as they lie: the scaled product
//                 of 32 x 32 x 64 takes 4-bit values with a scale for each lane's 32
//                 columns.  Its other operand holds six bits, so a query is the sum of
//                 three (Query6).  Three such products of 64 columns take a matrix core
//                 48 ns, the four of the same columns in bf16 62, and K is neither
//                 converted nor read from LDS in 16 bits.  (Two parts of eight bits, the
//                 other way to hold a bf16 value, take 59.)
//   O^T = V^T P^T V is contracted over keys, whose scales differ, so a tile is
//                 converted to bf16 once (by the block's four waves, on its way to LDS)
//                 and read by the transposing loads.
// 8192 tokens over 16384 keys, 64 query heads over 8 (3.3 TFLOP): 2.64 to 2.75 ms, 1.20 to
// 1.25 PFLOP/s, where a large bf16 product of this card's library reaches 1.13 to 1.25:
// matrix cores 0.50 busy at 2.05 GHz, vector units 0.58, loads and barriers 4% of a wave's
// time.  Blocks of 128 rows (two a compute unit) take 1.7 us for a tile, of 64 1.2.
#include <type_traits>

#include "device.h"
#include "internal.h"
#include "kv4.h"
#include "walk.h"
#include "walk_tile.h"

namespace specmemo {

namespace {

constexpr int D = kAttnHeadDim;
constexpr int TK = kAttnKeyTile;
constexpr int kRow4 = D / 2;                  // bytes of a row's codes
constexpr int kScales = D / kKv4Group;        // and of its scales
constexpr int kWaves4 = 4;
constexpr int kKTile4 = TK * kRow4;           // 4 KB of codes
constexpr int kVTile4 = TK * D * 2;           // 16 KB in bf16

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef uint32_t u32x6_t __attribute__((ext_vector_type(6)));
typedef float f32x32_t __attribute__((ext_vector_type(32)));

// A wave's queries as the scaled product's operands, in STEPS products over the
// columns: step s takes group (4 / STEPS) s + h of a lane's row.  A query is the sum of
// its parts, each of six bits (sign, two of exponent, three of mantissa: steps of 1/8
// under 2, 1/4 under 4, 1/2 up to 7.5) times 2^(e - shift), the rest of the one before:
//   bf16  3 parts, shifts 0, 4, 10: values of at least 2^-5 x 2^e are exact, smaller ones
//         leave up to 4 units of the last part and 1/8 of one at most in the end; the 32
//         columns' largest lies in (3.75, 7.5] x 2^e, so those are 2^-7 and 2^-14.9 of it
//         (shifts 0, 5, 10 with a largest under 4.25 would give 2^-15.1; a fourth part
//         2^-20.9, for a third more of the scores' products)
//   fp32  5 parts, shifts 0, 4, 9, 14, 19: a rest is at most 4 units of the next part and
//         leaves 1/8 of one, 2^-22 in the end: within 2^-23.9 of the largest
// Scale byte p % 4 of sc[s][p / 4] is part p's.
template <int STEPS, bool F32>
struct Query6 {
  static constexpr int PARTS = F32 ? 5 : 3;
  u32x6_t part[STEPS][PARTS];
  uint32_t sc[STEPS][(PARTS + 3) / 4];

  static constexpr int shift(int p) { return p == 0 ? 0 : F32 ? 5 * p - 1 : p == 1 ? 4 : 10; }
  __device__ __forceinline__ i32x8_t operand(int s, int p) const {
    const u32x6_t &w = part[s][p];
    return i32x8_t{(int)w[0], (int)w[1], (int)w[2], (int)w[3], (int)w[4], (int)w[5], 0, 0};
  }
  // row: the lane's row; groups of columns past `groups` are zero
  __device__ __forceinline__ void load(bool ok, const void *row, int h, int groups = 4) {
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int g = (4 / STEPS) * s + h;
      const bool has = ok && g < groups;
      // columns in two halves, even and odd, as the conversion takes and interleaves them
      f32x16 even, odd;
      if constexpr (F32) {
        const float *p = static_cast<const float *>(row) + kKv4Group * g;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          f32x4 w = {0.f, 0.f, 0.f, 0.f};
          if (has) w = *reinterpret_cast<const f32x4 *>(p + 4 * i);
          even[2 * i] = w[0];
          odd[2 * i] = w[1];
          even[2 * i + 1] = w[2];
          odd[2 * i + 1] = w[3];
        }
      } else {
        const uint16_t *p = static_cast<const uint16_t *>(row) + kKv4Group * g;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint4 w = ld16_or_zero(has, p + 8 * i);
          const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            even[4 * i + j] = __uint_as_float(u[j] << 16);
            odd[4 * i + j] = __uint_as_float(u[j] & 0xFFFF0000u);
          }
        }
      }
      float top = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(fmaxf(top, fabsf(even[i])), fabsf(odd[i]));
      // 7.5 = 1.875 x 4; a largest of 3.75 x 2^-103 or less is taken as that (scale bytes of all
      // parts stay normal numbers), so that columns far below it come out as 0
      const uint32_t u = __float_as_uint(top);
      const uint32_t e = max((int)(u >> 23) - 2 + ((u & 0x7FFFFFu) > 0x700000u), 24);
#pragma unroll
      for (int i = 0; i < (PARTS + 3) / 4; ++i) sc[s][i] = 0;
#pragma unroll
      for (int p = 0; p < PARTS; ++p) {
        const uint32_t ep = e - shift(p);
        const float unit = __uint_as_float(ep << 23);
        sc[s][p / 4] |= ep << (8 * (p % 4));
        part[s][p] = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, unit);
        if (p + 1 < PARTS) {
          const f32x32_t y = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(part[s][p], unit);
#pragma unroll
          for (int i = 0; i < 16; ++i) {       // exact
            even[i] -= y[2 * i];
            odd[i] -= y[2 * i + 1];
          }
        }
      }
    }
  }
};

template <int STEP, int PART>
__device__ __forceinline__ f32x16 qk_part(uint4 k, const Query6<2, false> &q, f32x16 c, uint32_t kscale) {
  const i32x8_t a = {(int)k.x, (int)k.y, (int)k.z, (int)k.w, 0, 0, 0, 0};
  const i32x8_t b = q.operand(STEP, PART);
  // formats: 4 = four bits, 2 = six bits; the scale byte of each operand is chosen by number
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 2, 2 * STEP, (int)kscale, PART, (int)q.sc[STEP][0]);
}

// Four waves per block; K codes and V values each have a two-slot ring of 64-key
// tiles.  KSPLIT as in the attention over rows of 16 bits: 1: every wave takes whole
// tiles for its 32 rows; 2: two groups of waves over the same rows, one for each half
// of a tile's keys, merged at the end.  (Tiles as loaded in a ring of four, three ahead
// of the products, V converted from there: 8192 tokens over 16384 keys 2790 us against
// 2682; no wave waits for memory as it is.)
template <int KSPLIT, bool TREE>
__device__ __forceinline__ void walk4(const WalkArgs &a, const WalkItem &it, uint8_t (*kring)[kKTile4], uint8_t (*vring)[kVTile4]) {
  constexpr int RW = kWaves4 / KSPLIT, RB = 32 * RW, NSB = 2 / KSPLIT;
  int *const par = reinterpret_cast<int *>(vring[1]);   // filled after the first loop barrier
  static_assert(kWaves4 * 64 >= kMaxNodes && kMaxNodes * 4 <= kVTile4, "one thread per tree node");
  static_assert(KSPLIT == 1 || (RW * 64 * 64 * 4 <= 2 * kVTile4 && RW * 2 * 64 * 4 <= kKTile4), "merge buffers fit the rings");

  const WalkSet &S = it.S;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int rwave = __builtin_amdgcn_readfirstlane(wave % RW), ksb = __builtin_amdgcn_readfirstlane(wave / RW);
  const int h = lane >> 5, g = a.group, L = S.L, P = S.P;
  const int rows = S.T * g;
  const int np = (P + TK - 1) / TK;                     // prefix tiles
  const int kend = walk_keys(S, it.rb, g);              // slab keys of this row block
  const int j0 = it.ch * S.ct, j1 = min(np + (kend + TK - 1) / TK, j0 + S.ct);

  const int64_t head = (int64_t)it.kvh * a.cap_total;
  const int64_t prow = head + S.pbase, srow = head + S.base;
  const uint8_t *const K0 = static_cast<const uint8_t *>(a.k), *const V0 = static_cast<const uint8_t *>(a.v);

  // K codes: wave w loads rows 16 w .. + 15 of a tile, lane l bytes [16 l, +16) of its
  // kilobyte: row 16 w + l / 4, whose logical chunk c lies at c ^ (row / 4 % 4), so that
  // 16 lanes that read one chunk of 16 rows meet 16 different bank groups.
  const int krow = 16 * wave + (lane >> 2);
  const uint32_t kcol = 16 * ((lane & 3) ^ ((lane >> 4) & 3));
  // V codes: thread t has word t % 4 of each of the four groups of row t / 4, so that the
  // values' 16-byte chunks 4 i + t % 4 spread over the banks as the rows' swizzle does.
  const int vrow = tid >> 2, vword = tid & 3;
  struct Raw {
    uint32_t code[4], scale;
  };
  auto place = [&](int j, int &kt, int &end, int64_t &row0) __attribute__((always_inline)) {
    const bool pre = j < np;
    kt = (pre ? j : j - np) * TK;
    end = pre ? P : kend;
    row0 = pre ? prow : srow;
  };
  // rows past the end repeat the last one (finite values, masked out)
  auto issue_k = [&](uint8_t *dst, int j) __attribute__((always_inline)) {
    int kt, end;
    int64_t row0;
    place(j, kt, end, row0);
    const uint8_t *src = uniform_ptr(K0 + row0 * kRow4);
    const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void_t *)(dst + 1024 * wave));
    lds_load16(src, (uint32_t)min(kt + krow, end - 1) * kRow4 + kcol, lds);
  };
  auto load_v = [&](Raw &w, int j) __attribute__((always_inline)) {
    int kt, end;
    int64_t row0;
    place(j, kt, end, row0);
    const uint32_t r = (uint32_t)min(kt + vrow, end - 1);
    const uint8_t *src = V0 + row0 * kRow4;
#pragma unroll
    for (int i = 0; i < 4; ++i) w.code[i] = *reinterpret_cast<const uint32_t *>(src + r * kRow4 + 16 * i + 4 * vword);
    w.scale = *reinterpret_cast<const uint32_t *>(a.vs + row0 * kScales + r * kScales);
  };
  auto store_v = [&](const Raw &w, uint8_t *dst) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<uint4 *>(dst + vrow * (D * 2) + 16 * vswz(vrow, 4 * i + vword)) =
          kv4_bf16x8(w.code[i], kv4_scale(w.scale >> (8 * i) & 255u));
  };
  // K scales: a lane's rows of the sub-blocks, shifted to its half's groups (h and 2 + h)
  auto load_ks = [&](uint32_t (&sc)[NSB], int j) __attribute__((always_inline)) {
    int kt, end;
    int64_t row0;
    place(j, kt, end, row0);
#pragma unroll
    for (int sb = 0; sb < NSB; ++sb) {
      const uint32_t r = (uint32_t)min(kt + 32 * (ksb * NSB + sb) + (lane & 31), end - 1);
      sc[sb] = *reinterpret_cast<const uint32_t *>(a.ks + row0 * kScales + r * kScales);
    }
  };

  Raw raw;
  uint32_t ksn[NSB];
  issue_k(kring[0], j0);
  load_v(raw, j0);
  load_ks(ksn, j0);
  const bool tree = TREE && S.slab;      // the set's slab rows end in a tree
  const int pn = tree && tid < S.T ? a.parent[S.row0 + tid] : -1;
  const int row0 = it.rb * RB + rwave * 32, my_row = row0 + (lane & 31);
  const bool row_ok = my_row < rows;
  const int node = row_ok ? my_row / g : S.T - 1;
  const int hq = it.kvh * g + (row_ok ? my_row % g : 0);
  Query6<2, false> Q;
  Q.load(row_ok, static_cast<const uint16_t *>(a.q) + ((int64_t)(S.row0 + node) * a.n_q + hq) * D, h);
  if (tree && tid < S.T) par[tid] = pn;
  WalkMask M{L, P, h, node};
  if (TREE) {
    ring_barrier();
    if (tree) M.root_path(par, node);
  }
  const int lim_hi = L + min(rows - 1, row0 + 31) / g;   // causal: the last slab key of the wave's last row
  const bool wave_rows = row0 < rows;    // a wave without rows only loads, converts and waits
  store_v(raw, vring[0]);
  if (j0 + 1 < j1) load_v(raw, j0 + 1);

  int kro[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) kro[s] = (lane & 31) * kRow4 + 16 * ((2 * s + h) ^ ((lane >> 2) & 3));
  int vro[D / 32];
  walk_v_offsets(vro);
  const int sb0 = ksb * NSB;
  WalkAcc A;

  // Scores of tile j, and whether the wave has rows that see any of its keys.
  auto sees = [&](int j) __attribute__((always_inline)) { return wave_rows && (TREE || j < np || (j - np) * TK + 32 * sb0 <= lim_hi); };
  auto scores = [&](f32x16 (&Sc)[NSB], const uint8_t *ks, const uint32_t (&ksc)[NSB]) __attribute__((always_inline)) {
    uint4 kf[NSB][2];
#pragma unroll
    for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
      for (int s = 0; s < 2; ++s) kf[sb][s] = *reinterpret_cast<const uint4 *>(ks + (sb0 + sb) * 32 * kRow4 + kro[s]);
#pragma unroll
    for (int sb = 0; sb < NSB; ++sb) {
#pragma unroll
      for (int r2 = 0; r2 < 16; ++r2) Sc[sb][r2] = 0.f;
      const uint32_t sc = ksc[sb] >> (8 * h);
      Sc[sb] = qk_part<0, 2>(kf[sb][0], Q, Sc[sb], sc);
      Sc[sb] = qk_part<1, 2>(kf[sb][1], Q, Sc[sb], sc);
      Sc[sb] = qk_part<0, 1>(kf[sb][0], Q, Sc[sb], sc);
      Sc[sb] = qk_part<1, 1>(kf[sb][1], Q, Sc[sb], sc);
      Sc[sb] = qk_part<0, 0>(kf[sb][0], Q, Sc[sb], sc);
      Sc[sb] = qk_part<1, 0>(kf[sb][1], Q, Sc[sb], sc);
    }
  };

  // Iteration j waits for its loads; after its barrier every wave is done with V of tile
  // j - 1, whose slot takes V of tile j + 1 from the registers that it was loaded to an
  // iteration ago.
  // AHEAD: tile j's scores were made an iteration ago, and tile j + 1's are made beside
  // tile j's weights; K's codes are loaded two tiles ahead.  Where a wave has half a tile's
  // keys its chain is what a tile takes (43 prompts of up to 8 tokens over 800 to 6300 keys:
  // 59.9 us, 52.7 ahead); with whole tiles two waves a SIMD fill each other's gaps and the
  // registers of a second tile cost more (8192 over 16384: 2708, 2795 ahead).
  constexpr bool AHEAD = KSPLIT == 2;
  f32x16 Sc[AHEAD ? 2 : 1][NSB];
  uint32_t ksc[NSB];
  auto next_k = [&](int slot, int j) __attribute__((always_inline)) {      // K of tile j, the next one; its scales become current
#pragma unroll
    for (int sb = 0; sb < NSB; ++sb) ksc[sb] = ksn[sb];
    if (j < j1) {
      issue_k(kring[slot], j);
      load_ks(ksn, j);
    }
  };
  if constexpr (AHEAD) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    ring_barrier();
    next_k(1, j0 + 1);
    scores(Sc[0], kring[0], ksc);
  }
  auto tile = [&](int j, auto slot_c) __attribute__((always_inline)) {
    constexpr int slot = decltype(slot_c)::value, cur = AHEAD ? slot : 0;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    ring_barrier();
    const bool more = j + 1 < j1, pre = j < np, now = sees(j);     // (if not now, at no later tile)
    next_k(AHEAD ? slot : slot ^ 1, AHEAD ? j + 2 : j + 1);
    auto put_v = [&]() __attribute__((always_inline)) {
      if (more) store_v(raw, vring[slot ^ 1]);
      if (j + 2 < j1) load_v(raw, j + 2);
    };
    if (!AHEAD) put_v();
    uint32_t pk[2 * NSB][4];
    if (now) {
      if (!AHEAD) scores(Sc[cur], kring[slot], ksc);
      walk_mask<NSB, TREE>(Sc[cur], M, pre, (pre ? j : j - np) * TK, pre ? P : kend, 32 * sb0);
      walk_max<NSB>(Sc[cur], A, a.scale_log2);
      if constexpr (AHEAD) scores(Sc[cur ^ 1], kring[slot ^ 1], ksc);        // after the last tile: of what the slot held, unused
      walk_weights<NSB>(Sc[cur], A, a.scale_log2, pk);
    }
    if (AHEAD) put_v();
    if (now) walk_pv<NSB>(pk, A, vring[slot] + 32 * sb0 * (D * 2), vro);
  };
  for (int j = j0; j < j1; j += 2) {
    tile(j, std::integral_constant<int, 0>{});
    if (j + 1 < j1) tile(j + 1, std::integral_constant<int, 1>{});
  }

  walk_finish<KSPLIT>(a, it, A, row_ok, wave_rows, node, hq, rwave, ksb, reinterpret_cast<float *>(vring[0]),
                      reinterpret_cast<float *>(kring[0]));
}

// Rows of few queries (up to 16: a token's query heads, or a small tree's nodes) are
// bound by memory: the waves of a block share nothing but the merge at the end, and
// each takes every fourth tile of the item with the next one's loads in flight
// (8.7 KB a wave, 70 KB a compute unit).  Queries fill the 16-wide products: a tile's
// scores are 16 to a lane, half of those of the 32-wide ones.  32 single tokens over 256
// to 16384 keys, 64 query heads over 8 (188 MB): 83.8 us as 64-row blocks, 41 so, 35 of
// them the walk: 6.7 TB/s between the start (6 us) and the last blocks' end, then the merge.
//   S^T: 16 keys x 128 columns a product.  A lane's operand is the codes of one group
//        of its key, 16 bytes as they lie in memory, and that group's scale.
//   O^T: V is converted as it arrives, through the wave's own 16 KB of LDS.  A product
//        contracts 32 keys, the four of each lane group from two blocks of 16, which is
//        where the scores left the weights.
// fp32 queries (DB groups of 32 columns) take the same way, up to 32 rows an item: past
// 16, two waves have rows 0 to 15 and two the others.  A weight is the sum of three bf16
// numbers, each the rest of the one before (24 bits), V is exact in bf16, and the sums
// are fp32: the products cost a sixth of the fp32 matrix instructions' (2 x 32 rows x 64
// keys x 128 columns: 6.9 us of those a wave).
constexpr int kFewRows = 16;

// Chunk of 16 bytes c of V row r: eight lanes that write (two rows, four groups) and 32
// that read (eight rows, one pair of chunks) meet different banks.
__device__ __forceinline__ int few_swz(int r, int c) { return c ^ ((r & 3) << 2) ^ (((r ^ (r >> 2)) & 1) << 1); }

// The maximum or sum over the four lanes l % 16 + 16 G.
__device__ __forceinline__ float max_of_groups(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max_with_other_half(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float sum_of_groups(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return sum_with_other_half(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

template <bool TREE, bool F32, int DB>
__device__ __forceinline__ void walk4_few(const WalkArgs &a, const WalkItem &it, uint8_t (*lds)[kVTile4], int *par) {
  constexpr int ROW = 16 * DB;            // bytes of a row's codes
  const WalkSet &S = it.S;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int q16 = lane & 15, G = lane >> 4, g = a.group, L = S.L, P = S.P;
  const int rows = S.T * g;
  const int nr = F32 && rows - 32 * it.rb > kFewRows ? 2 : 1;     // groups of 16 rows, each with 4 / nr waves
  const int my_row = 32 * it.rb + kFewRows * (wave & (nr - 1)) + q16;
  const int np = (P + TK - 1) / TK;
  const int kend = walk_keys(S, it.rb, g);
  const int j0 = it.ch * S.ct, j1 = min(np + (kend + TK - 1) / TK, j0 + S.ct);
  const int64_t head = (int64_t)it.kvh * a.cap_total;
  const int64_t prow = head + S.pbase, srow = head + S.base;
  const uint8_t *const K0 = static_cast<const uint8_t *>(a.k), *const V0 = static_cast<const uint8_t *>(a.v);
  uint8_t *const mem = lds[wave];

  // A tile as it is loaded: K codes of the four blocks of 16 keys (key q16, group G), V codes of
  // rows 16 n + lane / 4 (group lane % 4), and their scales.
  struct Raw {
    uint4 k[4], v[4];
    uint32_t ks[4], vs[4];
  };
  auto load = [&](Raw &w, int j) __attribute__((always_inline)) {
    const bool pre = j < np;
    const int kt = (pre ? j : j - np) * TK, end = pre ? P : kend;
    const int64_t row0 = pre ? prow : srow;
    const uint8_t *const kb = K0 + row0 * ROW, *const vb = V0 + row0 * ROW;
    const uint8_t *const ksb = a.ks + row0 * DB, *const vsb = a.vs + row0 * DB;
#pragma unroll
    for (int n = 0; n < 4; ++n) {       // rows past the end repeat the last one (finite values, masked out)
      const uint32_t r = (uint32_t)min(kt + 16 * n + q16, end - 1);
      w.k[n] = ld16_or_zero(DB == 4 || G < DB, kb + r * ROW + 16 * G);
      w.ks[n] = DB == 4 || G < DB ? ksb[r * DB + G] : 127u;
    }
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const uint32_t r = (uint32_t)min(kt + 16 * n + (lane >> 2), end - 1);
      w.v[n] = ld16_or_zero(DB == 4 || (lane & 3) < DB, vb + r * ROW + 16 * (lane & 3));
      w.vs[n] = DB == 4 || (lane & 3) < DB ? vsb[r * DB + (lane & 3)] : 127u;
    }
  };

  Raw nxt;
  const int stride = kWaves4 / nr, jw = j0 + (nr == 2 ? wave >> 1 : wave);
  if (jw < j1) load(nxt, jw);
  const bool tree = TREE && S.slab;
  const bool row_ok = my_row < rows;
  const int node = row_ok ? my_row / g : S.T - 1;
  const int hq = it.kvh * g + (row_ok ? my_row % g : 0);
  Query6<1, F32> Q;
  Q.load(row_ok, static_cast<const uint8_t *>(a.q) + ((int64_t)(S.row0 + node) * a.n_q + hq) * (32 * DB * (F32 ? 4 : 2)), G, DB);
  WalkMask M{L, P, 0, node};
  if (TREE) {
    if (tree && tid < S.T) par[tid] = a.parent[S.row0 + tid];
    ring_barrier();                       // (does not wait for the tile)
    if (tree) M.root_path(par, node);
  }

  float m = -INFINITY, lsum = 0.f;
  f32x4 O[2 * DB];
#pragma unroll
  for (int i = 0; i < 2 * DB; ++i) O[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const bf16x2_t ones = __builtin_bit_cast(bf16x2_t, 0x3F803F80u);

  for (int j = jw; j < j1; j += stride) {
    const Raw cur = nxt;
    if (j + stride < j1) load(nxt, j + stride);
    const bool pre = j < np;
    const int kt = (pre ? j : j - np) * TK;
    f32x4 Sc[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const i32x8_t ka = {(int)cur.k[n].x, (int)cur.k[n].y, (int)cur.k[n].z, (int)cur.k[n].w, 0, 0, 0, 0};
      auto part = [&](auto p) __attribute__((always_inline)) {       // smallest parts first
        Sc[n] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(ka, Q.operand(0, p), Sc[n], 4, 2, 0, (int)cur.ks[n], p % 4, (int)Q.sc[0][p / 4]);
      };
      Sc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
      if constexpr (F32) {
        part(std::integral_constant<int, 4>{});
        part(std::integral_constant<int, 3>{});
      }
      part(std::integral_constant<int, 2>{});
      part(std::integral_constant<int, 1>{});
      part(std::integral_constant<int, 0>{});
    }
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int r = 16 * n + (lane >> 2), c = lane & 3;
      const float unit = kv4_scale(cur.vs[n]);
      const uint32_t w[4] = {cur.v[n].x, cur.v[n].y, cur.v[n].z, cur.v[n].w};
      if (DB == 4 || c < DB) {
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4 *>(mem + r * (D * 2) + 16 * few_swz(r, 4 * c + i)) = kv4_bf16x8(w[i], unit);
      }
    }
    // entry r of block n is key kt + 16 n + 4 G + r
    if (TREE && !pre) {
      if (kt + TK > L) {
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int t = kt + 16 * n + 4 * G + r;
            const uint32_t rel = (uint32_t)(t - L) & 127u;
            const bool anc = ((rel < 64 ? M.alo : M.ahi) >> (rel & 63)) & 1u;
            Sc[n][r] = (t < kend) & ((t < L) | anc) ? Sc[n][r] : -INFINITY;
          }
      }
    } else if (kt + TK - 1 > (pre ? P - 1 : M.lim_lo)) {
      const int vis = (pre ? P - 1 : M.lim) - kt - 4 * G;
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) Sc[n][r] = 16 * n + r <= vis ? Sc[n][r] : -INFINITY;
    }
    float tm = fmaxf(fmaxf(Sc[0][0], Sc[0][1]), Sc[0][2]);
#pragma unroll
    for (int e = 3; e < 15; e += 2) tm = fmaxf(fmaxf(tm, Sc[e >> 2][e & 3]), Sc[(e + 1) >> 2][(e + 1) & 3]);
    tm = fmaxf(tm, Sc[3][3]);
    const float tmax = max_of_groups(tm) * a.scale_log2;
    const bool need = tmax > m + kRescaleSlack;       // as in walk_softmax_pv
    if (__builtin_amdgcn_ballot_w64(need)) {
      const float m_new = need ? tmax : m;
      const float alpha = need ? (m == -INFINITY ? 0.f : fast_exp2(m - m_new)) : 1.f;
      m = m_new;
      lsum *= alpha;
#pragma unroll
      for (int i = 0; i < 2 * DB; ++i) O[i] *= alpha;
    }
    const float m_use = m == -INFINITY ? 0.f : m;
    // bf16: weights are rounded to the product's operand type (2^-8 of a weight, as the
    // inputs' own type), and their sum is taken of the rounded ones.
    constexpr int WP = F32 ? 3 : 1;
    uint32_t pk[WP][2][4];
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        float p0 = fast_exp2(fmaf(Sc[n][r], a.scale_log2, -m_use)), p1 = fast_exp2(fmaf(Sc[n][r + 1], a.scale_log2, -m_use));
        if (F32) lsum += p0 + p1;
#pragma unroll
        for (int w = 0; w < WP; ++w) {
          const uint32_t u = pack_bf16x2(p0, p1);
          pk[w][n >> 1][2 * (n & 1) + (r >> 1)] = u;
          p0 -= __uint_as_float(u << 16);                // exact
          p1 -= __uint_as_float(u & 0xFFFF0000u);
        }
      }
    wave_fence();                         // V: from the lanes that converted it to those that multiply
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      if (!F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) lsum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pk[0][b][e]), ones, lsum, false);
      }
#pragma unroll
      for (int i = 0; i < 2 * DB; ++i) {
        // lane e of a group of 16 gives the place of piece e % 4 (8 bytes) of row e / 4 and gets column e of four rows
        const int r0 = 32 * b + 4 * G + (q16 >> 2), r1 = r0 + 16;
        const int at0 = r0 * (D * 2) + 16 * few_swz(r0, 2 * i + ((q16 & 3) >> 1)) + 8 * (q16 & 1);
        const int at1 = r1 * (D * 2) + 16 * few_swz(r1, 2 * i + ((q16 & 3) >> 1)) + 8 * (q16 & 1);
        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(mem + at0));
        const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(mem + at1));
        const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int w = WP - 1; w >= 0; --w)
          O[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, __builtin_bit_cast(bf16x8, uint4{pk[w][b][0], pk[w][b][1], pk[w][b][2], pk[w][b][3]}), O[i], 0, 0, 0);
      }
    }
    wave_fence();                         // the next tile, or the parts, take V's place
  }

  // The waves' parts: O[i] of a lane is columns 16 i + 4 G .. + 3 of row q16.
  constexpr int ML = 32 * DB * kFewRows;
  float *const part = reinterpret_cast<float *>(mem);
#pragma unroll
  for (int i = 0; i < 2 * DB; ++i) *reinterpret_cast<f32x4 *>(part + ((4 * i + G) * kFewRows + q16) * 4) = O[i];
  const float ltot = sum_of_groups(lsum);
  if (G == 0) {
    part[ML + q16] = m;
    part[ML + kFewRows + q16] = ltot;
  }
  __syncthreads();
  const bool direct = walk_direct(S, it.rb, g);
  float *const u = direct ? nullptr : a.part + (int64_t)walk_part(a, S, it.kvh, it.rb, it.ch) * walk_unit_floats(DB);
  for (int e = tid; e < 8 * DB * kFewRows * nr; e += 64 * kWaves4) {
    const int row = e & 15, grp = nr == 2 ? (e >> 4) & 1 : 0, quad = e >> (nr == 2 ? 5 : 4);     // columns 4 quad .. + 3
    const int urow = kFewRows * grp + row, at_row = 32 * it.rb + urow;
    if (at_row >= rows) continue;
    float w[kWaves4], mx = -INFINITY, lt = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < kWaves4; ++v) {
      w[v] = nr == 1 || (v & 1) == grp ? reinterpret_cast<const float *>(lds[v])[ML + row] : -INFINITY;
      mx = fmaxf(mx, w[v]);
    }
#pragma unroll
    for (int v = 0; v < kWaves4; ++v) {
      if (nr == 2 && (v & 1) != grp) continue;
      const float *pv = reinterpret_cast<const float *>(lds[v]);
      const float wt = w[v] == -INFINITY ? 0.f : fast_exp2(w[v] - mx);
      lt = fmaf(pv[ML + kFewRows + row], wt, lt);
      const f32x4 x = *reinterpret_cast<const f32x4 *>(pv + (quad * kFewRows + row) * 4);
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] = fmaf(x[c], wt, o[c]);
    }
    if (direct) {
      const float inv = 1.f / lt;
      const int64_t at = ((int64_t)(S.row0 + at_row / g) * a.n_q + it.kvh * g + at_row % g) * (32 * DB) + 4 * quad;
      if constexpr (F32)
        *reinterpret_cast<f32x4 *>(static_cast<float *>(a.out) + at) = f32x4{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
      else
        *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + at) = uint2{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
    } else {                              // in the order of write_part: row % 32 + 32 h, columns 32 i + 8 q + 4 h
      *reinterpret_cast<f32x4 *>(u + ((quad >> 1) * 64 + urow + 32 * (quad & 1)) * 4) = o;
      if (quad == 0) {
        u[DB * 1024 + urow] = mx;
        u[DB * 1024 + 32 + urow] = lt;
      }
    }
  }
}

template <bool TREE>
__global__ __launch_bounds__(kWaves4 * 64, 2) void walk4_attn_bf16(WalkArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t kring[2][kKTile4];
  __shared__ __attribute__((aligned(1024))) uint8_t vring[4][kVTile4];   // two slots, or a tile of each wave
  WalkItem it;
  decode_walk(a, blockIdx.x, it);
  if (it.S.rb == 32) walk4_few<TREE, false, 4>(a, it, vring, reinterpret_cast<int *>(kring[0]));
  else if (it.S.rb == 64) walk4<2, TREE>(a, it, kring, vring);
  else walk4<1, TREE>(a, it, kring, vring);
}

template <int DB, bool TREE>
__global__ __launch_bounds__(kWaves4 * 64, 2) void walk4_attn_f32(WalkArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kWaves4][kVTile4];
  __shared__ int par[kMaxNodes];
  WalkItem it;
  decode_walk(a, blockIdx.x, it);
  walk4_few<TREE, true, DB>(a, it, lds, par);
}

template <bool TREE>
void launch4_f32(const WalkArgs &a, hipStream_t st) {
  const dim3 grid(a.blocks), block(kWaves4 * 64);
  switch (a.head_dim / 32) {
    case 1: hipLaunchKernelGGL((walk4_attn_f32<1, TREE>), grid, block, 0, st, a); break;
    case 2: hipLaunchKernelGGL((walk4_attn_f32<2, TREE>), grid, block, 0, st, a); break;
    case 3: hipLaunchKernelGGL((walk4_attn_f32<3, TREE>), grid, block, 0, st, a); break;
    default: hipLaunchKernelGGL((walk4_attn_f32<4, TREE>), grid, block, 0, st, a);
  }
}

}  // namespace

hipError_t launch_walk4_attn(int dt, bool tree, const WalkArgs &a, hipStream_t st) {
  if (dt == 0) {
    tree ? launch4_f32<true>(a, st) : launch4_f32<false>(a, st);
  } else if (tree) {
    hipLaunchKernelGGL((walk4_attn_bf16<true>), dim3(a.blocks), dim3(kWaves4 * 64), 0, st, a);
  } else {
    hipLaunchKernelGGL((walk4_attn_bf16<false>), dim3(a.blocks), dim3(kWaves4 * 64), 0, st, a);
  }
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || !a.cblocks ? e : launch_walk_combine(dt, a, st);
}

}  // namespace specmemo

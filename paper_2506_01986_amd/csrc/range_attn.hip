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

#include "device.h"
#include "internal.h"
#include "walk.h"
#include "walk_tile.h"

namespace specmemo {

namespace {

constexpr int D = kAttnHeadDim;
constexpr int TK = kAttnKeyTile;

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
  WalkMask M{L, P, h, node};
  if (TREE) {
    ring_barrier();
    if (tree) M.root_path(par, node);
  }
  // causal: the last slab key of the wave's last row
  const int lim_hi = L + min(rows - 1, row0 + 31) / g;
  const bool wave_rows = row0 < rows;    // a wave without rows only loads and waits

  int kro[D / 16];
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) kro[ks] = (lane & 31) * (D * 2) + 16 * ((2 * ks + h) ^ (lane & 15));
  int vro[D / 32];
  walk_v_offsets(vro);
  const int sb0 = ksb * NSB;

  WalkAcc A;
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
    walk_mask<NSB, TREE>(Sc, M, pre, kt, pre ? P : kend, 32 * sb0);
    walk_softmax_pv<NSB>(Sc, A, vs + 32 * sb0 * (D * 2), vro, a.scale_log2);
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

  walk_finish<KSPLIT>(a, it, A, row_ok, wave_rows, node, hq, rwave, ksb, reinterpret_cast<float *>(kring[0]),
                      reinterpret_cast<float *>(vring[0]));
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
  walk_finish_f32<DB, W>(a, it, O, m, l, row_ok, node, hq, merge);
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
}

}  // namespace

hipError_t launch_walk_combine(int dt, const WalkArgs &a, hipStream_t st) {
  const dim3 grid(a.cblocks), block(256);
  if (dt != 0) {
    hipLaunchKernelGGL((walk_combine<D / 32, true>), grid, block, 0, st, a);
  } else {
    switch ((a.head_dim + 31) / 32) {
      case 1: hipLaunchKernelGGL((walk_combine<1, false>), grid, block, 0, st, a); break;
      case 2: hipLaunchKernelGGL((walk_combine<2, false>), grid, block, 0, st, a); break;
      case 3: hipLaunchKernelGGL((walk_combine<3, false>), grid, block, 0, st, a); break;
      default: hipLaunchKernelGGL((walk_combine<4, false>), grid, block, 0, st, a);
    }
  }
  return hipGetLastError();
}

hipError_t launch_walk_attn(int dt, bool tree, const WalkArgs &a, hipStream_t st) {
  if (dt == 0) tree ? launch_f32<true>(a, st) : launch_f32<false>(a, st);
  else tree ? launch_bf16<true>(a, st) : launch_bf16<false>(a, st);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || !a.cblocks ? e : launch_walk_combine(dt, a, st);
}

}  // namespace specmemo

// The bf16 tile loop of the attention over key ranges behind the scores: masks, one
// pass softmax and the product with V, and what becomes of a wave's rows at the end.
// A wave has 32 query rows; lane l and its other half l ^ 32 share row l % 32, and
// score entry r of a 32-key block is key 8 (r / 4) + 4 (l / 32) + r % 4 of the block.
#pragma once

#include "attn_tile.h"
#include "walk.h"

namespace specmemo {

constexpr float kRescaleSlack = 8.f;   // log2 units: softmax weights stay <= 256 between rescales

// What a lane's query row sees of the slab.
struct WalkMask {
  int L, P, h;
  int lim, lim_lo;           // causal: last slab key of this lane's row and of the wave's first row
  uint64_t alo = 0, ahi = 0; // trees: ancestor-or-self bits of this lane's node
  __device__ __forceinline__ WalkMask(int L, int P, int h, int node)
      : L(L), P(P), h(h), lim(L + node), lim_lo(L + __builtin_amdgcn_readfirstlane(node)) {}
  __device__ __forceinline__ void root_path(const int *par, int node) {
    for (int u = node; u >= 0; u = par[u]) {
      alo |= u < 64 ? 1ull << (u & 63) : 0ull;
      ahi |= u < 64 ? 0ull : 1ull << (u & 63);
    }
  }
};

// Masks the scores of keys kt + k0 .. of a prefix or slab tile (64 keys from kt); kend:
// slab keys of the row block.
template <int NSB, bool TREE>
__device__ __forceinline__ void walk_mask(f32x16 (&Sc)[NSB], const WalkMask &M, bool pre, int kt, int kend, int k0) {
  const int L = M.L, h = M.h;
  if (TREE && !pre) {
    if (kt + kAttnKeyTile > L) {
#pragma unroll
      for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
        for (int r2 = 0; r2 < 16; ++r2) {
          const int t = kt + k0 + 32 * sb + 8 * (r2 >> 2) + 4 * h + (r2 & 3);
          const uint32_t rel = (uint32_t)(t - L) & 127u;
          const bool anc = ((rel < 64 ? M.alo : M.ahi) >> (rel & 63)) & 1u;
          Sc[sb][r2] = (t < kend) & ((t < L) | anc) ? Sc[sb][r2] : -INFINITY;
        }
    }
  } else if (kt + kAttnKeyTile - 1 > (pre ? M.P - 1 : M.lim_lo)) {
    const int vis = (pre ? M.P - 1 : M.lim) - kt - k0 - 4 * h;
#pragma unroll
    for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
      for (int r2 = 0; r2 < 16; ++r2)
        Sc[sb][r2] = 32 * sb + 8 * (r2 >> 2) + (r2 & 3) <= vis ? Sc[sb][r2] : -INFINITY;
  }
}

// A wave's running maximum (log2 units), sum of weights and unnormalised O^T.
struct WalkAcc {
  float m = -INFINITY, lsum = 0.f;
  f32x16 O[kAttnHeadDim / 32];
  __device__ __forceinline__ WalkAcc() {
#pragma unroll
    for (int i = 0; i < kAttnHeadDim / 32; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) O[i][r] = 0.f;
  }
};

// A lane's byte offsets into a V tile (rows of 256 bytes, chunks swizzled by vswz)
// for the transposing loads of the four 32-column blocks.
__device__ __forceinline__ void walk_v_offsets(int (&vro)[kAttnHeadDim / 32]) {
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int tj = (lane & 15) >> 2, tq = lane & 3;
  const int te = 2 * ((lane >> 4) & 1) + (tq >> 1);
#pragma unroll
  for (int i = 0; i < kAttnHeadDim / 32; ++i) vro[i] = (4 * h + tj) * (kAttnHeadDim * 2) + 64 * (i ^ tj) + 16 * te + 8 * (tq & 1);
}

// The running maximum after NSB x 32 scores of every row.
template <int NSB>
__device__ __forceinline__ void walk_max(const f32x16 (&Sc)[NSB], WalkAcc &A, float scale_log2) {
  constexpr int D = kAttnHeadDim;
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
  const float tmax = max_with_other_half(tm) * scale_log2;
  // Lazy rescaling: m moves only when a score exceeds it by more than kRescaleSlack.
  const bool need = tmax > A.m + kRescaleSlack;
  if (__builtin_amdgcn_ballot_w64(need)) {
    const float m_new = need ? tmax : A.m;
    const float alpha = need ? (A.m == -INFINITY ? 0.f : fast_exp2(A.m - m_new)) : 1.f;
    A.m = m_new;
    A.lsum *= alpha;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int r2 = 0; r2 < 16; ++r2) A.O[i][r2] *= alpha;
  }
}

// The softmax weights of NSB x 32 keys in bf16, as the second operand of the product with V.
template <int NSB>
__device__ __forceinline__ void walk_weights(const f32x16 (&Sc)[NSB], WalkAcc &A, float scale_log2, uint32_t (&pk)[2 * NSB][4]) {
  const bf16x2_t ones = __builtin_bit_cast(bf16x2_t, 0x3F803F80u);
  const float m_use = A.m == -INFINITY ? 0.f : A.m;
  // Weights are rounded to bf16, the matrix product's operand type (2^-8 of a
  // weight, as the inputs' own type); their sum is taken of the rounded ones.
#pragma unroll
  for (int sb = 0; sb < NSB; ++sb)
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float p0 = fast_exp2(fmaf(Sc[sb][8 * half + 2 * q], scale_log2, -m_use));
        const float p1 = fast_exp2(fmaf(Sc[sb][8 * half + 2 * q + 1], scale_log2, -m_use));
        pk[2 * sb + half][q] = pack_bf16x2(p0, p1);
      }
#pragma unroll
  for (int mh = 0; mh < 2 * NSB; ++mh)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      A.lsum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pk[mh][q]), ones, A.lsum, false);
}

// Their product with V; vs: V row of the first of the keys.
template <int NSB>
__device__ __forceinline__ void walk_pv(const uint32_t (&pk)[2 * NSB][4], WalkAcc &A, const uint8_t *vs, const int (&vro)[kAttnHeadDim / 32]) {
  constexpr int D = kAttnHeadDim;
#pragma unroll
  for (int mh = 0; mh < 2 * NSB; ++mh) {
    const bf16x8 pf = __builtin_bit_cast(bf16x8, uint4{pk[mh][0], pk[mh][1], pk[mh][2], pk[mh][3]});
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const uint8_t *p = vs + 16 * mh * (D * 2) + vro[i];
      const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)p);
      const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(p + 8 * (D * 2)));
      const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      A.O[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf, A.O[i], 0, 0, 0);
    }
  }
}

template <int NSB>
__device__ __forceinline__ void walk_softmax_pv(const f32x16 (&Sc)[NSB], WalkAcc &A, const uint8_t *vs, const int (&vro)[kAttnHeadDim / 32],
                                                float scale_log2) {
  uint32_t pk[2 * NSB][4];
  walk_max<NSB>(Sc, A, scale_log2);
  walk_weights<NSB>(Sc, A, scale_log2, pk);
  walk_pv<NSB>(pk, A, vs, vro);
}

// The end of a row block's walk: KSPLIT = 2 merges the two wave groups through LDS (mo:
// 32 KB, ml: 2 KB, both free after the last tile), then the wave's rows go to `out`
// or, unnormalised, to the parts.
template <int KSPLIT>
__device__ __forceinline__ void walk_finish(const WalkArgs &a, const WalkItem &it, WalkAcc &A, bool row_ok, bool wave_rows, int node,
                                            int hq, int rwave, int ksb, float *mo, float *ml) {
  constexpr int D = kAttnHeadDim;
  const WalkSet &S = it.S;
  const int lane = threadIdx.x & 63, h = lane >> 5, g = a.group;
  float m = A.m, ltot = sum_with_other_half(A.lsum);
  if constexpr (KSPLIT == 2) {
    // Every wave is past its last read of the rings and no load is in flight.
    ring_barrier();
    if (ksb == 1) {
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int r2 = 0; r2 < 16; ++r2) mo[(rwave * 64 + 16 * i + r2) * 64 + lane] = A.O[i][r2];
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
      for (int r2 = 0; r2 < 16; ++r2) A.O[i][r2] = A.O[i][r2] * w0 + mo[(rwave * 64 + 16 * i + r2) * 64 + lane] * w1;
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
        const auto &o = A.O[i];
        const uint32_t a0 = pack_bf16x2(o[8 * p] * inv, o[8 * p + 1] * inv), a1 = pack_bf16x2(o[8 * p + 2] * inv, o[8 * p + 3] * inv);
        const uint32_t b0 = pack_bf16x2(o[8 * p + 4] * inv, o[8 * p + 5] * inv), b1 = pack_bf16x2(o[8 * p + 6] * inv, o[8 * p + 7] * inv);
        const auto s0 = __builtin_amdgcn_permlane32_swap(a0, b0, false, false), s1 = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
        *reinterpret_cast<uint4 *>(op + 32 * i + 16 * p + 8 * h) = uint4{s0[0], s1[0], s0[1], s1[1]};
      }
  } else {
    write_part<D / 32>(a.part + (int64_t)(walk_part(a, S, it.kvh, it.rb, it.ch) + rwave) * walk_unit_floats(D / 32), A.O, m, ltot, row_ok);
  }
}

// The end of an fp32 row block: its W waves' parts of the same 32 rows are merged
// through LDS, wave w taking entries 4 DB / W w ... of the accumulator order, then
// written to `out` or to the parts.
template <int DB, int W>
__device__ __forceinline__ void walk_finish_f32(const WalkArgs &a, const WalkItem &it, const f32x16 (&O)[DB], float m, float l,
                                                bool row_ok, int node, int hq, float (&merge)[W][walk_unit_floats(DB)]) {
  constexpr int UF = walk_unit_floats(DB);
  const WalkSet &S = it.S;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, g = a.group, d = a.head_dim;
  write_part<DB>(merge[wave], O, m, sum_with_other_half(l), true);
  __syncthreads();
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
    const int col = 32 * (iq >> 2) + 8 * (iq & 3) + 4 * h;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const f32x4 v = *reinterpret_cast<const f32x4 *>(&merge[w][(iq * 64 + lane) * 4]);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = fmaf(v[e], mw[w], o[e]);
    }
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

}  // namespace specmemo

// Work items of the attention over key ranges (prompts, candidate trees over shared
// prefixes), whatever type the pool's rows are held in: which set, KV head, row
// block and chunk a block has, and where its parts go.  The kernels take a WalkArgs
// as their first argument.
#pragma once

#include "device.h"
#include "internal.h"

namespace specmemo {

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

}  // namespace specmemo

// Rules on a verify step's logits before acceptance or sampling: penalties for
// tokens that already occurred, added biases, grammar masks; and the token counts
// the penalties read.
//
// A node's history is the sequence's committed tokens and the tokens on its own
// root path (SpecMemo App. A.1: each candidate is verified as the continuation of
// its path).  Per token v of node u's row:
//
//   c = counts[b][v] + occurrences of v on the root path
//   x = z;  c > 0: x = (x > 0 ? x / repetition : x * repetition) - frequency c - presence
//   x = x + bias[b][v];  not allowed by the node's mask: x = -inf
//
// in fp32, rounded once to the logits' type.
#include "device.h"
#include "internal.h"

namespace specmemo {

namespace {

constexpr int kNT = 256;          // threads of a rules block
constexpr int kRows = 16;         // node rows a block works through
constexpr int kInFlight = 4;      // rows whose loads are in flight at once

// Chunks of 16 bytes at 16-byte aligned addresses; a row whose length keeps it from
// starting or ending on one has up to 2 (V - 1) single values, before and after.
template <int DT>
struct Chunk {
  static constexpr int V = DT == 0 ? 4 : 8;
  static __device__ __forceinline__ float get(const uint4 &w, int e) {
    const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
    if (DT == 0) return __uint_as_float(ws[e]);
    return __uint_as_float(e & 1 ? ws[e >> 1] & 0xFFFF0000u : ws[e >> 1] << 16);
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[V]) {
    if constexpr (DT == 0)
      return uint4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
    else
      return uint4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
  }
};

// One block: kRows rows of a sequence, one segment of kNT chunks of the vocabulary.
// The segment's counts and biases are read once for all the rows and kept in LDS
// (element e of chunk i at e * kStride + i: any alignment of the rows reads them
// without bank conflicts).
template <int DT>
__global__ __launch_bounds__(kNT) void logit_rules_kernel(RulesArgs a) {
  constexpr int V = Chunk<DT>::V, SEG = kNT * V, COLS = SEG + V, kStride = kNT + 2;
  __shared__ int s_cnt[V * kStride];
  __shared__ int s_bias[V * kStride];              // index + 1 of the token's last bias entry, then its value
  __shared__ uint8_t s_any[kNT + 1];               // chunk-sized groups with a count or a bias
  __shared__ int s_par[kMaxNodes], s_loc[kMaxNodes], s_hit[kMaxNodes], s_after[kMaxNodes];
  const int tid = threadIdx.x;
  const int b = blockIdx.y / a.groups, r0 = blockIdx.y % a.groups * kRows;
  const int n0 = a.node_off[b], N = a.node_off[b + 1] - n0;
  if (r0 >= N) return;
  const int col0 = blockIdx.x * SEG;
  auto at = [&](int c) { return c % V * kStride + c / V; };   // column of the segment -> LDS

  for (int c = tid; c < V * kStride; c += kNT) s_bias[c] = 0;
  for (int c = tid; c < COLS; c += kNT)
    s_cnt[at(c)] = a.counts && col0 + c < a.vocab ? a.counts[(int64_t)b * a.vocab + col0 + c] : 0;
  if (a.penalties)
    for (int n = tid; n < N; n += kNT) {
      const int t = a.node_tok[n0 + n];
      s_par[n] = n == 0 ? -1 : a.parent[n0 + n];
      s_loc[n] = t >= col0 && t < min(col0 + COLS, a.vocab) ? t - col0 : -1;
    }
  __syncthreads();
  // Nearest node at or above n, and strictly above it, whose token lies in the segment.
  if (a.penalties)
    for (int n = tid; n < N; n += kNT) {
      int u = s_par[n];
      while (u >= 0 && s_loc[u] < 0) u = s_par[u];
      s_after[n] = u;
      s_hit[n] = s_loc[n] >= 0 ? n : u;
    }
  if (a.n_bias > 0) {
    const int j1 = min(max(a.bias_off[b + 1], 0), a.n_bias);
    for (int j = max(a.bias_off[b], 0) + tid; j < j1; j += kNT) {
      const int c = a.bias_id[j] - col0;
      if (a.bias_id[j] >= 0 && c >= 0 && c < COLS) atomicMax(&s_bias[at(c)], j + 1);   // the last entry of an id counts
    }
    __syncthreads();
    for (int c = tid; c < V * kStride; c += kNT) s_bias[c] = s_bias[c] ? __float_as_int(a.bias_val[s_bias[c] - 1]) : 0;
  }
  __syncthreads();
  for (int i = tid; i <= kNT; i += kNT) {
    int any = 0;
#pragma unroll
    for (int e = 0; e < V; ++e) any |= (a.penalties ? s_cnt[e * kStride + i] : 0) | s_bias[e * kStride + i];
    s_any[i] = any != 0;
  }
  __syncthreads();

  const float rep = a.repetition ? a.repetition[b] : 1.f, inv_rep = 1.f / rep;
  const float pres = a.presence ? a.presence[b] : 0.f, freq = a.frequency ? a.frequency[b] : 0.f;
  // (x / repetition as a product with its reciprocal: one rounding of 2^-24 more, far below the logits' own)
  auto apply = [&](float x, int c, float bias, bool allowed) {
    const float y = fmaf(-freq, (float)c, (x > 0.f ? x * inv_rep : x * rep) - pres);
    x = c > 0 ? y : x;
    return allowed ? x + bias : -INFINITY;
  };
  auto mask_bits = [&](int m, int col) -> uint32_t {   // bit e: column col + e is allowed
    const uint32_t *w = a.mask + (int64_t)m * a.mask_words;
    const int i = col >> 5;
    return (uint32_t)(((uint64_t)w[min(i + 1, a.mask_words - 1)] << 32 | w[i]) >> (col & 31));
  };

  const int r1 = min(N, r0 + kRows);
  for (int rr = r0; rr < r1; rr += kInFlight) {
    uint4 w[kInFlight];
    uint32_t bits[kInFlight];
    int head[kInFlight], nch[kInFlight], mi[kInFlight];
    const int chunk = blockIdx.x * kNT + tid;
#pragma unroll
    for (int f = 0; f < kInFlight; ++f) {
      const int r = min(rr + f, r1 - 1);
      const int64_t base = (int64_t)(n0 + r) * a.vocab;
      head[f] = min((int)(-base & (V - 1)), a.vocab);
      nch[f] = (a.vocab - head[f]) / V;
      mi[f] = a.mask ? a.mask_idx[n0 + r] : -1;
      if (mi[f] >= a.n_masks) mi[f] = -1;
      if (chunk < nch[f]) {
        w[f] = *reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(a.logits) + (base + head[f] + (int64_t)V * chunk) * (16 / V));
        bits[f] = mi[f] >= 0 ? mask_bits(mi[f], head[f] + V * chunk) : ~0u;
      }
    }
#pragma unroll
    for (int f = 0; f < kInFlight; ++f) {
      if (rr + f >= r1) break;
      const int r = rr + f;
      const int64_t base = (int64_t)(n0 + r) * a.vocab;
      const int first = a.penalties ? s_hit[r] : -1;
      if (chunk < nch[f]) {
        const int l0 = head[f] + V * tid;          // first column in the segment
        const bool touched = s_any[tid] | (head[f] ? s_any[tid + 1] : 0);
        if (touched || first >= 0 || (bits[f] & ((1u << V) - 1)) != (1u << V) - 1) {
          int c[V];
          float x[V];
#pragma unroll
          for (int e = 0; e < V; ++e) c[e] = s_cnt[at(l0 + e)];
          for (int u = first; u >= 0; u = s_after[u])
#pragma unroll
            for (int e = 0; e < V; ++e) c[e] += s_loc[u] == l0 + e;
#pragma unroll
          for (int e = 0; e < V; ++e)
            x[e] = apply(Chunk<DT>::get(w[f], e), a.penalties ? c[e] : 0, __int_as_float(s_bias[at(l0 + e)]), (bits[f] >> e) & 1u);
          w[f] = Chunk<DT>::pack(x);
        }
        *reinterpret_cast<uint4 *>(static_cast<uint8_t *>(a.out) + (base + head[f] + (int64_t)V * chunk) * (16 / V)) = w[f];
      }
      // single values: those before the first chunk, those after the last
      int col = -1;
      if (blockIdx.x == 0 && tid < head[f]) col = tid;
      else if ((int)blockIdx.x == nch[f] / kNT) {
        const int t = tid - (blockIdx.x == 0 ? head[f] : 0);
        if (t >= 0 && head[f] + V * nch[f] + t < a.vocab) col = head[f] + V * nch[f] + t;
      }
      if (col >= 0) {
        const int l = col - col0;
        int c = s_cnt[at(l)];
        for (int u = first; u >= 0; u = s_after[u]) c += s_loc[u] == l;
        const float z = DT == 0 ? static_cast<const float *>(a.logits)[base + col]
                                : bf16_to_f32(static_cast<const uint16_t *>(a.logits)[base + col]);
        const float y = apply(z, a.penalties ? c : 0, __int_as_float(s_bias[at(l)]),
                              mi[f] < 0 || ((a.mask[(int64_t)mi[f] * a.mask_words + (col >> 5)] >> (col & 31)) & 1u));
        if (DT == 0) static_cast<float *>(a.out)[base + col] = y;
        else static_cast<uint16_t *>(a.out)[base + col] = (uint16_t)(pack_bf16x2(y, 0.f) & 0xFFFFu);
      }
    }
  }
}

// Counts of a sequence's tokens: one block per segment of the vocabulary, counted
// in LDS (integers: the order of the additions does not matter) and written out
// whole, so that the table needs no clearing.
constexpr int kCountThreads = 512;
constexpr int kCountSeg = 4096;

__global__ __launch_bounds__(kCountThreads) void token_counts_kernel(CountArgs a) {
  __shared__ int s[kCountSeg];
  const int b = blockIdx.y, col0 = blockIdx.x * kCountSeg, n = min(kCountSeg, a.vocab - col0);
  int *const out = a.counts + (int64_t)b * a.vocab + col0;
  for (int c = threadIdx.x; c < n; c += kCountThreads) s[c] = a.accumulate ? out[c] : 0;
  __syncthreads();
  const int t1 = min(a.tok_off[b + 1], a.total);
  constexpr int U = 8;
  for (int t = max(a.tok_off[b], 0) + threadIdx.x; t < t1; t += U * kCountThreads) {
    int v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = t + u * kCountThreads < t1 ? a.tokens[t + u * kCountThreads] : -1;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if ((unsigned)v[u] < (unsigned)a.vocab && (unsigned)(v[u] - col0) < (unsigned)n) atomicAdd(&s[v[u] - col0], 1);
  }
  __syncthreads();
  for (int c = threadIdx.x; c < n; c += kCountThreads) out[c] = s[c];
}

// The accepted path's tokens, one wave a sequence.
__global__ __launch_bounds__(64) void count_accepted_kernel(AcceptedArgs a) {
  const int b = blockIdx.x, lane = threadIdx.x;
  const int n0 = a.node_off[b], N = a.node_off[b + 1] - n0, len = a.accept_len[b];
  if (len < 0 || len >= N || len >= kMaxPath || len >= a.path_stride) return;
  const int *path = a.path + (int64_t)b * a.path_stride;
  const int u = lane <= len ? path[lane] : 0, before = lane > 0 && lane <= len ? path[lane - 1] : -1;
  if (__builtin_amdgcn_ballot_w64(lane <= len && (u <= before || u >= N))) return;   // not increasing, or past the tree
  if (lane > len) return;
  const int t = a.node_tok[n0 + u];
  if ((unsigned)t < (unsigned)a.vocab) atomicAdd(&a.counts[(int64_t)b * a.vocab + t], 1);
}

}  // namespace

hipError_t launch_logit_rules(int dt, const RulesArgs &args, int B, int max_nodes, hipStream_t st) {
  RulesArgs a = args;
  a.groups = (max_nodes + kRows - 1) / kRows;
  const int seg = kNT * (dt == 0 ? 4 : 8);
  const dim3 grid((a.vocab + seg - 1) / seg, B * a.groups);
  if (dt == 0) hipLaunchKernelGGL(logit_rules_kernel<0>, grid, dim3(kNT), 0, st, a);
  else hipLaunchKernelGGL(logit_rules_kernel<1>, grid, dim3(kNT), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_token_counts(const CountArgs &a, int B, hipStream_t st) {
  hipLaunchKernelGGL(token_counts_kernel, dim3((a.vocab + kCountSeg - 1) / kCountSeg, B), dim3(kCountThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_count_accepted(const AcceptedArgs &a, int B, hipStream_t st) {
  hipLaunchKernelGGL(count_accepted_kernel, dim3(B), dim3(64), 0, st, a);
  return hipGetLastError();
}

}  // namespace specmemo

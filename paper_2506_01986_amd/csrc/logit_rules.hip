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
static_assert(kNT >= kMaxNodes, "one thread per tree node");
constexpr int kRows = kRulesRows;   // most node rows of a block, all their loads in flight at once

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

// One block: up to kRows rows of a sequence, one segment of kNT chunks of the
// vocabulary.  The rows' loads go first; while they are on their way the segment's
// counts and biases are put into LDS, once for all the rows (element e of chunk i
// at e * kStride + i: any alignment of the rows reads them without bank conflicts).
template <int DT>
__global__ __launch_bounds__(kNT) void logit_rules_kernel(RulesArgs a) {
  constexpr int V = Chunk<DT>::V, SEG = kNT * V, COLS = SEG + V, kStride = kNT + 2;
  __shared__ int s_cnt[V * kStride];
  __shared__ int s_bias[V * kStride];              // index + 1 of the token's last bias entry
  __shared__ float s_val[V * kStride];             // its value
  __shared__ uint8_t s_any[kNT + 1];               // chunk-sized groups with a count or a bias
  __shared__ int s_par[kMaxNodes], s_loc[kMaxNodes], s_hit[kMaxNodes], s_after[kMaxNodes];
  const int tid = threadIdx.x;
  const int b = blockIdx.y / a.groups, r0 = blockIdx.y % a.groups * a.rows;
  const int n0 = a.node_off[b], N = a.node_off[b + 1] - n0;
  if (r0 >= N) return;
  const int nrow = min(a.rows, N - r0);
  // The tree's rows, those that begin at the same place of a chunk one after another
  // (every q-th, q = V / gcd(V, vocab)), rows r0 .. of that order: what a block keeps from
  // row to row holds for most of its rows (640 rows of 31999 bf16 values 31.3 us in tree
  // order, 24.7).
  int row[kRows];
  const int q = V / min(a.vocab & -a.vocab, V);
#pragma unroll
  for (int f = 0; f < kRows; ++f) row[f] = r0 + f;
  if (q > 1 && a.rows > 1) {
    const int size = N / q, big = N % q;   // `big` classes of size + 1, q - big of size
    const int past = r0 - big * (size + 1);
    int cls = past < 0 ? r0 / (size + 1) : big + past / max(size, 1);
    row[0] = cls + q * (past < 0 ? r0 % (size + 1) : past % max(size, 1));
#pragma unroll
    for (int f = 1; f < kRows; ++f) {
      const bool same = row[f - 1] + q < N;
      cls += !same;
      row[f] = same ? row[f - 1] + q : cls;
    }
  }
  const float rep = a.repetition ? a.repetition[b] : 1.f;
  // fp32 quotients are rounded once (640 rows of 32000: 34.0 us, 31.9 with the reciprocal,
  // whose products are off in the last place).  For bf16 x / rep is a product with the reciprocal
  // (2^-24 of a quotient more; the result's own rounding is 2^-8; dividing on the path alone
  // takes 640 rows of 32000 from 22.4 to 23.3 us).  Where fp32 does not hold the reciprocal
  // as a normal number it is that of rep times a power of two, and a counted token is
  // treated one by one, as those on the path.
  const float fit = rep < 0x1p-126f ? 0x1p64f : rep > 0x1p126f ? 0x1p-64f : 1.f, inv_rep = 1.f / (rep * fit);
  const bool single = DT == 1 && fit != 1.f;
  const float pres = a.presence ? a.presence[b] : 0.f, freq = a.frequency ? a.frequency[b] : 0.f;
  const int j0 = a.n_bias > 0 ? max(a.bias_off[b], 0) : 0, j1 = a.n_bias > 0 ? min(a.bias_off[b + 1], a.n_bias) : 0;
  const int col0 = blockIdx.x * SEG, chunk = blockIdx.x * kNT + tid;
  auto at = [&](int c) { return c % V * kStride + c / V; };   // column of the segment -> LDS
  auto row_at = [&](int f) { return (int64_t)(n0 + row[f]) * a.vocab; };
  auto row_head = [&](int f) { return min((int)(-row_at(f) & (V - 1)), a.vocab); };   // values before the first chunk
  auto row_mask = [&](int f) {
    const int m = a.mask ? a.mask_idx[n0 + row[f]] : -1;
    return m < a.n_masks ? m : -1;
  };

  // What the segment's tables are made of, before the rows: loads return in order,
  // and the tables are built while the rows are on their way.
  int cnt[V], cnt_last = 0;           // counts of chunk tid's columns; of column SEG + tid, past the last chunk
#pragma unroll
  for (int e = 0; e < V; ++e) cnt[e] = 0;
  if (a.counts) {
    const int *c = a.counts + (int64_t)b * a.vocab + col0;
    if (((uintptr_t)c & 15) == 0 && chunk * V + V <= a.vocab) {
#pragma unroll
      for (int e = 0; e < V; e += 4) *reinterpret_cast<int4 *>(cnt + e) = *reinterpret_cast<const int4 *>(c + V * tid + e);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (chunk * V + e < a.vocab) cnt[e] = c[V * tid + e];
    }
    if (tid < V && col0 + SEG + tid < a.vocab) cnt_last = c[SEG + tid];
  }
  int tok = -1, par = -1;
  if (a.penalties && tid < N) {
    tok = a.node_tok[n0 + tid];
    par = a.parent[n0 + tid];         // -1 at the root
  }
  // a bias entry's token as a column of the segment, or -1
  auto bias_col = [&](int j) {
    const int v = a.bias_id[j];
    return v >= 0 && v >= col0 && v - col0 < COLS ? v - col0 : -1;
  };
  const int my_col = j0 + tid < j1 ? bias_col(j0 + tid) : -1;   // the first entry of each thread, read with its value
  const float my_val = j0 + tid < j1 ? a.bias_val[j0 + tid] : 0.f;

  uint4 w[kRows];
  uint32_t bits[kRows];               // bit e: the chunk's column e is allowed
#pragma unroll
  for (int f = 0; f < kRows; ++f) {
    bits[f] = ~0u;
    if (f < nrow) {
      const int head = row_head(f), m = row_mask(f);
      if (chunk < (a.vocab - head) / V) {
        w[f] = *reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(a.logits) + (row_at(f) + head + (int64_t)V * chunk) * (16 / V));
        if (m >= 0) {
          const uint32_t *mw = a.mask + (int64_t)m * a.mask_words;
          const int col = head + V * chunk, i = col >> 5;
          bits[f] = (uint32_t)(((uint64_t)mw[min(i + 1, a.mask_words - 1)] << 32 | mw[i]) >> (col & 31));
        }
      }
    }
  }
  {
    int any = 0;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      any |= cnt[e];
      s_cnt[e * kStride + tid] = cnt[e];
      s_bias[e * kStride + tid] = 0;
      s_val[e * kStride + tid] = 0.f;
    }
    s_any[tid] = any != 0;
    const uint64_t last = __builtin_amdgcn_ballot_w64(tid < V && cnt_last != 0);
    if (tid < V) {
      s_cnt[tid * kStride + kNT] = cnt_last;
      s_bias[tid * kStride + kNT] = 0;
      s_val[tid * kStride + kNT] = 0.f;
    }
    if (tid == 0) s_any[kNT] = last != 0;
  }
  if (tid < N) {
    s_par[tid] = par;
    s_loc[tid] = tok >= col0 && tok < min(col0 + COLS, a.vocab) ? tok - col0 : -1;
  }
  __syncthreads();
  // Nearest node at or above n, and strictly above it, whose token lies in the segment.
  if (a.penalties && tid < N) {
    int u = par;
    while (u >= 0 && s_loc[u] < 0) u = s_par[u];
    s_after[tid] = u;
    s_hit[tid] = s_loc[tid] >= 0 ? tid : u;
  }
  if (j0 < j1) {                      // of equal ids the last entry counts
    if (my_col >= 0) atomicMax(&s_bias[at(my_col)], j0 + tid + 1);
    for (int j = j0 + kNT + tid; j < j1; j += kNT) {
      const int c = bias_col(j);
      if (c >= 0) atomicMax(&s_bias[at(c)], j + 1);
    }
    __syncthreads();
    const bool mine = my_col >= 0 && s_bias[at(my_col)] == j0 + tid + 1;
    for (int j = j0 + kNT + tid; j < j1; j += kNT) {
      const int c = bias_col(j);
      if (c >= 0 && s_bias[at(c)] == j + 1) {
        s_val[at(c)] = a.bias_val[j];
        s_any[c / V] = 1;
      }
    }
    if (mine) {
      s_val[at(my_col)] = my_val;
      s_any[my_col / V] = 1;
    }
  }
  __syncthreads();

  auto apply = [&](float x, int c, float bias, bool allowed) {
    const float y = fmaf(-freq, (float)c, (x > 0.f ? (DT == 0 ? x / rep : x * inv_rep * fit) : x * rep) - pres);
    x = c > 0 ? y : x;
    return allowed ? x + bias : -INFINITY;
  };
  // What the rules do to this thread's columns in a row whose path adds no count:
  // x times one of two factors, plus a term.  Kept from row to row while the rows
  // begin at the same place of a chunk (every row where vocab is a multiple of V):
  // four instructions a value instead of twenty, which bound the kernel (640 rows
  // of 32000 bf16 values 30.1 us before).
  float pos[V], neg[V], add[V];
  int kept = -1;
  bool touched = false;
#pragma unroll
  for (int f = 0; f < kRows; ++f) {
    if (f >= nrow) break;
    const int head = row_head(f), nch = (a.vocab - head) / V;
    const int first = a.penalties ? s_hit[row[f]] : -1;
    if (chunk < nch) {
      const int l0 = head + V * tid;             // first column in the segment
      float x[V];
      if (kept != head) {
        kept = head;
        touched = s_any[tid] | (head ? s_any[tid + 1] : 0);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const int c = s_cnt[at(l0 + e)];
          pos[e] = c > 0 ? inv_rep : 1.f;
          neg[e] = c > 0 ? rep : 1.f;
          add[e] = s_val[at(l0 + e)] - (c > 0 ? fmaf(freq, (float)c, pres) : 0.f);
        }
      }
      // tokens of this row's path among the thread's columns
      uint32_t onpath = single && touched ? (1u << V) - 1 : 0;
      for (int u = first; u >= 0; u = s_after[u]) onpath |= (unsigned)(s_loc[u] - l0) < V ? 1u << (s_loc[u] - l0) : 0u;
      const bool masked = (bits[f] & ((1u << V) - 1)) != (1u << V) - 1;
      if (touched || masked || onpath) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float z = Chunk<DT>::get(w[f], e);
          x[e] = DT == 0 ? (z > 0.f ? z / neg[e] : z * neg[e]) + add[e] : fmaf(z, z > 0.f ? pos[e] : neg[e], add[e]);
        }
        if (onpath) {
#pragma unroll
          for (int e = 0; e < V; ++e)
            if ((onpath >> e) & 1u) {
              int c = s_cnt[at(l0 + e)];
              for (int u = first; u >= 0; u = s_after[u]) c += s_loc[u] == l0 + e;
              x[e] = apply(Chunk<DT>::get(w[f], e), c, s_val[at(l0 + e)], true);
            }
        }
        if (masked) {
#pragma unroll
          for (int e = 0; e < V; ++e) x[e] = (bits[f] >> e) & 1u ? x[e] : -INFINITY;
        }
        w[f] = Chunk<DT>::pack(x);
      }
      *reinterpret_cast<uint4 *>(static_cast<uint8_t *>(a.out) + (row_at(f) + head + (int64_t)V * chunk) * (16 / V)) = w[f];
    }
    // single values: those before the first chunk, those after the last
    int col = -1;
    if (blockIdx.x == 0 && tid < head) col = tid;
    else if ((int)blockIdx.x == nch / kNT) {
      const int t = tid - (blockIdx.x == 0 ? head : 0);
      if (t >= 0 && head + V * nch + t < a.vocab) col = head + V * nch + t;
    }
    if (col >= 0) {
      const int l = col - col0, m = row_mask(f);
      int c = s_cnt[at(l)];
      for (int u = first; u >= 0; u = s_after[u]) c += s_loc[u] == l;
      const float z = DT == 0 ? static_cast<const float *>(a.logits)[row_at(f) + col]
                              : bf16_to_f32(static_cast<const uint16_t *>(a.logits)[row_at(f) + col]);
      const float y = apply(z, c, s_val[at(l)],
                            m < 0 || ((a.mask[(int64_t)m * a.mask_words + (col >> 5)] >> (col & 31)) & 1u));
      if (DT == 0) static_cast<float *>(a.out)[row_at(f) + col] = y;
      else static_cast<uint16_t *>(a.out)[row_at(f) + col] = (uint16_t)(pack_bf16x2(y, 0.f) & 0xFFFFu);
    }
  }
}

// Counts of a sequence's tokens: one block per segment of the vocabulary, counted
// in LDS (integers: the order of the additions does not matter) and written out
// whole, so that the table needs no clearing.
constexpr int kCountThreads = 1024;
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

hipError_t launch_logit_rules(int dt, const RulesArgs &args, int B, int total, int max_nodes, hipStream_t st) {
  RulesArgs a = args;
  const int seg = kNT * (dt == 0 ? 4 : 8), segs = (a.vocab + seg - 1) / seg;
  a.rows = rules_rows(segs, B, total, max_nodes, device_cus());
  a.groups = (max_nodes + a.rows - 1) / a.rows;
  const dim3 grid(segs, B * a.groups);
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

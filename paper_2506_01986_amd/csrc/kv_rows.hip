// New rows of the pool: norm, position rotation and append of q, k and v in one pass,
// into a pool of the inputs' type or of 4 bits (kv4.h), and the 4-bit pool's own row
// moves (compaction, reading back).
//
// SpecMemo Sec. 3.1: a step's tokens (a prompt's, or a tree's nodes) bring their K/V
// rows to the preallocated cache before the attention reads them.  For a head's row x
// at position p, with norm weights w and rotated columns (a, b) at angle t:
//   y = x / sqrt(mean(x^2) + eps) w,   y_a cos t - y_b sin t,   y_b cos t + y_a sin t
// for q and k; v is stored as it is.  Everything is one read of the inputs and one
// write of the outputs: the kernels are bound by memory, or where there are few rows
// by one launch's latency.  1024 tokens of 32 + 32 + 32 heads (50 MB) 8.2 us on one set of
// buffers, 10.0 on sets that change; 19k of 64 + 8 + 8 (722 MB, into 4 bits) 143 us: 5.0
// TB/s; one tree 3.1 to 4.2 us.  Reading the 4-bit rows of those 19k back (99 MB): 19 us,
// 29 right behind the append that wrote them.  Compaction, three dependent loads and a
// store: 4.6 to 5.2 us whatever the batch.
#include <algorithm>
#include <type_traits>

#include "device.h"
#include "internal.h"
#include "kv4.h"

namespace specmemo {

namespace {

constexpr int kThreads = 256;

// The sequence that holds token `tok`: the last one with off <= tok.  The wave's first
// token is searched 64 ways a round, by all lanes of the wave (no call from a branch that
// only some of them take); the other lanes' lie a few sequences on.
__device__ __forceinline__ int find_seq(const RowsSeq *seq, int nseq, int tok) {
  const int lane = threadIdx.x & 63, first = __builtin_amdgcn_readfirstlane(tok);
  int lo = 0, cnt = nseq;
  while (cnt > 1) {
    const int st = (cnt + 63) >> 6, at = lane * st;
    const int off = at < cnt ? seq[lo + at].off : 0;
    const int p = __builtin_popcountll(__builtin_amdgcn_ballot_w64(at < cnt && off <= first)) - 1;
    lo += p * st;
    cnt = min(st, cnt - p * st);
  }
  while (lo + 1 < nseq && seq[lo + 1].off <= tok) ++lo;
  return lo;
}
__device__ __forceinline__ int64_t pool_row(const RowsSeq *seq, int nseq, int tok) {
  const RowsSeq s = seq[find_seq(seq, nseq, tok)];
  return (int64_t)((uint64_t)(uint32_t)s.row0_hi << 32 | (uint32_t)s.row0_lo) + tok;
}

// The 16 bytes of a row that a lane has, as E numbers.
template <int E>
__device__ __forceinline__ void unpack(float (&x)[E], uint4 w) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < E; ++i) x[i] = E == 8 ? bf16_to_f32((uint16_t)(u[i >> 1] >> (16 * (i & 1)))) : __uint_as_float(u[i & 3]);
}

// fp64 -> fp32, cut to 20 bits of fraction and the last of them set where any are lost:
// comparisons with numbers of fewer bits (the borders between codes) come out as they
// would in 64 bits.  (Numbers between fp32's largest and 2^128 come out below it.)
__device__ __forceinline__ float sticky_f32(double d) {
  const uint64_t u = __double_as_longlong(d);
  return (float)__longlong_as_double((long long)((uint64_t)((uint32_t)(u >> 32) | min((uint32_t)u, 1u)) << 32));
}

// Sum over the lph lanes of a head, in each of them: a row of 16 lanes by DPP, as in
// wave_max.
__device__ __forceinline__ float head_sum(float v, int lph) {
  if (lph == 16) {
    v += dpp_f<0xB1>(v);
    v += dpp_f<0x4E>(v);
    v += dpp_f<0x141>(v);
    return v + dpp_f<0x140>(v);
  }
  for (int m = 1; m < lph; m <<= 1) v += __shfl_xor(v, m);
  return v;
}
template <int CTRL>
__device__ __forceinline__ double dpp_d(double v) {
  const uint64_t u = __double_as_longlong(v);
  return __longlong_as_double((long long)((uint64_t)(uint32_t)dpp_i<CTRL>((int)(u >> 32)) << 32 | (uint32_t)dpp_i<CTRL>((int)u)));
}
__device__ __forceinline__ double head_sum(double v, int lph) {
  if (lph == 16) {
    v += dpp_d<0xB1>(v);
    v += dpp_d<0x4E>(v);
    v += dpp_d<0x141>(v);
    return v + dpp_d<0x140>(v);
  }
  for (int m = 1; m < lph; m <<= 1) v += __shfl_xor(v, m);
  return v;
}

// 1 / sqrt(x): the instruction's result (one unit off at most), in 64 bits improved
// from half the digits by two steps of y (3 - x y^2) / 2 (of infinity it is 0, which the
// steps would make a NaN: a row with one has zeros beside it).
__device__ __forceinline__ float inv_sqrt(float x) { return __builtin_amdgcn_rsqf(x); }
__device__ __forceinline__ double inv_sqrt(double x) {
  double y = __builtin_amdgcn_rsq(x);
#pragma unroll
  for (int i = 0; i < 2; ++i) y = fma(0.5 * y, fma(-x * y, y, 1.0), y);
  return x == INFINITY ? 0.0 : y;
}

// How a lane's E columns of a head turn: out = x fx + y fy with y the columns that x's
// turn with, of another lane of the head or its own pairs; fx and fy are cos and sin,
// times the columns' norm weights in fp32.
template <int E>
struct Lane {
  static constexpr int ES = 16 / E;
  int c, c2, from;          // first column of the lane's and of those they turn with; the lane that has them
  bool pairs, turns, live;  // live: the token has a position, and the lane columns
  int p, half;

  __device__ __forceinline__ Lane(const AppendArgs &a, int lph, int tok, bool on) {
    half = a.rot_dim >> 1;
    c = (threadIdx.x & (lph - 1)) * E;
    turns = c < a.rot_dim;
    pairs = a.pairs;
    const bool low = c < half, own = !turns || pairs;
    from = (threadIdx.x & 63) + (own ? 0 : low ? half / E : -(half / E));
    c2 = own ? c : low ? c + half : c - half;
    p = a.pos ? a.pos[tok] : 0;
    live = on && c < a.head_dim && (!a.pos || (uint32_t)p < (uint32_t)a.n_pos);   // no such position: the rows are left as they were
    turns = turns && live;
  }
  __device__ __forceinline__ void angles(const AppendArgs &a, float (&co)[E], float (&si)[E]) const {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      co[i] = 1.f;
      si[i] = 0.f;
    }
    if (!turns) return;
    const float *cs = a.cos + (int64_t)p * half, *sn = a.sin + (int64_t)p * half;
    if (pairs) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        co[i] = cs[(c >> 1) + (i >> 1)];
        si[i] = i & 1 ? sn[(c >> 1) + (i >> 1)] : -sn[(c >> 1) + (i >> 1)];
      }
    } else {
      const bool low = c < half;
      const int at = low ? c : c2;
#pragma unroll
      for (int i = 0; i < E; i += 4) {
        const f32x4 x = *reinterpret_cast<const f32x4 *>(cs + at + i), y = *reinterpret_cast<const f32x4 *>(sn + at + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          co[i + e] = x[e];
          si[i + e] = low ? -y[e] : y[e];
        }
      }
    }
  }
  // The columns that the lane's turn with, in its own columns' order; x: the lane's own, w: as loaded.
  __device__ __forceinline__ void other(float (&y)[E], const float (&x)[E], uint4 w, int lph) const {
    if (pairs) {
#pragma unroll
      for (int i = 0; i < E; ++i) y[i] = x[i ^ 1];
    } else if (lph == 16 && half == 8 * E) {       // of the lane eight on in its row of 16
#pragma unroll
      for (int i = 0; i < E; ++i) y[i] = dpp_f<0x128>(x[i]);
    } else {
      unpack(y, uint4{(uint32_t)__shfl((int)w.x, from), (uint32_t)__shfl((int)w.y, from), (uint32_t)__shfl((int)w.z, from),
                      (uint32_t)__shfl((int)w.w, from)});
    }
  }
  __device__ __forceinline__ void weights(float (&own)[E], float (&far)[E], const void *norm, int d) const {
    const uint4 x = ld16_or_zero(c < d, static_cast<const char *>(norm) + c * ES), y = ld16_or_zero(c < d, static_cast<const char *>(norm) + c2 * ES);
    unpack(own, x);
    unpack(far, y);
    if (pairs) {
#pragma unroll
      for (int i = 0; i < E; i += 2) {
        const float z = far[i];
        far[i] = far[i + 1];
        far[i + 1] = z;
      }
    }
  }
};

// The row's 1 / sqrt(mean of squares + eps); inv_d = 1 / d.
template <typename T, int E>
__device__ __forceinline__ T row_norm(const float (&x)[E], float eps, T inv_d, int lph) {
  T s = 0;
#pragma unroll
  for (int i = 0; i < E; ++i) s += T(x[i]) * T(x[i]);
  return inv_sqrt(fma(head_sum(s, lph), inv_d, T(eps)));
}

// 16 bytes past the caches' own rules: what reads them next runs on all XCDs, behind
// other L2s, and the end of the kernel has nothing to write back (1024 rows of 32 + 32 +
// 32 heads 12.0 us as ordinary stores, 8.2).
__device__ __forceinline__ void store16(void *p, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  __builtin_nontemporal_store(u32x4{x, y, z, w}, static_cast<u32x4 *>(p));
}
template <int E>
__device__ __forceinline__ void store_row(void *p, const float (&x)[E]) {
  if constexpr (E == 8) store16(p, pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
  else store16(p, __float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}

// Columns c .. of a row in 4 bits; the lanes of a group (32 / E of them) find its scale together.
template <int E>
__device__ __forceinline__ void store_row4(uint8_t *codes, uint8_t *scales, int c, const float (&y)[E], bool on) {
  float top = 0.f;
  bool odd = false;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    top = fmaxf(top, fabsf(y[i]));
    odd |= !(fabsf(y[i]) < INFINITY);
  }
  top = odd ? INFINITY : top;
  top = fmaxf(top, dpp_f<0xB1>(top));
  top = fmaxf(top, dpp_f<0x4E>(top));
  if (E == 4) top = fmaxf(top, dpp_f<0x141>(top));
  if (!on) return;
  const uint32_t byte = kv4_scale_byte(top);
  const float unit = kv4_scale(byte);
  uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, y[0], y[1], unit, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], unit, 1);
  if constexpr (E == 8) {
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], unit, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], unit, 3);
    *reinterpret_cast<uint32_t *>(codes + c / 2) = w;
  } else {
    *reinterpret_cast<uint16_t *>(codes + c / 2) = (uint16_t)w;
  }
  if (c % kKv4Group == 0) scales[c / kKv4Group] = (uint8_t)byte;
}

// lph lanes have a head's row, and a block 256 / lph of them (slots).  A block has heads
// of one kind (keys, queries, values), and its slots those of one token, or of several
// where a token has few: 1 << log2 slots each, HB heads a slot with their loads together,
// so that a lane loads cos, sin and the norm's weights, and brings them to fp64, once.
// Keys that go to 4 bits are normed and turned in fp64, so that a value next to a border
// between two codes falls on its own side of it (a sum of d squares and its root are off
// by some 11 roundings, the turn and the products by 4: 2^-49 of the terms, which is as
// near as a value may come); they take longest and begin first.
// 19k tokens of 64 + 8 + 8 heads into 4 bits: 179 us with one key or value head a slot,
// 144 so; 8k of 32 + 32 + 32: 137, 84.  (fp32 with a bound on its error, and fp64 for the
// rows of which a column's interval holds a border: 174 and 117, and 1024 tokens 17 us
// against 11: the second way's registers and latency.)
template <bool BF16, bool FOUR, int HB>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a) {
  constexpr int E = BF16 ? 8 : 4, ES = BF16 ? 2 : 4;
  const int kind = (blockIdx.x >= a.kind[1].block0) + (blockIdx.x >= a.kind[2].block0);
  const AppendKind K = a.kind[kind];
  const int lph = 1 << a.lph_log2, d = a.head_dim, all = kThreads >> a.lph_log2, slot = threadIdx.x >> a.lph_log2;
  const int c = (threadIdx.x & (lph - 1)) * E, slots = 1 << K.log2;
  const uint32_t bid = blockIdx.x - K.block0, group = bid / (uint32_t)K.turns;
  const RowsToken at = rows_token(a.tok0, a.tok1, (int)group * (all >> K.log2) + (slot >> K.log2));
  const int tok = at.tok;
  const int h0 = (slot & (slots - 1)) + (int)(bid - group * K.turns) * HB * slots;
  const bool on = at.on, has = on && c < d;
  const char *const src = static_cast<const char *>(K.in) + (K.stride * tok + (int64_t)h0 * d + c) * ES;
  const int step = slots * d * ES;
  uint4 row[HB];
#pragma unroll
  for (int n = 0; n < HB; ++n) row[n] = ld16_or_zero(has && h0 + n * slots < K.heads, src + (int64_t)n * step);
  const Lane<E> l(a, lph, tok, on);
  const int64_t row0 = kind == kQueries ? (int64_t)tok * a.n_q + h0 : h0 * a.cap_total + pool_row(a.seq, a.nseq, tok);
  const int64_t row_step = kind == kQueries ? slots : a.cap_total * slots;
  if (!FOUR || kind == kQueries) {
    char *const dst = static_cast<char *>(K.out) + (row0 * d + c) * ES;
    const int64_t out_step = row_step * d * ES;
    if (kind == kValues) {
#pragma unroll
      for (int n = 0; n < HB; ++n)
        if (l.live && h0 + n * slots < K.heads) store16(dst + n * out_step, row[n].x, row[n].y, row[n].z, row[n].w);
      return;
    }
    float fx[E], fy[E];
    l.angles(a, fx, fy);
    if (K.norm) {
      float wx[E], wy[E];
      l.weights(wx, wy, K.norm, d);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        fx[i] *= wx[i];
        fy[i] *= wy[i];
      }
    }
#pragma unroll
    for (int n = 0; n < HB; ++n) {
      if (h0 + n * slots >= K.heads) break;
      float x[E], y[E];
      unpack(x, row[n]);
      l.other(y, x, row[n], lph);
      const float r = K.norm ? row_norm(x, a.eps, a.inv_d, lph) : 1.f;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        x[i] *= fx[i];
        if (l.turns) x[i] = fmaf(y[i], fy[i], x[i]);
        if (K.norm) x[i] *= r;
      }
      if (l.live) store_row(dst + n * out_step, x);
    }
    return;
  }
  uint8_t *const codes = static_cast<uint8_t *>(K.out) + row0 * (d / 2);
  uint8_t *const scales = (kind == kKeys ? a.ks : a.vs) + row0 * (d / kKv4Group);
  const int64_t code_step = row_step * (d / 2), scale_step = row_step * (d / kKv4Group);
  if (kind == kValues) {
#pragma unroll
    for (int n = 0; n < HB; ++n) {
      if (h0 + n * slots >= K.heads) break;
      float x[E];
      unpack(x, row[n]);
      store_row4(codes + n * code_step, scales + n * scale_step, c, x, l.live);
    }
    return;
  }
  double fx[E], fy[E];                // products of two fp32 numbers: exact
  {
    float co[E], si[E], wx[E], wy[E];
    l.angles(a, co, si);
    if (K.norm) l.weights(wx, wy, K.norm, d);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      fx[i] = co[i];
      fy[i] = si[i];
      if (K.norm) {
        fx[i] *= wx[i];
        fy[i] *= wy[i];
      }
    }
  }
#pragma unroll
  for (int n = 0; n < HB; ++n) {
    if (h0 + n * slots >= K.heads) break;
    float x[E], y[E];
    unpack(x, row[n]);
    l.other(y, x, row[n], lph);
    const double r = K.norm ? row_norm(x, a.eps, 1.0 / d, lph) : 1.0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      double v = x[i] * fx[i];
      if (l.turns) v = fma((double)y[i], fy[i], v);
      if (K.norm) v *= r;
      x[i] = sticky_f32(v);
    }
    store_row4(codes + n * code_step, scales + n * scale_step, c, x, l.live);
  }
}

// Rows of a 4-bit pool as values: a thread has eight columns of one head of K or V and
// takes them for TB tokens, one after another.  A token's chunks take `blocks` blocks, or
// 1 << log2 threads of one that has several tokens' worth.
template <bool BF16, int TB>
__global__ __launch_bounds__(kThreads) void kv4_read_kernel(ReadArgs a, int blocks, int log2) {
  const int cw = a.head_dim >> 3, d = a.head_dim;           // chunks of a row
  const int per = 2 * a.n_kv * cw;                          // and of a token
  const int in = (int)(blockIdx.x % blocks) * kThreads + (threadIdx.x & ((1 << log2) - 1));
  const int tok0 = ((int)(blockIdx.x / blocks) * (kThreads >> log2) + (threadIdx.x >> log2)) * TB;   // of the launch's
  const int x = min(in, per - 1), c = x % cw, head = x / cw;
  const bool v = head >= a.n_kv;
  const int hk = v ? head - a.n_kv : head;
  const uint8_t *const codes = (v ? a.v : a.k), *const scales = v ? a.vs : a.ks;
  int s = find_seq(a.seq, a.nseq, rows_token(a.tok0, a.tok1, tok0).tok);
  uint32_t w[TB], byte[TB];
#pragma unroll
  for (int n = 0; n < TB; ++n) {
    const int tok = rows_token(a.tok0, a.tok1, tok0 + n).tok;
    while (s + 1 < a.nseq && a.seq[s + 1].off <= tok) ++s;
    const int64_t r = (int64_t)hk * a.cap_total + (int64_t)((uint64_t)(uint32_t)a.seq[s].row0_hi << 32 | (uint32_t)a.seq[s].row0_lo) + tok;
    w[n] = *reinterpret_cast<const uint32_t *>(codes + r * (d >> 1) + 4 * c);
    byte[n] = scales[r * (d / kKv4Group) + (c >> 2)];
  }
  if (in >= per) return;
#pragma unroll
  for (int n = 0; n < TB; ++n) {
    const RowsToken t = rows_token(a.tok0, a.tok1, tok0 + n);
    if (!t.on) return;
    const bool nan = byte[n] == kKv4Nan;
    const float unit = kv4_scale(byte[n]);
    const int64_t o = ((int64_t)t.tok * a.n_kv + hk) * d + 8 * c;
    void *const out = v ? a.v_out : a.k_out;
    if constexpr (BF16) {
      const uint4 y = kv4_bf16x8(w[n], unit);
      constexpr uint32_t q = 0x7FC07FC0u;
      store16(static_cast<uint16_t *>(out) + o, nan ? q : y.x, nan ? q : y.y, nan ? q : y.z, nan ? q : y.w);
    } else {
      const f32x2_t p[4] = {kv4_f32x2<0>(w[n], unit), kv4_f32x2<1>(w[n], unit), kv4_f32x2<2>(w[n], unit), kv4_f32x2<3>(w[n], unit)};
      float y[2][4];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i >> 2][i & 3] = nan ? __uint_as_float(0x7FC00000u) : p[i >> 1][i & 1];
      store_row(static_cast<float *>(out) + o, y[0]);
      store_row(static_cast<float *>(out) + o + 4, y[1]);
    }
  }
}

// Compaction of a 4-bit pool: rows L + path[j] -> L + j of codes and scales.  One wave
// per (sequence, KV head); a lane owns one word of the codes or one scale byte of K or
// V and reads it of every source row before it writes any, so no two lanes touch the
// same bytes and overlapping rows need no barrier.
__global__ __launch_bounds__(64) void kv4_compact_kernel(Compact4Args a) {
  const int s = blockIdx.x, kvh = blockIdx.y, b = a.b0 + s, lane = threadIdx.x;
  const Compact4Seq S = a.seq[s];
  const int acc = a.accept_len[b];
  const int np = min(kMaxPath, a.path_stride);
  int src[kMaxPath];
#pragma unroll
  for (int j = 0; j < kMaxPath; ++j) src[j] = j < np ? a.path[(int64_t)b * a.path_stride + j] : -1;
  bool ok = acc >= 0 && acc < np && acc < S.N && src[0] == 0;
#pragma unroll
  for (int j = 1; j < kMaxPath; ++j)
    if (j <= acc) ok = ok && src[j] < S.N && src[j] > src[j - 1];
  if (!ok) return;                       // an invalid path leaves the sequence untouched
  const int words = a.head_dim / 8, groups = a.head_dim / kKv4Group;
  const int64_t row = (int64_t)kvh * a.cap_total + S.base + S.L;
  if (lane < 2 * words) {
    const int w = lane % words;
    uint32_t *p = reinterpret_cast<uint32_t *>(lane < words ? a.k : a.v) + row * words + w;
    uint32_t tmp[kMaxPath];
#pragma unroll
    for (int j = 0; j < kMaxPath; ++j)
      if (j <= acc) tmp[j] = p[(int64_t)src[j] * words];
#pragma unroll
    for (int j = 0; j < kMaxPath; ++j)
      if (j <= acc) p[(int64_t)j * words] = tmp[j];
  } else if (lane < 2 * words + 2 * groups) {
    const int w = lane - 2 * words;
    uint8_t *p = (w < groups ? a.ks : a.vs) + row * groups + w % groups;
    uint8_t tmp[kMaxPath];
#pragma unroll
    for (int j = 0; j < kMaxPath; ++j)
      if (j <= acc) tmp[j] = p[(int64_t)src[j] * groups];
#pragma unroll
    for (int j = 0; j < kMaxPath; ++j)
      if (j <= acc) p[(int64_t)j * groups] = tmp[j];
  }
  if (kvh == 0 && lane == 0) a.seq_len[b] = S.L + acc + 1;
}

}  // namespace

namespace {

template <bool BF16, bool FOUR>
void append(AppendArgs &a, int cus, hipStream_t st) {
  a.lph_log2 = 0;
  while ((BF16 ? 8 : 4) << a.lph_log2 < a.head_dim) ++a.lph_log2;
  a.inv_d = 1.f / (float)a.head_dim;
  const int all = kThreads >> a.lph_log2, toks = a.tok1 - a.tok0;
  // heads a slot: as many as there are, and as leave every compute unit two blocks (256
  // tokens of 32 + 32 + 32 heads into 4 bits: 5.4 us with two a slot, 6.6 with one or
  // four; 1024 of 64 + 8 + 8: 11.2 with four, 12.8 with two)
  const int64_t blocks = (int64_t)toks * (a.kind[kQueries].heads + a.kind[kKeys].heads + a.kind[kValues].heads) / all;
  const int most = std::max(a.kind[kQueries].heads, a.kind[kKeys].heads);
  const int hb = most >= 4 && blocks >= 4 * 2 * cus ? 4 : most >= 2 && blocks >= 2 * 2 * cus ? 2 : 1;
  uint32_t block = 0;
  for (int i = 0; i < 3; ++i) {
    AppendKind &k = a.kind[i];
    k.log2 = 0;
    while (hb << k.log2 < k.heads && 1 << k.log2 < all) ++k.log2;
    const int per = hb << k.log2;
    k.turns = std::max(1, (k.heads + per - 1) / per);
    k.block0 = block;
    if (k.heads > 0) block += (uint32_t)((toks + (all >> k.log2) - 1) / (all >> k.log2)) * k.turns;
  }
  const dim3 grid(block), threads(kThreads);
  if (hb == 4) hipLaunchKernelGGL((append_kernel<BF16, FOUR, 4>), grid, threads, 0, st, a);
  else if (hb == 2) hipLaunchKernelGGL((append_kernel<BF16, FOUR, 2>), grid, threads, 0, st, a);
  else hipLaunchKernelGGL((append_kernel<BF16, FOUR, 1>), grid, threads, 0, st, a);
}

}  // namespace

hipError_t launch_append(int dt, bool four, AppendArgs &a, int cus, hipStream_t st) {
  if (dt == 0) four ? append<false, true>(a, cus, st) : append<false, false>(a, cus, st);
  else four ? append<true, true>(a, cus, st) : append<true, false>(a, cus, st);
  return hipGetLastError();
}

hipError_t launch_kv4_read(int dt, const ReadArgs &a, int cus, hipStream_t st) {
  const int per = 2 * a.n_kv * (a.head_dim / 8), blocks = (per + kThreads - 1) / kThreads, toks = a.tok1 - a.tok0;
  int log2 = 8;
  while (log2 > 0 && 1 << (log2 - 1) >= per) --log2;
  const int tpb = kThreads >> log2;                         // tokens at once of a block
  // four tokens a thread where that leaves every compute unit eight blocks
  const int tb = (int64_t)blocks * toks >= (int64_t)4 * 8 * cus * tpb ? 4 : 1;
  const dim3 grid((uint32_t)blocks * ((toks + tb * tpb - 1) / (tb * tpb))), block(kThreads);
  if (dt == 0) {
    if (tb == 4) hipLaunchKernelGGL((kv4_read_kernel<false, 4>), grid, block, 0, st, a, blocks, log2);
    else hipLaunchKernelGGL((kv4_read_kernel<false, 1>), grid, block, 0, st, a, blocks, log2);
  } else {
    if (tb == 4) hipLaunchKernelGGL((kv4_read_kernel<true, 4>), grid, block, 0, st, a, blocks, log2);
    else hipLaunchKernelGGL((kv4_read_kernel<true, 1>), grid, block, 0, st, a, blocks, log2);
  }
  return hipGetLastError();
}

hipError_t launch_kv4_compact(const Compact4Args &a, hipStream_t st) {
  hipLaunchKernelGGL(kv4_compact_kernel, dim3(a.nseq, a.n_kv), dim3(64), 0, st, a);
  return hipGetLastError();
}

}  // namespace specmemo

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
// by one launch's latency.
#include "device.h"
#include "internal.h"
#include "kv4.h"

namespace specmemo {

namespace {

constexpr int kThreads = 256;

// The sequence that holds token `tok`: the last one with off <= tok.  The wave's first
// token is searched 64 ways a round; the other lanes' lie a few sequences on.
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

template <typename T, int E>
__device__ __forceinline__ void load_cols(T (&x)[E], const void *p, bool bf16) {
  if (bf16) {
    const uint4 w = *static_cast<const uint4 *>(p);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = bf16_to_f32((uint16_t)(u[i >> 1] >> (16 * (i & 1))));
  } else {
    const f32x4 w = *static_cast<const f32x4 *>(p);
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = w[i & 3];
  }
}

// fp64 -> fp32 with the last bit set where bits are lost: comparisons with numbers of
// fewer bits (the borders between codes) come out as they would in 64 bits.
__device__ __forceinline__ float sticky_f32(double d) {
  const uint64_t u = __double_as_longlong(d);
  const uint64_t cut = u & ~0x1FFFFFFFull;
  return (float)__longlong_as_double((long long)(cut | (u != cut ? 0x20000000ull : 0ull)));
}
__device__ __forceinline__ float sticky_f32(float f) { return f; }

// One row chunk of E columns a lane (16 bytes of the inputs), LPH lanes to a head.  T
// is the type of the arithmetic: 32 bits, and 64 for keys that go to 4 bits, where a
// value next to a border between two codes must fall on its own side of it.
template <typename T, int E, bool BF16>
struct Chunk {
  T x[E];

  __device__ __forceinline__ void norm(const void *w, int d, int lph, float eps, bool on) {
    T s = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) s += on ? x[i] * x[i] : T(0);
    for (int m = 1; m < lph; m <<= 1) s += __shfl_xor(s, m);
    const T r = T(1) / sqrt(s / T(d) + T(eps));
    T g[E];
    if (on) load_cols(g, w, BF16);
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = on ? x[i] * r * g[i] : T(0);
  }

  // Columns c .. c + E - 1 of a head of which `rot` are rotated; halves: column c < rot / 2
  // turns with c + rot / 2, which another lane of the head holds; pairs: 2 i with 2 i + 1.
  __device__ __forceinline__ void rotate(const float *cs, const float *sn, int c, int rot, bool pairs) {
    if (pairs) {
      if (c >= rot) return;
#pragma unroll
      for (int i = 0; i < E; i += 2) {
        const T co = cs[(c + i) >> 1], si = sn[(c + i) >> 1], a = x[i], b = x[i + 1];
        x[i] = a * co - b * si;
        x[i + 1] = b * co + a * si;
      }
      return;
    }
    const int half = rot >> 1;
    const bool low = c < half;
    const int other = (threadIdx.x & 63) + (c >= rot ? 0 : low ? half / E : -(half / E));
    T y[E];
#pragma unroll
    for (int i = 0; i < E; ++i) y[i] = __shfl(x[i], other);
    if (c >= rot) return;
    const int at = low ? c : c - half;
#pragma unroll
    for (int i = 0; i < E; i += 4) {
      const f32x4 co = *reinterpret_cast<const f32x4 *>(cs + at + i), si = *reinterpret_cast<const f32x4 *>(sn + at + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[i + e] = low ? x[i + e] * T(co[e]) - y[i + e] * T(si[e]) : x[i + e] * T(co[e]) + y[i + e] * T(si[e]);
    }
  }

  __device__ __forceinline__ void store(void *p) const {
    if constexpr (BF16) {
      uint32_t u[E / 2];
#pragma unroll
      for (int i = 0; i < E; i += 2) u[i / 2] = pack_bf16x2((float)x[i], (float)x[i + 1]);
      *static_cast<uint4 *>(p) = uint4{u[0], u[1], u[2], u[3]};
    } else {
      *static_cast<f32x4 *>(p) = f32x4{(float)x[0], (float)x[1], (float)x[2], (float)x[3]};
    }
  }

  // Columns c .. of a row in 4 bits; the lanes of a group (32 / E of them) find its scale together.
  __device__ __forceinline__ void store4(uint8_t *codes, uint8_t *scales, int c, bool on) const {
    float y[E], top = 0.f;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      y[i] = sticky_f32(x[i]);
      top = fmaxf(top, fabsf(y[i]));
      odd |= !(fabsf(y[i]) < INFINITY);
    }
    top = odd ? INFINITY : top;
#pragma unroll
    for (int m = 1; m < kKv4Group / E; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
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
};

// LPH lanes have a head's row; a wave's rows follow one another, token by token: the
// token's query heads, then its key heads, then its value heads.
template <bool BF16, bool FOUR>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a, int lph_log2) {
  constexpr int E = BF16 ? 8 : 4, ES = BF16 ? 2 : 4;
  using TK = typename std::conditional<FOUR, double, float>::type;
  const int lph = 1 << lph_log2, heads = a.n_q + 2 * a.n_kv, d = a.head_dim;
  const int64_t unit = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> lph_log2;
  const int64_t units = (int64_t)(a.tok1 - a.tok0) * heads;
  const int c = (threadIdx.x & (lph - 1)) * E;
  const bool on = unit < units && c < d;
  const int64_t u = unit < units ? unit : units - 1;
  const int tok = a.tok0 + (int)(u / heads), head = (int)(u % heads);
  const int kind = head < a.n_q ? 0 : head < a.n_q + a.n_kv ? 1 : 2;
  const int hk = kind == 0 ? head : kind == 1 ? head - a.n_q : head - a.n_q - a.n_kv;
  const char *src = static_cast<const char *>(kind == 0 ? a.q : kind == 1 ? a.k : a.v) +
                    ((kind == 0 ? a.q_stride : kind == 1 ? a.k_stride : a.v_stride) * tok + (int64_t)hk * d + c) * ES;
  float x[E];
#pragma unroll
  for (int i = 0; i < E; ++i) x[i] = 0.f;
  if (on) load_cols(x, src, BF16);
  const int p = a.pos ? a.pos[tok] : 0;
  const bool live = on && (!a.pos || (uint32_t)p < (uint32_t)a.n_pos);   // no such position: the row is left as it was
  const int64_t row = pool_row(a.seq, a.nseq, tok);
  const int64_t at = (int64_t)hk * a.cap_total + row;
  const int pc = a.pos ? min(max(p, 0), a.n_pos - 1) : 0;
  const float *cs = a.cos + (int64_t)pc * (a.rot_dim >> 1), *sn = a.sin + (int64_t)pc * (a.rot_dim >> 1);
  auto turn = [&](auto &y, const void *w) __attribute__((always_inline)) {
    if (w) y.norm(static_cast<const char *>(w) + c * ES, d, lph, a.eps, on);
    if (a.pos) y.rotate(cs, sn, c, a.rot_dim, a.pairs);
  };
  // A wave may hold rows of all three kinds; the lanes of one head agree.
  if (kind == 0) {
    Chunk<float, E, BF16> y;
#pragma unroll
    for (int i = 0; i < E; ++i) y.x[i] = x[i];
    turn(y, a.q_norm);
    if (live) y.store(static_cast<char *>(a.q_out) + (((int64_t)tok * a.n_q + hk) * d + c) * ES);
  } else if (kind == 1) {
    Chunk<TK, E, BF16> y;
#pragma unroll
    for (int i = 0; i < E; ++i) y.x[i] = x[i];
    turn(y, a.k_norm);
    if constexpr (FOUR) y.store4(static_cast<uint8_t *>(a.pool_k) + at * (d / 2), a.ks + at * (d / kKv4Group), c, live);
    else if (live) y.store(static_cast<char *>(a.pool_k) + (at * d + c) * ES);
  } else {
    Chunk<float, E, BF16> y;
#pragma unroll
    for (int i = 0; i < E; ++i) y.x[i] = x[i];
    if constexpr (FOUR) y.store4(static_cast<uint8_t *>(a.pool_v) + at * (d / 2), a.vs + at * (d / kKv4Group), c, live);
    else if (live) y.store(static_cast<char *>(a.pool_v) + (at * d + c) * ES);
  }
}

// Rows of a 4-bit pool as values: eight columns a lane.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void kv4_read_kernel(ReadArgs a) {
  const int cw = a.head_dim >> 3, d = a.head_dim;           // chunks of a row
  const int64_t per = (int64_t)2 * a.n_kv * cw;             // and of a token
  const int64_t all = per * (a.tok1 - a.tok0), at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t i = at < all ? at : all - 1;
  const int tok = a.tok0 + (int)(i / per), in = (int)(i % per);
  const int c = in % cw, head = in / cw, hk = head % a.n_kv;
  const bool v = head >= a.n_kv;
  const int64_t row = (int64_t)hk * a.cap_total + pool_row(a.seq, a.nseq, tok);
  if (at >= all) return;
  const uint32_t w = *reinterpret_cast<const uint32_t *>((v ? a.v : a.k) + row * (d >> 1) + 4 * c);
  const uint32_t byte = (v ? a.vs : a.ks)[row * (d / kKv4Group) + (c >> 2)];
  const float unit = byte == kKv4Nan ? __uint_as_float(0x7FC00000u) : kv4_scale(byte);
  const int64_t o = ((int64_t)tok * a.n_kv + hk) * d + 8 * c;
  if (BF16) {
    *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(v ? a.v_out : a.k_out) + o) =
        byte == kKv4Nan ? uint4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u} : kv4_bf16x8(w, unit);
  } else {
    const f32x2_t p0 = kv4_f32x2<0>(w, unit), p1 = kv4_f32x2<1>(w, unit), p2 = kv4_f32x2<2>(w, unit), p3 = kv4_f32x2<3>(w, unit);
    f32x4 *dst = reinterpret_cast<f32x4 *>(static_cast<float *>(v ? a.v_out : a.k_out) + o);
    const bool nan = byte == kKv4Nan;
    dst[0] = nan ? f32x4{unit, unit, unit, unit} : f32x4{p0[0], p0[1], p1[0], p1[1]};
    dst[1] = nan ? f32x4{unit, unit, unit, unit} : f32x4{p2[0], p2[1], p3[0], p3[1]};
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

hipError_t launch_append(int dt, bool four, const AppendArgs &a, hipStream_t st) {
  int lph_log2 = 0;
  const int chunks = a.head_dim / (dt == 0 ? 4 : 8);
  while (1 << lph_log2 < chunks) ++lph_log2;
  const int64_t threads = ((int64_t)(a.tok1 - a.tok0) * (a.n_q + 2 * a.n_kv)) << lph_log2;
  const dim3 grid((uint32_t)((threads + kThreads - 1) / kThreads)), block(kThreads);
  if (dt == 0 && four) hipLaunchKernelGGL((append_kernel<false, true>), grid, block, 0, st, a, lph_log2);
  else if (dt == 0) hipLaunchKernelGGL((append_kernel<false, false>), grid, block, 0, st, a, lph_log2);
  else if (four) hipLaunchKernelGGL((append_kernel<true, true>), grid, block, 0, st, a, lph_log2);
  else hipLaunchKernelGGL((append_kernel<true, false>), grid, block, 0, st, a, lph_log2);
  return hipGetLastError();
}

hipError_t launch_kv4_read(int dt, const ReadArgs &a, hipStream_t st) {
  const int64_t threads = (int64_t)(a.tok1 - a.tok0) * 2 * a.n_kv * (a.head_dim / 8);
  const dim3 grid((uint32_t)((threads + kThreads - 1) / kThreads)), block(kThreads);
  if (dt == 0) hipLaunchKernelGGL((kv4_read_kernel<false>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((kv4_read_kernel<true>), grid, block, 0, st, a);
  return hipGetLastError();
}

hipError_t launch_kv4_compact(const Compact4Args &a, hipStream_t st) {
  hipLaunchKernelGGL(kv4_compact_kernel, dim3(a.nseq, a.n_kv), dim3(64), 0, st, a);
  return hipGetLastError();
}

}  // namespace specmemo

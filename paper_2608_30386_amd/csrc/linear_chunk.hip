// Linear attention with a decay for each head: the chunked form, for prompts (dk = 64 or 128).
//
// Over a chunk of 64 tokens with running log-decays G (from the chunk's start) and D_ts =
// e^{G_t - G_s} for s <= t, else 0:
//     P = (Q K^T) . D                        A = Diag(beta) ((K K^T) . D) below the diagonal
//     U = V   (plain rule)                   T = (I + A)^-1 Diag(beta),
//                                            U = T (V - e^G (K S))   (delta rule)
//     O = scale (e^G (Q S) + P U)            S <- e^{G_C} S + K^T (e^{G_C - G} U)
// Every exponent is a difference of running sums in the order of the tokens, so no factor of a decay
// overflows, whatever the log-decays are; the running sums are 64-bit, which keeps the difference
// of two large ones exact.
//
// A wave holds the whole state of 16 columns in accumulators and walks over the chunks.  An operand
// of a matrix instruction is eight consecutive channels or tokens of a lane's row: accumulators chain
// as B operands without leaving registers if row m of tile t stands for row
//     sigma(t, m) = 32 (t / 2) + 8 (m / 4) + 4 (t % 2) + m % 4
// of the matrix, because lane (q, n) then holds rows 8 q .. 8 q + 7 of each group of 32 in the tiles
// 2 s and 2 s + 1.  Keys as K^T and values as B operands come from LDS through the transposing read.
//
// Precision.  Keys, queries and values are bf16, products with them are exact.  A 32-bit operand of a
// sum that reaches the state is cut into three bf16 planes of eight bits each, 24 bits in all, so the
// state is as good as in fp32 arithmetic (two planes leave 5e-6 of its norm, three 2e-7).  What only
// the output needs (S in Q S, P, U in P U) has two planes, 16 bits, before its rounding to bf16.

#include "linear_attn.h"

#include <hip/hip_runtime.h>

#include <cstdint>

#include "launch_common.h"
#include "wy_ops.h"

namespace dasc {
namespace {

using dasc_wy::bf16x8;
using dasc_wy::f32x4;
using dasc_wy::mma;
using dasc_wy::mma32;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int kC = 64;                       // tokens of a chunk

// ---- what is known of a request's chunks -------------------------------------------------------

struct ChunkArgs {
  LinearArgs a;
  int32_t q_tok, k_tok, v_tok, o_tok;        // token strides, below 2^31
  char* packets;                             // delta: what the factor kernel leaves for each chunk and head
  float* seg_state;                          // plain: [segments, H, dk, dv]
  double* seg_log2;                          // plain: [segments, H], the decay over a segment
  int32_t seg_chunks;                        // plain: chunks of a segment
  int32_t col_blocks;
};

__device__ inline int64_t clamp_row(const LinearArgs& a, int i) {
  const int64_t b = a.cu[i];
  return b < 0 ? 0 : b > a.n_tokens ? a.n_tokens : b;
}

// Units of `len` tokens (chunks, segments) of all requests are numbered so that request i's start at
// cu[i] / len + i: numbers ascend, no two requests share one, and there are at most
// n_tokens / len + n_req of them.
__device__ inline int64_t first_unit(const LinearArgs& a, int i, int len) { return clamp_row(a, i) / len + i; }

// the request that unit u belongs to
__device__ inline int unit_request(const LinearArgs& a, int64_t u, int len) {
  int lo = 0, hi = a.n_req - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (first_unit(a, mid, len) <= u) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// ---- operands ------------------------------------------------------------------------------------

__device__ inline int sigma(int t, int m) { return 32 * (t / 2) + 8 * (m / 4) + 4 * (t % 2) + m % 4; }

// Where the 16-byte unit u of a row lies among the row's U units in LDS.  A row of A operands is read
// by eight lanes at a time (tokens 0 .. 3 and 8 .. 11 of one unit), the transposing read takes four
// tokens of four units: neither meets a bank twice.
template <int U>
__device__ inline int swizzle(int row, int u) {
  if constexpr (U == 16) return u ^ (((row & 3) << 2) | ((row >> 2) & 3));
  else if constexpr (U == 8) return u ^ ((((row >> 1) & 1) << 2) | (((row >> 3) & 1) << 1) | ((row >> 2) & 1));
  else return u;
}

template <int U>
__device__ inline bf16x8 row_unit(const char* base, int row, int u) {
  return *reinterpret_cast<const bf16x8*>(base + (row * U + swizzle<U>(row, u)) * 16);
}

// Rows r0 + 8 q .. + 7 of 16 columns as an operand whose lane (q, m) holds eight rows of one column:
// the columns are four runs of four, run c at 8-byte position `half0 + step c` of a row.
template <int U>
__device__ inline bf16x8 columns(const char* base, int r0, int half0, int step, int lane) {
  const int q = lane / 16, k = lane % 16 / 4, c = lane % 4;
  const int half = half0 + step * c;
  union { s16x4 h[2]; bf16x8 v; } x;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int row = r0 + 8 * q + 4 * j + k;
    const char* p = base + (row * U + swizzle<U>(row, half / 2)) * 16 + (half % 2) * 8;
    x.h[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p));
  }
  return x.v;
}

__device__ inline uint32_t high_halves(float x0, float x1) {
  return __builtin_amdgcn_perm(__float_as_uint(x1), __float_as_uint(x0), 0x07060302u);
}
__device__ inline float rest(float x) { return x - __uint_as_float(__float_as_uint(x) & 0xFFFF0000u); }

// x = p[0] + p[1] (+ p[2]): planes of eight bits, cut off, not rounded; three of them are exact
template <int N>
__device__ inline void planes(const float (&x)[8], bf16x8 (&p)[N]) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    u32x4 w = {high_halves(r[0], r[1]), high_halves(r[2], r[3]), high_halves(r[4], r[5]), high_halves(r[6], r[7])};
    p[n] = __builtin_bit_cast(bf16x8, w);
    if (n + 1 < N) {
#pragma unroll
      for (int e = 0; e < 8; ++e) r[e] = rest(r[e]);
    }
  }
}

template <int N>
__device__ inline void planes(f32x4 lo, f32x4 hi, bf16x8 (&p)[N]) {
  const float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  planes<N>(x, p);
}

__device__ inline void widen8(bf16x8 b, float (&x)[8]) {
  const u32x4 w = __builtin_bit_cast(u32x4, b);
  const uint32_t v[4] = {w[0], w[1], w[2], w[3]};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = bf16_lo(v[e]);
    x[2 * e + 1] = bf16_hi(v[e]);
  }
}

// ---- the decays of a chunk --------------------------------------------------------------------------

struct Decays {
  double G[kC];            // running log2-decays
  float eo[kC];            // scale e^G
  float e[kC];             // e^G
  float er[kC];            // e^{G_C - G}
  float m;                 // the state's decay: S m, or S + S m if near
  int32_t near;
  int32_t pad[2];
};

// One wave fills in a chunk's decays, one token per lane; g: the token's log-decay, 0 past the end.
// A log-decay below -2000 (in powers of two) is as good as -2000: both are a decay of 0.
__device__ inline void make_decays(Decays& d, float g, float scale, int lane) {
  double x = double(g) * 1.4426950408889634;
  if (x < -2000.0) x = -2000.0;
#pragma unroll
  for (int s = 1; s < kC; s *= 2) {
    const double y = __shfl_up(x, s);
    if (lane >= s) x += y;
  }
  const double end = __shfl(x, kC - 1);
  const float e = dasc_wy::ex2(float(x));
  d.G[lane] = x;
  d.e[lane] = e;
  d.eo[lane] = scale * e;
  d.er[lane] = dasc_wy::ex2(float(end - x));
  if (lane == 0) {
    const double f = exp2(end);
    const bool near = end > -0.72;
    d.m = float(near ? f - 1.0 : f);
    d.near = near;
  }
}

// D_ts for s <= t from the running sums
__device__ inline float decay_of(double gt, double gs) { return dasc_wy::ex2(float(gt - gs)); }

template <int NT>
__device__ inline void decay_state(f32x4 (&S)[NT], const Decays& d) {
  const float m = d.m;
  if (d.near) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) S[t][i] = fmaf(S[t][i], m, S[t][i]);
  } else {
#pragma unroll
    for (int t = 0; t < NT; ++t) S[t] *= m;
  }
}

// the block's waves see each other's LDS writes; loads from memory stay in flight
__device__ inline void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// ---- the walk over the chunks -------------------------------------------------------------------------

// Lower blocks (t, s) of a 64 x 64 matrix in A-operand order: rows sigma(t, .), columns 32 s .. + 31,
// s <= t / 2, 1 KB each
__device__ inline constexpr int block_of(int t, int s) { return t < 2 ? t : 2 + 2 * (t - 2) + s; }
constexpr int kBlocks = 6;
constexpr int kPBytes = 2 * kBlocks * 1024;       // P: two planes
constexpr int kTBytes = 3 * kBlocks * 1024;       // T: three planes
constexpr int kPacket = kTBytes + kPBytes + int(sizeof(Decays));
static_assert(sizeof(Decays) % 16 == 0, "packets are copied in 16-byte units");

// P for one query tile c (tokens 16 c ..) and key group s, written into its A-operand blocks
template <int DK, typename LoadK, typename LoadQ>
__device__ inline void make_p(char* P, const double* G, float scale, int c, int s, int lane, LoadK&& ku, LoadQ&& qu) {
  const int q = lane / 16, n = lane % 16;
  f32x4 a0 = {0, 0, 0, 0}, a1 = {0, 0, 0, 0};
#pragma unroll
  for (int kk = 0; kk < DK / 32; ++kk) {
    const bf16x8 b = qu(16 * c + n, 4 * kk + q);
    a0 = mma(ku(sigma(2 * s, n), 4 * kk + q), b, a0);
    a1 = mma(ku(sigma(2 * s + 1, n), 4 * kk + q), b, a1);
  }
  // this lane: query token 16 c + n, key tokens 32 s + 8 q ..
  const int tq = 16 * c + n, tk = 32 * s + 8 * q;
  const double gq = G[tq];
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float v = (e < 4 ? a0[e & 3] : a1[e & 3]) * (scale * decay_of(gq, G[tk + e]));
    x[e] = tk + e <= tq ? v : 0.0f;
  }
  bf16x8 hi, lo;
  dasc_wy::split8(x, hi, lo);
  const int r = tq % 32, t = 2 * (tq / 32) + (r / 4) % 2, m = 4 * (r / 8) + r % 4;
  char* at = P + block_of(t, s) * 1024 + (16 * q + m) * 16;
  *reinterpret_cast<bf16x8*>(at) = hi;
  *reinterpret_cast<bf16x8*>(at + kBlocks * 1024) = lo;
}

template <int DK, int NW, bool DELTA, bool OUT>
struct Layout {
  static constexpr int kRow = kC * DK * 2;
  static constexpr int kV = kRow * (OUT ? 2 : 1);
  static constexpr int kP = kV + kC * NW * 32;
  static constexpr int kT = kP + (OUT ? kPBytes : 0);
  static constexpr int kD = kT + (DELTA ? kTBytes : 0);
  static constexpr int kBytes = kD + int(sizeof(Decays)) * (DELTA ? 1 : 2);
};

// One block walks one request (delta) or one segment of one (plain) of a head, 16 NW columns.
// LOCAL: only what the segment adds to a state of zero, left in seg_state for the join.
template <int DK, int NW, bool DELTA, bool OUT, bool LOCAL>
__global__ __launch_bounds__(64 * NW) void linear_chunk_kernel(ChunkArgs p) {
  constexpr int NT = 64 * NW, KT = DK / 16, U = DK / 8, UV = 2 * NW;
  using L = Layout<DK, NW, DELTA, OUT>;
  __shared__ __attribute__((aligned(16))) char lds[L::kBytes];
  char* const K = lds;
  char* const Q = lds + L::kRow;
  char* const V = lds + L::kV;
  char* const P = lds + L::kP;
  char* const T = lds + L::kT;
  Decays* const dec = reinterpret_cast<Decays*>(lds + L::kD);

  const LinearArgs& a = p.a;
  const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64, q = lane / 16, n = lane % 16;
  const int cb = blockIdx.x % p.col_blocks;
  const int h = blockIdx.x / p.col_blocks % a.H;
  const int64_t unit = blockIdx.x / p.col_blocks / a.H;
  const int hk = h / a.rep, dv = a.dv;

  // the tokens of this block
  int i, c0, chunks;
  bool first = true, last = true;
  Span sp;
  if constexpr (DELTA) {
    i = int(unit);
    sp = request_span(a, i);
    c0 = 0;
    chunks = (sp.len + kC - 1) / kC;
  } else {
    const int seg = p.seg_chunks;
    if (seg == 0) {
      i = int(unit);
      sp = request_span(a, i);
      c0 = 0;
      chunks = (sp.len + kC - 1) / kC;
    } else {
      i = unit_request(a, unit, seg * kC);
      sp = request_span(a, i);
      const int64_t j = unit - first_unit(a, i, seg * kC);
      const int all = (sp.len + kC - 1) / kC;
      if (j < 0 || (j * seg >= all && j > 0)) return;
      c0 = int(j) * seg;
      chunks = all - c0 < seg ? all - c0 : seg;
      first = false;                        // the join has left every segment's start
      last = c0 + chunks >= all;
    }
  }
  const int64_t row0 = sp.begin + int64_t(c0) * kC;
  const int len = sp.len - c0 * kC;         // tokens from row0 to the request's end

  // the state: lane (q, n) holds channels sigma(t, 4 q + i) of column n
  const int col = 16 * (cb * NW + wave) + n;
  const bool in = col < dv;
  f32x4 S[KT];
  {
    const float* from = LOCAL ? nullptr
                       : first ? slot_state(a, a.src, i, h, DK)
                               : p.seg_state + (unit * a.H + h) * int64_t(DK) * dv;
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        S[t][e] = from && in ? from[int64_t(sigma(t, 4 * q + e)) * dv + col] : 0.0f;
  }

  // staging: 16-byte units of K, Q and V rows, and the packet, through registers
  constexpr int kRowsPass = NT / U, kPasses = kC / kRowsPass;
  constexpr int kVRows = NT / UV, kVPasses = kC / kVRows;
  constexpr int kPk = DELTA ? ((OUT ? kPacket : kPacket - kPBytes) / 16 + NT - 1) / NT : 0;
  u32x4 rk[kPasses], rq[OUT ? kPasses : 1], rv[kVPasses], rp[kPk ? kPk : 1];
  float g_next = 0;
  const uint16_t* const kb = a.io.k + row0 * p.k_tok + hk * a.io.k_head + 8 * (tid % U);
  const uint16_t* const qb = OUT ? a.io.q + row0 * p.q_tok + hk * a.io.q_head + 8 * (tid % U) : nullptr;
  const int vcol = 16 * NW * cb + 8 * (tid % UV);
  const uint16_t* const vb = a.io.v + row0 * p.v_tok + h * a.io.v_head + vcol;
  const int64_t slot0 = DELTA ? first_unit(a, i, kC) + c0 : 0;

  const auto load = [&](int c) {
    const int at = c * kC, end = len - 1;   // rows past the end repeat the last one
#pragma unroll
    for (int j = 0; j < kPasses; ++j) {
      int r = at + j * kRowsPass + tid / U;
      r = r < end ? r : end;
      rk[j] = *reinterpret_cast<const u32x4*>(kb + int64_t(r) * p.k_tok);
      if (OUT) rq[j] = *reinterpret_cast<const u32x4*>(qb + int64_t(r) * p.q_tok);
    }
#pragma unroll
    for (int j = 0; j < kVPasses; ++j) {    // values past the end are zero, and so is what they add
      const int r = at + j * kVRows + tid / UV;
      rv[j] = r <= end && vcol < dv ? *reinterpret_cast<const u32x4*>(vb + int64_t(r) * p.v_tok) : u32x4{0, 0, 0, 0};
    }
    if constexpr (DELTA) {
      const char* pk = p.packets + ((slot0 + c) * a.H + h) * kPacket;
#pragma unroll
      for (int j = 0; j < kPk; ++j) {
        int off = (j * NT + tid) * 16;
        if (!OUT && off >= kTBytes) off += kPBytes;
        if (off < kPacket) rp[j] = *reinterpret_cast<const u32x4*>(pk + off);
      }
    }
  };
  const auto load_g = [&](int c) {
    const int r = c * kC + lane;
    return r < len ? a.io.g[(row0 + r) * a.io.g_tok + h * a.io.g_head] : 0.0f;
  };
  const auto stage = [&]() {
#pragma unroll
    for (int j = 0; j < kPasses; ++j) {
      const int r = j * kRowsPass + tid / U, at = (r * U + swizzle<U>(r, tid % U)) * 16;
      *reinterpret_cast<u32x4*>(K + at) = rk[j];
      if (OUT) *reinterpret_cast<u32x4*>(Q + at) = rq[j];
    }
#pragma unroll
    for (int j = 0; j < kVPasses; ++j) {
      const int r = j * kVRows + tid / UV;
      *reinterpret_cast<u32x4*>(V + (r * UV + swizzle<UV>(r, tid % UV)) * 16) = rv[j];
    }
    if constexpr (DELTA) {
#pragma unroll
      for (int j = 0; j < kPk; ++j) {
        int off = (j * NT + tid) * 16;
        if (!OUT && off >= kTBytes) off += kPBytes;
        if (off < kPacket) {
          char* to = off < kTBytes ? T + off
                     : off < kTBytes + kPBytes ? P + (off - kTBytes)
                                               : reinterpret_cast<char*>(dec) + (off - kTBytes - kPBytes);
          *reinterpret_cast<u32x4*>(to) = rp[j];
        }
      }
    }
  };

  double log2_sum = 0;                      // LOCAL: the segment's decay
  if (chunks > 0) {
    load(0);
    if constexpr (!DELTA) {
      if (wave == NW - 1) {
        make_decays(dec[0], load_g(0), a.scale, lane);
        g_next = load_g(1);
      }
    }
    stage();
  }
  __syncthreads();

  for (int c = 0; c < chunks; ++c) {
    const Decays& d = DELTA ? dec[0] : dec[c & 1];
    if (c + 1 < chunks) load(c + 1);
    f32x4 O[4], X[4];
    bf16x8 v[2];
    // what needs the state: Q S, K S
    if constexpr (OUT || DELTA) {
#pragma unroll
      for (int t = 0; t < 4; ++t) O[t] = X[t] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < DK / 32; ++s) {
        bf16x8 sp_[3];
        planes<3>(S[2 * s], S[2 * s + 1], sp_);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int r = sigma(t, n);
          if constexpr (DELTA) {
            const bf16x8 k = row_unit<U>(K, r, 4 * s + q);
            X[t] = mma(k, sp_[2], X[t]);
            X[t] = mma(k, sp_[1], X[t]);
            X[t] = mma(k, sp_[0], X[t]);
          }
          if constexpr (OUT) {
            const bf16x8 x = row_unit<U>(Q, r, 4 * s + q);
            O[t] = mma(x, sp_[1], O[t]);
            O[t] = mma(x, sp_[0], O[t]);
          }
        }
      }
    }
    if constexpr (!DELTA) {
      if constexpr (OUT) {
        for (int w = wave; w < kBlocks; w += NW) {
          const int qt = w < 2 ? w : 2 + (w - 2) / 2, s = w < 2 ? 0 : (w - 2) % 2;
          make_p<DK>(P, d.G, a.scale, qt, s, lane,
                     [&](int r, int u) { return row_unit<U>(K, r, u); },
                     [&](int r, int u) { return row_unit<U>(Q, r, u); });
        }
      }
      if (wave == NW - 1 && c + 1 < chunks) {
        make_decays(dec[(c + 1) & 1], g_next, a.scale, lane);
        g_next = load_g(c + 2);
      }
      if constexpr (OUT) lds_barrier();     // P is whole
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) v[s] = columns<UV>(V, 32 * s, 4 * wave, 1, lane);

    f32x4 Uf[4];                            // U in fp32
    if constexpr (DELTA) {
      bf16x8 y[2][3];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        float x[8];
        widen8(v[s], x);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          x[e] = fmaf(-d.e[32 * s + 8 * q + e], X[2 * s + e / 4][e % 4], x[e]);
        planes<3>(x, y[s]);
      }
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        Uf[t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s <= t / 2; ++s) {
          const char* b = T + block_of(t, s) * 1024 + lane * 16;
          const bf16x8 t0 = *reinterpret_cast<const bf16x8*>(b);
          const bf16x8 t1 = *reinterpret_cast<const bf16x8*>(b + kBlocks * 1024);
          const bf16x8 t2 = *reinterpret_cast<const bf16x8*>(b + 2 * kBlocks * 1024);
          Uf[t] = mma(t2, y[s][0], Uf[t]);
          Uf[t] = mma(t0, y[s][2], Uf[t]);
          Uf[t] = mma(t1, y[s][1], Uf[t]);
          Uf[t] = mma(t1, y[s][0], Uf[t]);
          Uf[t] = mma(t0, y[s][1], Uf[t]);
          Uf[t] = mma(t0, y[s][0], Uf[t]);
        }
      }
    } else {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        float x[8];
        widen8(v[s], x);
#pragma unroll
        for (int e = 0; e < 8; ++e) Uf[2 * s + e / 4][e % 4] = x[e];
      }
    }

    if constexpr (OUT) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) O[t][e] *= d.eo[32 * (t / 2) + 8 * q + 4 * (t % 2) + e];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        bf16x8 u[2];
        if constexpr (DELTA) planes<2>(Uf[2 * s], Uf[2 * s + 1], u);
#pragma unroll
        for (int t = 2 * s; t < 4; ++t) {
          const char* b = P + block_of(t, s) * 1024 + lane * 16;
          const bf16x8 p0 = *reinterpret_cast<const bf16x8*>(b);
          const bf16x8 p1 = *reinterpret_cast<const bf16x8*>(b + kBlocks * 1024);
          if constexpr (DELTA) {
            O[t] = mma(p0, u[1], O[t]);
            O[t] = mma(p1, u[0], O[t]);
            O[t] = mma(p0, u[0], O[t]);
          } else {
            O[t] = mma(p1, v[s], O[t]);
            O[t] = mma(p0, v[s], O[t]);
          }
        }
      }
      if (in) {
        uint16_t* ob = a.io.o + (row0 + int64_t(c) * kC) * p.o_tok + h * a.io.o_head + col;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = 32 * (t / 2) + 8 * q + 4 * (t % 2) + e;
            if (c * kC + r < len) ob[int64_t(r) * p.o_tok] = __builtin_bit_cast(uint16_t, __bf16(O[t][e]));
          }
      }
    }

    // the state
    decay_state<KT>(S, d);
    if constexpr (LOCAL) log2_sum += d.G[kC - 1];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      bf16x8 u[3];
      f32x4 x0, x1;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x0[e] = Uf[2 * s][e] * d.er[32 * s + 8 * q + e];
        x1[e] = Uf[2 * s + 1][e] * d.er[32 * s + 8 * q + 4 + e];
      }
      planes<3>(x0, x1, u);
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        const bf16x8 k = columns<U>(K, 32 * s, 8 * (t / 2) + t % 2, 2, lane);
        S[t] = mma(k, u[2], S[t]);
        S[t] = mma(k, u[1], S[t]);
        S[t] = mma(k, u[0], S[t]);
      }
    }
    lds_barrier();                          // everybody is done with this chunk
    if (c + 1 < chunks) {
      stage();
      lds_barrier();
    }
  }

  float* to = nullptr;
  if constexpr (LOCAL) {
    to = p.seg_state + (unit * a.H + h) * int64_t(DK) * dv;
    if (tid == 0 && cb == 0) p.seg_log2[unit * a.H + h] = log2_sum;
  } else if (last) {
    to = slot_state(a, a.dst, i, h, DK);
  }
  if (to && in) {
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) to[int64_t(sigma(t, 4 * q + e)) * dv + col] = S[t][e];
  }
}

// ---- plain rule: the segments of a request joined ------------------------------------------------------

// Segment j's start: its own from the request's first state, and what the segments before it add.
// Replaces the segments' sums by their starts; with no output to come, writes the last state.
__global__ __launch_bounds__(256) void linear_join_kernel(ChunkArgs p, int dk, bool finish) {
  const LinearArgs& a = p.a;
  const int64_t per = int64_t(dk) * a.dv;
  const int64_t x = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 4;     // dv is a multiple of 4
  if (x >= per) return;
  const int h = blockIdx.y, i = blockIdx.z;
  const int len = p.seg_chunks * kC;
  const Span sp = request_span(a, i);
  const int segs = sp.len > 0 ? (sp.len + len - 1) / len : 1;
  const int64_t u0 = first_unit(a, i, len);
  const float* from = slot_state(a, a.src, i, h, dk);
  f32x4 S = from ? *reinterpret_cast<const f32x4*>(from + x) : f32x4{0, 0, 0, 0};
  for (int j = 0; j < segs; ++j) {
    const int64_t u = u0 + j;
    f32x4* at = reinterpret_cast<f32x4*>(p.seg_state + (u * a.H + h) * per + x);
    const f32x4 add = *at;
    *at = S;
    if (j + 1 < segs || finish) {
      const double end = p.seg_log2[u * a.H + h];
      const double f = exp2(end);
      if (end > -0.72) {
        const float m = float(f - 1.0);
#pragma unroll
        for (int e = 0; e < 4; ++e) S[e] = fmaf(S[e], m, S[e]) + add[e];
      } else {
        S = S * float(f) + add;
      }
    }
  }
  if (finish) {
    float* to = slot_state(a, a.dst, i, h, dk);
    if (to) *reinterpret_cast<f32x4*>(to + x) = S;
  }
}

// ---- delta rule: T, P and the decays of every chunk -----------------------------------------------------

constexpr int kTS = 68;                     // floats from row to row of a 64 x 64 matrix in LDS

// 16 x 16 block product on fp32 matrix instructions: c + x y, x and y in LDS, y's rows `ys` apart
__device__ inline f32x4 block_mul(const float* x, const float* y, int ys, f32x4 c, int lane) {
  const int q = lane / 16, r = lane % 16;
#pragma unroll
  for (int k = 0; k < 4; ++k) c = mma32(x[r * kTS + 4 * k + q], y[(4 * k + q) * ys + r], c);
  return c;
}

template <int DK, bool OUT>
__global__ __launch_bounds__(256) void linear_factor_kernel(ChunkArgs p) {
  constexpr int NW = 4;
  __shared__ __attribute__((aligned(16))) float A[kC * kTS], T[kC * kTS], W[NW][16 * 20];
  __shared__ __attribute__((aligned(16))) Decays dec;
  __shared__ float bt[kC];
  const LinearArgs& a = p.a;
  const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64, q = lane / 16, n = lane % 16;
  const int h = blockIdx.x % a.H;
  const int64_t unit = blockIdx.x / a.H;
  const int hk = h / a.rep;
  const int i = unit_request(a, unit, kC);
  const Span sp = request_span(a, i);
  const int64_t c = unit - first_unit(a, i, kC);
  if (c < 0 || c * kC >= sp.len) return;
  const int64_t row0 = sp.begin + c * kC;
  const int len = sp.len - int(c) * kC;     // tokens from row0 to the request's end

  const uint16_t* const kb = a.io.k + row0 * p.k_tok + hk * a.io.k_head;
  const uint16_t* const qb = OUT ? a.io.q + row0 * p.q_tok + hk * a.io.q_head : nullptr;
  const auto ku = [&](int r, int u) {
    r = r < len ? r : len - 1;
    return *reinterpret_cast<const bf16x8*>(kb + int64_t(r) * p.k_tok + 8 * u);
  };
  const auto qu = [&](int r, int u) {
    r = r < len ? r : len - 1;
    return *reinterpret_cast<const bf16x8*>(qb + int64_t(r) * p.q_tok + 8 * u);
  };

  // K K^T, rows 16 wave .., in registers until the decays are there
  f32x4 kk[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) kk[t] = f32x4{0, 0, 0, 0};
#pragma unroll
  for (int s = 0; s < DK / 32; ++s) {
    const bf16x8 x = ku(16 * wave + n, 4 * s + q);
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (t <= wave) kk[t] = mma(x, ku(16 * t + n, 4 * s + q), kk[t]);
  }
  if (wave == 0) {
    const bool on = lane < len;
    const int64_t r = row0 + lane;
    bt[lane] = on ? a.io.beta[r * a.io.beta_tok + h * a.io.beta_head] : 0.0f;
    make_decays(dec, on ? a.io.g[r * a.io.g_tok + h * a.io.g_head] : 0.0f, a.scale, lane);
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 16 * wave + 4 * q + e, s = 16 * t + n;
      A[r * kTS + s] = s < r ? bt[r] * kk[t][e] * decay_of(dec.G[r], dec.G[s]) : 0.0f;
      T[r * kTS + s] = 0.0f;
    }
  __syncthreads();

  // T = (I + A)^-1: the diagonal blocks by substitution, a column per lane
  if (lane < 16) {
    const float* Ad = A + (16 * wave) * kTS + 16 * wave;
    float x[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float s = r == lane ? 1.0f : 0.0f;
#pragma unroll
      for (int j = 0; j < r; ++j) s = fmaf(-Ad[r * kTS + j], x[j], s);
      x[r] = s;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) T[(16 * wave + r) * kTS + 16 * wave + lane] = x[r];
  }
  __syncthreads();
  // the blocks below, one diagonal after another: T_ij = -T_ii sum_k A_ik T_kj
#pragma unroll
  for (int d = 1; d < 4; ++d) {
    if (wave < 4 - d) {
      const int bi = wave + d, bj = wave;
      f32x4 x = {0, 0, 0, 0};
      for (int k = bj; k < bi; ++k) x = block_mul(A + 16 * bi * kTS + 16 * k, T + 16 * k * kTS + 16 * bj, kTS, x, lane);
#pragma unroll
      for (int e = 0; e < 4; ++e) W[wave][(4 * q + e) * 20 + n] = -x[e];
      dasc_wy::wave_lds_sync();
      x = block_mul(T + 16 * bi * kTS + 16 * bi, W[wave], 20, f32x4{0, 0, 0, 0}, lane);
#pragma unroll
      for (int e = 0; e < 4; ++e) T[(16 * bi + 4 * q + e) * kTS + 16 * bj + n] = x[e];
    }
    __syncthreads();
  }

  char* const pk = p.packets + (unit * a.H + h) * kPacket;
  for (int b = wave; b < kBlocks; b += NW) {
    const int t = b < 2 ? b : 2 + (b - 2) / 2, s = b < 2 ? 0 : (b - 2) % 2;
    const float* row = T + sigma(t, n) * kTS + 32 * s + 8 * q;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = row[e] * bt[32 * s + 8 * q + e];
    bf16x8 pl[3];
    planes<3>(x, pl);
#pragma unroll
    for (int j = 0; j < 3; ++j)
      *reinterpret_cast<bf16x8*>(pk + (j * kBlocks + b) * 1024 + lane * 16) = pl[j];
  }
  if constexpr (OUT) {
    for (int b = wave; b < kBlocks; b += NW) {
      const int qt = b < 2 ? b : 2 + (b - 2) / 2, s = b < 2 ? 0 : (b - 2) % 2;
      make_p<DK>(pk + kTBytes, dec.G, a.scale, qt, s, lane, ku, qu);
    }
  }
  for (int b = tid; b < int(sizeof(Decays)) / 16; b += 256)
    reinterpret_cast<u32x4*>(pk + kTBytes + kPBytes)[b] = reinterpret_cast<const u32x4*>(&dec)[b];
}

// ---- launches --------------------------------------------------------------------------------------------

// Blocks that fill the chip: two on each of 256 CUs
constexpr int64_t kFill = 512;
constexpr int kMinSegment = 8;              // chunks of a segment at least: its state costs what 4 chunks do

int waves_of(int dv) { return dv <= 32 ? 2 : dv <= 64 ? 4 : 8; }

// chunks of a segment of the plain rule, 0: requests are not split
int segment_chunks(const ChunkPlan& c) {
  if (c.delta) return 0;
  const int64_t blocks = int64_t(c.n_req) * c.H * ((c.dv + 127) / 128);
  if (blocks >= kFill / 2) return 0;
  const int64_t per = kFill / blocks;       // segments a request can use
  int64_t chunks = (c.n_tokens / kC / c.n_req + per) / (per > 0 ? per : 1);
  if (chunks < kMinSegment) chunks = kMinSegment;
  return c.max_len > 2 * chunks * kC ? int(chunks) : 0;
}

int64_t units_of(const ChunkPlan& c, int64_t tokens) { return c.n_tokens / tokens + c.n_req; }

template <int DK, int NW, bool DELTA, bool OUT, bool LOCAL>
void launch_walk(const ChunkArgs& p, int64_t units, hipStream_t st) {
  linear_chunk_kernel<DK, NW, DELTA, OUT, LOCAL><<<uint32_t(units * p.a.H * p.col_blocks), 64 * NW, 0, st>>>(p);
}

template <int DK, int NW>
void launch_rule(const ChunkPlan& c, ChunkArgs& p, char* ws, hipStream_t st) {
  const bool out = p.a.io.o;
  p.col_blocks = (c.dv + 16 * NW - 1) / (16 * NW);
  if (c.delta) {
    p.packets = ws;
    const uint32_t grid = uint32_t(units_of(c, kC) * c.H);
    if (out) {
      linear_factor_kernel<DK, true><<<grid, 256, 0, st>>>(p);
      launch_walk<DK, NW, true, true, false>(p, c.n_req, st);
    } else {
      linear_factor_kernel<DK, false><<<grid, 256, 0, st>>>(p);
      launch_walk<DK, NW, true, false, false>(p, c.n_req, st);
    }
    return;
  }
  p.seg_chunks = segment_chunks(c);
  if (p.seg_chunks == 0) {
    if (out) launch_walk<DK, NW, false, true, false>(p, c.n_req, st);
    else launch_walk<DK, NW, false, false, false>(p, c.n_req, st);
    return;
  }
  const int64_t units = units_of(c, int64_t(p.seg_chunks) * kC);
  p.seg_state = reinterpret_cast<float*>(ws);
  p.seg_log2 = reinterpret_cast<double*>(ws + units * c.H * int64_t(DK) * c.dv * 4);
  launch_walk<DK, NW, false, false, true>(p, units, st);
  linear_join_kernel<<<dim3((DK * c.dv + 1023) / 1024, c.H, c.n_req), 256, 0, st>>>(p, DK, !out);
  if (out) launch_walk<DK, NW, false, true, false>(p, units, st);
}

}  // namespace

bool linear_chunk_supported(const ChunkPlan& c) {
  return (c.dk == 64 || c.dk == 128) && c.dv % 16 == 0 && c.n_tokens > 0;
}

int64_t linear_chunk_workspace(const ChunkPlan& c) {
  if (c.delta) return units_of(c, kC) * c.H * kPacket;
  const int seg = segment_chunks(c);
  return seg ? units_of(c, int64_t(seg) * kC) * c.H * (int64_t(c.dk) * c.dv * 4 + 8) : 0;
}

void launch_linear_chunks(const ChunkPlan& c, const LinearArgs& a, void* ws, hipStream_t st) {
  ChunkArgs p{};
  p.a = a;
  p.q_tok = int32_t(a.io.q_tok);
  p.k_tok = int32_t(a.io.k_tok);
  p.v_tok = int32_t(a.io.v_tok);
  p.o_tok = int32_t(a.io.o_tok);
  char* w = static_cast<char*>(ws);
  switch (waves_of(c.dv)) {
#define DASC_WAVES(N)                                        \
  case N:                                                    \
    if (c.dk == 64) launch_rule<64, N>(c, p, w, st);         \
    else launch_rule<128, N>(c, p, w, st);                   \
    break;
    DASC_WAVES(2) DASC_WAVES(4) DASC_WAVES(8)
#undef DASC_WAVES
  }
}

}  // namespace dasc

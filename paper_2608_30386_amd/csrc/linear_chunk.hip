// Linear attention with a decay for each head: the chunked form, for prompts (dk = 64 or 128).
//
// Over a chunk of 64 tokens with running log-decays G (from the chunk's start) and D_ts =
// e^{G_t - G_s} for s <= t, else 0:
//     P = (Q K^T) . D                        A = Diag(beta) ((K K^T) . D) below the diagonal
//     U = V   (plain rule)                   T = (I + A)^-1 Diag(beta),
//                                            U = T (V - e^G (K S))   (delta rule)
//     O = scale (e^G (Q S) + P U)            S <- e^{G_C} S + K^T (e^{G_C - G} U)
// Every exponent is a difference of running sums in the order of the tokens, so no factor passes the growth
// over a chunk, one if nothing grows; the running sums are 64-bit, which keeps the difference of two large
// ones exact.  Log-decays above kGrowth are left to the token-by-token form: over a state of zero their
// product may pass what fp32 holds, and infinity times zero is NaN.
//
// A wave holds the whole state of 16 columns in accumulators and walks over the chunks.  An operand
// of a matrix instruction is eight consecutive channels or tokens of a lane's row: accumulators chain
// as B operands without leaving registers if row m of tile t stands for row
//     sigma(t, m) = 32 (t / 2) + 8 (m / 4) + 4 (t % 2) + m % 4
// of the matrix, because lane (q, n) then holds rows 8 q .. 8 q + 7 of each group of 32 in the tiles
// 2 s and 2 s + 1.  Keys as K^T and values as B operands come from LDS through the transposing read.
//
// What bounds it, 32 heads of 128 x 128.  Few heads: the chain of a chunk, 1.7 us with three exchanges
// through LDS, of which matrix instructions are a fifth (delta rule, 8192 tokens of one request: 224 us
// and 50 for the factors).  Many heads: a block for each request and head, one on a CU, so the call lasts
// as long as its longest request (8 requests of 777 tokens on average, of 1300 at most: 148 us, of which a
// wave lives half on average, and 26 for the factors); in a block, the issue of matrix and vector
// instructions, 40% of its time each.  The plain rule's segments are of one length and bound by that issue
// alone (16384 tokens of one request: 80, 8 and 152 us).  Memory traffic would take 42, 35 and 83 us.
//
// What is not finite.  T and P are multiplied a block at a time, the zeros above their diagonals with it, and
// zero times an infinity or NaN is NaN: one such value, key, state or factor reaches the outputs of tokens
// before it in its chunk.  It also reaches the state, and a state once NaN or infinite is so to the end.  So
// a walk looks at the last state of its columns, and where that is not finite takes those columns of the
// request again token by token, from the source slot, which nothing has written yet; the other columns
// keep theirs.  (A query that is not finite reaches its own outputs alone.)  The look costs 0.3 us a call.
//
// Precision.  Keys, queries and values are bf16, products with them are exact.  A 32-bit operand of a
// sum that reaches the state is cut into three bf16 planes of eight bits each, 24 bits in all, so the
// state is as good as in fp32 arithmetic (two planes leave 5e-6 of its norm, three 2e-7).  Of T Y, both
// of whose operands are cut, the products of two lowest planes and of a lowest with a middle one are left
// out, 2^-24 of the largest.  What only the output needs has 16 bits before its rounding to bf16, 8: S in
// Q S and U in P U two planes, cut off and so up to 2^-16 towards zero, P two rounded ones, and of P U the
// product of the two lower planes is left out, 2^-16.  An output whose terms cancel shows it, up to 2^-14 of
// |scale| |q| |S|.  Decays are the hardware's exponentials, within an ulp.

#include "linear_attn.h"

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "launch_common.h"
#include "linear_steps.h"
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
  int32_t q_tok, k_tok, v_tok, o_tok;        // token strides, below 2^24
  // delta: the call goes in windows of units (numbered chunks), whose packets share a workspace
  char* packets;                             // what the factor kernel leaves for each chunk and head of a window
  int64_t u0, u1;                            // this window
  const float* carry_in;                     // [H, dk, dv]: of the request that began in the window before
  float* carry_out;                          // and of the one that goes on in the next
  float* seg_state;                          // plain: [segments, H, dk, dv]
  double* seg_log2;                          // plain: [segments, H], the decay over a segment
  int32_t* seg_bad;                          // plain: [requests, H, blocks of the join, tiles], not finite at the end
  int32_t seg_chunks;                        // plain: chunks of a segment
  int32_t seg_each;                          // plain: segments of every request, 0: as many as it has tokens for
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

// A request's segments: numbered as units, or the same number for every request, where the last takes
// what is left (of a request that is longer than the caller said).
__device__ inline int64_t first_segment(const ChunkArgs& p, int i) {
  return p.seg_each ? int64_t(i) * p.seg_each : first_unit(p.a, i, p.seg_chunks * kC);
}
__device__ inline int segments(const ChunkArgs& p, int len) {
  const int seg = p.seg_chunks * kC, n = len > 0 ? (len - 1) / seg + 1 : 1;
  return p.seg_each && n > p.seg_each ? p.seg_each : n;
}

// the request that unit u belongs to
__device__ inline int unit_request(const LinearArgs& a, int64_t u, int len) {
  int lo = 0, hi = a.n_req - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (first_unit(a, mid, len) <= u) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// What is the same in every lane of a wave, said so: it then lives in scalar registers
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ inline int64_t uniform(int64_t x) {
  return int64_t(uint64_t(uint32_t(uniform(int(uint64_t(x) >> 32)))) << 32 | uint32_t(uniform(int(x))));
}

// ---- operands ------------------------------------------------------------------------------------

__device__ inline int sigma(int t, int m) { return 32 * (t / 2) + 8 * (m / 4) + 4 * (t % 2) + m % 4; }

// Rows in LDS lie 20 (or 12) 16-byte units apart, those of every other group of eight one unit on.  That
// spreads the transposing read's four rows of four units over the banks, and the eight rows (0 .. 3 and
// 8 .. 11 of one unit) in which a row of A operands is read.  (Not everything: 19% of the LDS cycles of the
// split walk and a third of those of the walk by columns are conflicts still; of which accesses is not
// known.)  Every address is a lane's base and a constant.
template <int U>
constexpr int kStride = U + 4;
template <int U>
constexpr int kRowsBytes = (kC * kStride<U> + 1) * 16;   // 64 rows
// values, of which a wave reads two units of four rows at a time
template <int U>
constexpr int kVStride = U + 2;

template <int U>
__device__ inline int row_at(int row) { return (row * kStride<U> + (row >> 3 & 1)) * 16; }

template <int U>
__device__ inline bf16x8 row_unit(const char* base, int row, int u) {
  return *reinterpret_cast<const bf16x8*>(base + row_at<U>(row) + u * 16);
}

// Row sigma(t, n) of a matrix in LDS is row sigma(0, n) and a constant on
template <int U>
__device__ inline bf16x8 sigma_unit(const char* base, int t, int n, int u) {
  return *reinterpret_cast<const bf16x8*>(base + row_at<U>(sigma(0, n)) + sigma(t, 0) * kStride<U> * 16 + u * 16);
}

// Rows r0 + 8 q .. + 7 of 16 columns as an operand whose lane (q, m) holds eight rows of one column: the
// columns are four runs of four, run c at byte step c from `lane_base`, this lane's place in row 8 q + k
template <int STRIDE>
__device__ inline bf16x8 columns(const char* lane_base, int r0, int at) {
  const char* p = lane_base + (r0 * STRIDE + at);
  union { s16x4 h[2]; bf16x8 v; } x;
  x.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p));
  x.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * STRIDE));
  return x.v;
}
template <int U>
__device__ inline int key_column(int lane) {
  return row_at<U>(lane / 16 * 8 + lane % 16 / 4) + lane % 4 * 16;
}
template <int U>
__device__ inline int value_column(int lane) {
  return (lane / 16 * 8 + lane % 16 / 4) * kVStride<U> * 16 + lane % 4 * 8;
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

// x of the lane that a DPP control names, 0 where there is none or the row is masked out
template <int CTRL, int ROWS>
__device__ inline double from_lane(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, int(uint32_t(u)), CTRL, ROWS, 0xF, true);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, int(uint32_t(u >> 32)), CTRL, ROWS, 0xF, true);
  return __builtin_bit_cast(double, uint64_t(hi) << 32 | lo);
}

// The most that a token's factor may grow by in chunks, in powers of two: 2^16 over a chunk, far from what
// fp32 cannot hold.  Beyond it the chunk's decay is NaN, and so the state, which the walk's end finds.
constexpr double kGrowth = 0.25;

// One wave fills in a chunk's decays, one token per lane; g: the token's log-decay, 0 past the end.
// A log-decay below -2000 (in powers of two) is as good as -2000: both are a decay of 0, as is what the
// rest of the chunk grows it to.
__device__ inline void make_decays(Decays& d, float g, float scale, int lane) {
  double x = double(g) * 1.4426950408889634;
  const bool grows = __any(x > kGrowth);
  if (x < -2000.0) x = -2000.0;
  x += from_lane<0x111, 0xF>(x);            // the lanes before it in a row of 16
  x += from_lane<0x112, 0xF>(x);
  x += from_lane<0x114, 0xF>(x);
  x += from_lane<0x118, 0xF>(x);
  x += from_lane<0x142, 0xA>(x);            // the last lane of the row before
  x += from_lane<0x143, 0xC>(x);            // the last lane of the first half
  const double end = __shfl(x, kC - 1);
  const float e = dasc_wy::ex2(float(x));
  d.G[lane] = x;
  d.e[lane] = e;
  d.eo[lane] = scale * e;
  d.er[lane] = dasc_wy::ex2(float(end - x));
  if (lane == 0) {
    const bool near = end > -0.72;
    d.m = grows ? __builtin_nanf("") : near ? expm1f(float(end * 0.6931471805599453)) : dasc_wy::ex2(float(end));
    d.near = near;
  }
}

// D_ts for s <= t from the running sums
__device__ inline float decay_of(double gt, double gs) { return dasc_wy::ex2(float(gt - gs)); }

// Results of matrix instructions that are read behind a branch.  The compiler waits for a result within a
// block of code, but not always on the paths that leave it: with a branch on the kind of the state's decay
// the outputs of a prompt's last chunk were read two instructions after the product that forms them, eight
// too few.  So the wait is written out where results cross a branch or leave the loop (ten instructions'
// time, against eight that the next read waits in any case).
#define DASC_SETTLE "s_nop 7\n\ts_nop 1"
__device__ inline void settle(f32x4& x) { asm volatile(DASC_SETTLE : "+v"(x)); }
template <int N>
__device__ inline void settle(f32x4 (&x)[N]) {
  static_assert(N == 1 || N == 2 || N == 4 || N == 8);
  if constexpr (N == 1) settle(x[0]);
  if constexpr (N == 2) asm volatile(DASC_SETTLE : "+v"(x[0]), "+v"(x[1]));
  if constexpr (N == 4) asm volatile(DASC_SETTLE : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]));
  if constexpr (N == 8)
    asm volatile(DASC_SETTLE
                 : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(x[4]), "+v"(x[5]), "+v"(x[6]), "+v"(x[7]));
}
#undef DASC_SETTLE

// The state's decay, without a branch on the chunk's kind: an instruction more for each element
template <int NT>
__device__ inline void decay_state(f32x4 (&S)[NT], const Decays& d) {
  const float m = d.m;
  const bool near = d.near;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) S[t][i] = fmaf(S[t][i], m, near ? S[t][i] : 0.0f);
}

// Whether all of these are finite: zero times anything else is NaN
template <int N>
__device__ inline bool finite(const f32x4 (&x)[N]) {
  float z = 0;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) z = fmaf(x[i][e], 0.0f, z);
  return z == 0.0f;
}

// the wave's stores are done: what it stores next to the same place comes after them
__device__ inline void stores_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// the block's waves see each other's LDS writes; loads from memory stay in flight
__device__ inline void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// ---- the walk over the chunks -------------------------------------------------------------------------

// Lower blocks (t, s) of a 64 x 64 matrix in A-operand order: rows sigma(t, .), columns 32 s .. + 31,
// s <= t / 2, 1 KB each
__device__ inline constexpr int block_of(int t, int s) { return t < 2 ? t : 2 + 2 * (t - 2) + s; }
constexpr int kBlocks = 6;
constexpr int kPBytes = 2 * kBlocks * 1024;       // P: two planes
constexpr int kTBytes = 3 * kBlocks * 1024;       // T: three planes
constexpr int kFBytes = kBlocks * 2048;           // T in fp32
static_assert(sizeof(Decays) % 16 == 0, "packets are copied in 16-byte units");

// What the factor kernel leaves for a chunk and head of the delta rule: decays and T, as planes and with
// P for the split walk, which has no instruction to spare; in fp32 and alone for the walk by columns,
// which is short of memory bandwidth and cuts T, and forms P, once for all its columns.
template <bool PLANES>
constexpr int kPacket = int(sizeof(Decays)) + (PLANES ? kTBytes + kPBytes : kFBytes);
constexpr int kPacketT = int(sizeof(Decays)), kPacketP = kPacketT + kTBytes;

// Block (t, s) of P as an A operand.  The product is formed transposed, keys as rows: its lane (q, n)
// then holds keys 32 s + 8 q .. + 7 of query sigma(t, n), which is what the operand's lane holds.
template <int DK, typename LoadK, typename LoadQ>
__device__ inline void make_p(const double* G, float scale, int t, int s, int lane, LoadK&& ku, LoadQ&& qu,
                              bf16x8& hi, bf16x8& lo) {
  const int q = lane / 16, n = lane % 16;
  f32x4 a0 = {0, 0, 0, 0}, a1 = {0, 0, 0, 0};
#pragma unroll
  for (int kk = 0; kk < DK / 32; ++kk) {
    const bf16x8 b = qu(kk);
    a0 = mma(ku(2 * s, 4 * kk + q), b, a0);
    a1 = mma(ku(2 * s + 1, 4 * kk + q), b, a1);
  }
  const int tq = sigma(t, n), tk = 32 * s + 8 * q;
  const double gq = G[tq];
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float v = (e < 4 ? a0[e & 3] : a1[e & 3]) * (scale * decay_of(gq, G[tk + e]));
    x[e] = tk + e <= tq ? v : 0.0f;
  }
  dasc_wy::split8(x, hi, lo);
}

// four values cut into planes, as half of an operand's eight
template <int N>
__device__ inline void half_planes(f32x4 x, uint2 (&p)[N]) {
  float r[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
  for (int j = 0; j < N; ++j) {
    p[j] = uint2{high_halves(r[0], r[1]), high_halves(r[2], r[3])};
    if (j + 1 < N) {
#pragma unroll
      for (int e = 0; e < 4; ++e) r[e] = rest(r[e]);
    }
  }
}

// Operands that the four waves of a column tile build together: one KB per group of 32 rows and plane,
// lane l's eight values at 16 l, of which tile 2 s holds the first four and tile 2 s + 1 the others.
template <int N>
__device__ inline void put_half(char* base, int t, int lane, const uint2 (&p)[N]) {
#pragma unroll
  for (int j = 0; j < N; ++j)
    *reinterpret_cast<uint2*>(base + ((t / 2) * N + j) * 1024 + lane * 16 + (t % 2) * 8) = p[j];
}
__device__ inline bf16x8 get(const char* base, int index, int lane) {
  return *reinterpret_cast<const bf16x8*>(base + index * 1024 + lane * 16);
}

// The rows of a chunk from row `row` on, of which `left` are left: a buffer resource that ends with
// the last of them
__device__ inline __amdgpu_buffer_rsrc_t chunk_rows(const uint16_t* base, int tok, int width, int64_t row, int left) {
  const int n = left < 0 ? 0 : left < kC ? left : kC;
  return dasc_wy::rsrc(base + row * tok, n ? ((n - 1) * tok + width) * 2 : 0);
}

// A tensor's chunks, or packets, one after another: a resource for each in turn, of `bytes` until the
// last chunk's `tail`, then of nothing.  A pointer that moves on costs a chunk four scalar instructions
// where an address formed anew cost fifteen.
struct Stream {
  const char* at;
  int64_t step;
  int bytes, tail;

  __device__ inline __amdgpu_buffer_rsrc_t next(int c, int last) {
    const __amdgpu_buffer_rsrc_t r = dasc_wy::rsrc(at, c < last ? bytes : c == last ? tail : 0);
    at += step;
    return r;
  }
};

// What a block of either walk works on: a head's request (delta) or segment of one (plain), some columns
struct Walk {
  int cb, h, i, chunks, len;                // chunks < 0: nothing; len: tokens from row0 to the request's end
  int64_t unit, row0, pk0, pk_step;
  bool first, last;                         // it begins with the request's first token, ends with its last

  // where its state comes from and where it goes; LOCAL: what a segment adds to a state of zero
  template <bool DELTA, bool LOCAL>
  __device__ inline const float* start(const ChunkArgs& p, int dk) const {
    const int64_t head = int64_t(dk) * p.a.dv;
    if (LOCAL) return nullptr;
    if (DELTA) return first ? slot_state(p.a, p.a.src, i, h, dk) : p.carry_in + h * head;
    return p.seg_chunks ? p.seg_state + (unit * p.a.H + h) * head : slot_state(p.a, p.a.src, i, h, dk);
  }
  template <bool DELTA, bool LOCAL>
  __device__ inline float* end(const ChunkArgs& p, int dk) const {
    const int64_t head = int64_t(dk) * p.a.dv;
    if (LOCAL) return p.seg_state + (unit * p.a.H + h) * head;
    if (last) return slot_state(p.a, p.a.dst, i, h, dk);
    return DELTA ? p.carry_out + h * head : nullptr;
  }

  // the chunks of a tensor, the last of which ends with the request (or the segment), and the packets
  __device__ inline Stream rows(const uint16_t* base, int tok, int width) const {
    const int left = len - (chunks - 1) * kC, n = left < kC ? left : kC;
    return {reinterpret_cast<const char*>(base + row0 * tok), int64_t(kC) * tok * 2, ((kC - 1) * tok + width) * 2,
            ((n - 1) * tok + width) * 2};
  }
  template <bool PLANES>
  __device__ inline Stream packets(const ChunkArgs& p) const {
    return {p.packets + pk0, pk_step, kPacket<PLANES>, kPacket<PLANES>};
  }
  // this lane's log-decay of chunk c, 0 past the request's end
  __device__ inline float gate(const LinearArgs& a, int c) const {
    const int r = c * kC + int(threadIdx.x % 64);
    const float g = a.io.g[(row0 + (r < len ? r : len - 1)) * a.io.g_tok + h * a.io.g_head];
    return r < len ? g : 0.0f;
  }
};

template <bool DELTA, bool PLANES>
__device__ inline Walk walk_of(const ChunkArgs& p) {
  const LinearArgs& a = p.a;
  Walk w;
  // blocks go round the eight XCDs: those of a head, and heads that share keys, are put on one
  uint32_t bid = blockIdx.x;
  if (gridDim.x % 8 == 0) bid = bid % 8 * (gridDim.x / 8) + bid / 8;
  w.cb = bid % p.col_blocks;
  w.h = bid / p.col_blocks % a.H;
  w.unit = bid / p.col_blocks / a.H;
  w.first = w.last = true;
  Span sp;
  int c0 = 0;
  if (DELTA || p.seg_chunks == 0) {
    w.i = int(w.unit);
    sp = request_span(a, w.i);
    w.chunks = (sp.len + kC - 1) / kC;
    if constexpr (DELTA) {                  // the request's part of the window
      const int64_t u = first_unit(a, w.i, kC);
      const int all = w.chunks;
      c0 = u < p.u0 ? int(p.u0 - u) : 0;
      const int c1 = u + all > p.u1 ? int(p.u1 - u) : all;
      if (u >= p.u1 || (c0 > 0 && c0 >= all)) {
        w.chunks = -1;
        return w;
      }
      w.chunks = c1 - c0;
      w.first = c0 == 0;
      w.last = c1 == all;
    }
  } else {
    const int seg = p.seg_chunks;
    w.i = uniform(p.seg_each ? int(w.unit / p.seg_each) : unit_request(a, w.unit, seg * kC));
    sp = request_span(a, w.i);
    const int64_t j = w.unit - first_segment(p, w.i);
    const int all = (sp.len + kC - 1) / kC;
    if (j < 0 || j >= segments(p, sp.len)) {
      w.chunks = -1;
      return w;
    }
    c0 = int(j) * seg;
    w.chunks = all - c0 < seg || j + 1 == p.seg_each ? all - c0 : seg;
    w.first = j == 0;
    w.last = c0 + w.chunks >= all;
  }
  c0 = uniform(c0);
  w.chunks = uniform(w.chunks);
  w.row0 = uniform(sp.begin + int64_t(c0) * kC);
  w.len = uniform(sp.len - c0 * kC);
  w.pk0 = DELTA ? uniform(((first_unit(a, w.i, kC) + c0 - p.u0) * a.H + w.h) * int64_t(kPacket<PLANES>)) : 0;
  w.pk_step = int64_t(a.H) * kPacket<PLANES>;
  return w;
}

// What only the end of a walk needs is not held in scalar registers over its chunks, which have none to spare
// (with them the walk of a 32-head layer's prompts takes 160 us, without 143): the call's arguments are read
// again from where the kernel found them, and the walk's own numbers wait in vector registers.
__device__ inline ChunkArgs arguments_again() {
  typedef const __attribute__((address_space(4))) uint32_t* Words;
  static_assert(sizeof(ChunkArgs) % 4 == 0);
  uint64_t at = reinterpret_cast<uint64_t>(__builtin_amdgcn_kernarg_segment_ptr());
  asm volatile("" : "+s"(at));
  struct { uint32_t w[sizeof(ChunkArgs) / 4]; } words;
#pragma unroll
  for (uint32_t i = 0; i < sizeof(ChunkArgs) / 4; ++i) words.w[i] = reinterpret_cast<Words>(at)[i];
  return __builtin_bit_cast(ChunkArgs, words);
}

// Whether the join found this tile of 16 columns not to be finite at the request's end: a lane asks for what
// each of its blocks, of 1024 elements of a state, says
__device__ inline int marked(const ChunkArgs& p, int dk, int i, int h, int tile, int lane) {
  const int tiles = p.a.dv / 16, parts = dk * p.a.dv / 1024;
  return lane < parts ? p.seg_bad[((int64_t(i) * p.a.H + h) * parts + lane) * tiles + tile] : 0;
}

struct Kept {
  int i, h, cb, ends;
  int64_t unit;

  __device__ inline explicit Kept(const Walk& w) : i(w.i), h(w.h), cb(w.cb), ends(w.first + 2 * w.last), unit(w.unit) {
    asm volatile("" : "+v"(i), "+v"(h), "+v"(cb), "+v"(ends), "+v"(unit));
  }
  __device__ inline Walk walk() const {
    Walk w{};
    w.i = uniform(i), w.h = uniform(h), w.cb = uniform(cb), w.unit = uniform(unit);
    const int e = uniform(ends);
    w.first = e & 1, w.last = e & 2;
    return w;
  }
};

constexpr int kOutside = int(0x80000000u);  // an offset past the end of any resource

// LDS of a block of CT NG column tiles.  Delta: keys and decays twice, S, Y, e^{G_C - G} U in three
// planes, U in two.  Plain: S in two planes, V, e^{G_C - G} V in three.
template <int DK, int TILES, bool DELTA, bool OUT>
struct Layout {
  static constexpr int kK = kRowsBytes<DK / 8>;
  static constexpr int kKeys = DELTA ? 2 : 1;
  static constexpr int kSPlanes = DELTA ? 3 : OUT ? 2 : 0;
  static constexpr int kVPlanes = OUT ? (DELTA ? 2 : 1) : 0;
  static constexpr int kDecays = DELTA ? 2 : 3;
  static constexpr int kSBytes = DK / 32 * kSPlanes * 1024;
  static constexpr int kS = kKeys * kK;
  static constexpr int kY = kS + TILES * kSBytes;
  static constexpr int kU = kY + TILES * (DELTA ? 6 * 1024 : 0);
  static constexpr int kW = kU + TILES * 6 * 1024;
  static constexpr int kD = kW + TILES * kVPlanes * 2 * 1024;
  static constexpr int kBytes = kD + kDecays * int(sizeof(Decays));
};

// Whether what the next state does not need (Q S, P U, the output) and the staging of keys is done by
// waves of their own, as many again, beside those that carry the state.  us per chunk of the delta rule,
// dk = dv = 128, without | with: 1.94 | 1.70 on 32 heads, 3.37 | 3.00 on 64 (two tiles); dk = dv = 64,
// 4 heads: 1.39 | 1.04.  With two column tiles a wave there are no registers for them.
template <int CT, bool DELTA>
constexpr bool kHelpers = DELTA && CT == 1;
template <int CT, int NG, bool DELTA>
constexpr int kSplitThreads = 256 * NG * (kHelpers<CT, DELTA> ? 2 : 1);

// One block walks one request of a head over 16 CT NG columns.
// Its waves are NG groups of four; a group has CT column tiles, and wave m of it has tokens sigma(m, .)
// of every product over channels and DK / 4 channels of the state.  What the others need of a wave's
// part goes through LDS in operand order.
template <int DK, int CT, int NG, bool DELTA, bool OUT>
__global__ __launch_bounds__((kSplitThreads<CT, NG, DELTA>)) void linear_split_kernel(ChunkArgs p) {
  constexpr bool HELP = kHelpers<CT, DELTA>;
  constexpr int NT = 256 * NG, U = DK / 8, SK = DK / 32, TW = DK / 64, TILES = CT * NG;
  using L = Layout<DK, TILES, DELTA, OUT>;
  __shared__ __attribute__((aligned(16))) char lds[L::kBytes];
  Decays* const dec = reinterpret_cast<Decays*>(lds + L::kD);

  const LinearArgs& a = p.a;
  const int tid = threadIdx.x % NT, wave = uniform(tid / 64), lane = tid % 64, q = lane / 16, n = lane % 16;
  const int m = wave % 4, grp = wave / 4;
  const bool helper = HELP && uniform(int(threadIdx.x / NT)) != 0;
  const Walk w = walk_of<DELTA, true>(p);
  if (w.chunks < 0) return;
  const Kept kept(w);
  const int k_col = key_column<U>(lane);
  const int h = w.h, hk = h / a.rep, dv = a.dv, chunks = w.chunks;

  // the state: lane (q, n) holds channels sigma(TW m + t, 4 q + e) of column n of each column tile
  const int tile0 = grp * CT;               // this group's first column tile in the block
  const int col0 = 16 * (w.cb * TILES + tile0) + n;
  f32x4 S[CT][TW];
  {
    const float* from = helper ? nullptr : w.start<DELTA, false>(p, DK);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int t = 0; t < TW; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          S[ct][t][e] = from && col0 + 16 * ct < dv
                            ? from[int64_t(sigma(TW * m + t, 4 * q + e)) * dv + col0 + 16 * ct] : 0.0f;
  }

  // What a chunk takes from memory is asked for a chunk ahead: keys (staged by all waves), and this
  // wave's queries, values, blocks of T and of P.  Rows come through buffer resources that end with the
  // request's last row of the chunk: what lies past it reads as zero, and stores there are dropped.
  // Every load is issued on every path, so that a wait for one never waits for those behind it.
  constexpr int kRows = NT / U, kPasses = kC / kRows;
  u32x4 rk[kPasses], rd;
  bf16x8 rq[OUT ? SK : 1], rt[DELTA ? 2 : 1][3], rp[2][2];
  uint16_t rv[CT][4];
  float rg = 0;
  const bool deep = m >= 2;                 // a wave of the later tokens has two blocks, (m, 0) and (m, 1)
  const uint16_t* const kb = a.io.k + hk * a.io.k_head;
  const uint16_t* const qb = a.io.q + (OUT ? hk * a.io.q_head : 0);
  const uint16_t* const vb = a.io.v + h * a.io.v_head;
  uint16_t* const ob = a.io.o + (OUT ? h * a.io.o_head : 0);
  const int k_off = (tid / U * p.k_tok + 8 * (tid % U)) * 2;
  const int q_off = (sigma(m, n) * p.q_tok + 8 * q) * 2;
  int v_off[CT], o_off[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const bool in = col0 + 16 * ct < dv;
    v_off[ct] = in ? (sigma(m, 4 * q) * p.v_tok + col0 + 16 * ct) * 2 : kOutside;
    o_off[ct] = in ? (sigma(m, 4 * q) * p.o_tok + col0 + 16 * ct) * 2 : kOutside;
  }
  // a packet: the decays by all waves, this wave's blocks (a wave of the earlier tokens has one, and the
  // other lies outside)
  constexpr int kLast = int(sizeof(Decays)) / 16 - 1;
  const int d_off = (tid < kLast ? tid : kLast) * 16;
  const int b_off[2] = {block_of(m, 0) * 1024 + lane * 16, deep ? block_of(m, 1) * 1024 + lane * 16 : kOutside};
  const int last = chunks - 1;
  Stream ks = w.rows(kb, p.k_tok, DK), qs = w.rows(qb, p.q_tok, DK), vs = w.rows(vb, p.v_tok, dv),
         os = w.rows(ob, p.o_tok, dv), ds = w.packets<true>(p), ts = ds, ps = ds;

  const auto load_k = [&](int c) {
    const __amdgpu_buffer_rsrc_t r = ks.next(c, last);
#pragma unroll
    for (int j = 0; j < kPasses; ++j)
      rk[j] = __builtin_bit_cast(u32x4, dasc_wy::ldf4(r, k_off, j * kRows * p.k_tok * 2));
    if constexpr (DELTA) rd = __builtin_bit_cast(u32x4, dasc_wy::ldf4(ds.next(c, last), d_off, 0));
  };
  const auto put_k = [&](int c) {
    char* K = lds + (DELTA ? (c & 1) * L::kK : 0);
#pragma unroll
    for (int j = 0; j < kPasses; ++j) {
      const int r = j * kRows + tid / U;
      *reinterpret_cast<u32x4*>(K + row_at<U>(r) + tid % U * 16) = rk[j];
    }
    if constexpr (DELTA) {
      if (tid < int(sizeof(Decays)) / 16) reinterpret_cast<u32x4*>(dec + (c & 1))[tid] = rd;
    }
  };
  const auto load_q = [&](int c) {
    if constexpr (OUT) {
      const __amdgpu_buffer_rsrc_t r = qs.next(c, last);
#pragma unroll
      for (int s = 0; s < SK; ++s) rq[s] = __builtin_bit_cast(bf16x8, dasc_wy::ldf4(r, q_off, 64 * s));
    }
  };
  const auto load_v = [&](int c) {
    const __amdgpu_buffer_rsrc_t r = vs.next(c, last);
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
        rv[ct][e] = uint16_t(__builtin_amdgcn_raw_buffer_load_b16(r, v_off[ct], e * p.v_tok * 2, 0));
  };
  const auto load_t = [&](int c) {
    if constexpr (DELTA) {
      const __amdgpu_buffer_rsrc_t r = ts.next(c, last);
#pragma unroll
      for (int j = 0; j < 3; ++j)
#pragma unroll
        for (int s = 0; s < 2; ++s)
          rt[s][j] = __builtin_bit_cast(bf16x8, dasc_wy::ldf4(r, b_off[s], kPacketT + j * kBlocks * 1024));
    }
  };
  const auto load_p = [&](int c) {
    if constexpr (DELTA && OUT) {
      const __amdgpu_buffer_rsrc_t r = ps.next(c, last);
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int s = 0; s < 2; ++s)
          rp[s][j] = __builtin_bit_cast(bf16x8, dasc_wy::ldf4(r, b_off[s], kPacketP + j * kBlocks * 1024));
    }
  };
  const auto put_s = [&]() {                // the state's planes, for all waves of the column tile
    if constexpr (L::kSPlanes > 0) {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int t = 0; t < TW; ++t) {
          uint2 h2[L::kSPlanes];
          half_planes(S[ct][t], h2);
          put_half(lds + L::kS + (tile0 + ct) * L::kSBytes, TW * m + t, lane, h2);
        }
    }
  };
  const auto put_v = [&](const Decays& d) { // plain: the values, and what they add to the state
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      if constexpr (OUT) {
        const uint2 raw[1] = {uint2{rv[ct][0] | uint32_t(rv[ct][1]) << 16, rv[ct][2] | uint32_t(rv[ct][3]) << 16}};
        put_half(lds + L::kW + (tile0 + ct) * 2048, m, lane, raw);
      }
      f32x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(uint32_t(rv[ct][e]) << 16) * d.er[sigma(m, 4 * q + e)];
      uint2 h3[3];
      half_planes(x, h3);
      put_half(lds + L::kU + (tile0 + ct) * 6144, m, lane, h3);
    }
  };

  constexpr int SP = L::kSPlanes ? L::kSPlanes : 1;
  const auto get_s = [&](bf16x8 (&sp)[CT][SK][SP]) {
    if constexpr (L::kSPlanes > 0) {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int s = 0; s < SK; ++s)
#pragma unroll
          for (int j = 0; j < SP; ++j)
            sp[ct][s][j] = get(lds + L::kS + (tile0 + ct) * L::kSBytes, s * SP + j, lane);
    }
  };
  f32x4 O[CT];
  const auto read_out = [&](const bf16x8 (&sp)[CT][SK][SP], const Decays& d) {      // Q S
    if constexpr (OUT) {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) O[ct] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < SK; ++s)
#pragma unroll
        for (int j = 1; j >= 0; --j)
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) O[ct] = mma(rq[s], sp[ct][s][j], O[ct]);
      const f32x4 eo = *reinterpret_cast<const f32x4*>(d.eo + sigma(m, 4 * q));
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) O[ct] *= eo;
    }
  };
  const auto write_out = [&](int c) {       // P U, and the output
    if constexpr (OUT) {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        const char* wb = lds + L::kW + (tile0 + ct) * (DELTA ? 4096 : 2048);
#pragma unroll
        for (int s = 0; s < 2; ++s)
          if (s == 0 || deep) {
            if constexpr (DELTA) {
              const bf16x8 u0 = get(wb, 2 * s, lane), u1 = get(wb, 2 * s + 1, lane);
              O[ct] = mma(rp[s][0], u1, O[ct]);
              O[ct] = mma(rp[s][1], u0, O[ct]);
              O[ct] = mma(rp[s][0], u0, O[ct]);
            } else {
              const bf16x8 v = get(wb, s, lane);
              O[ct] = mma(rp[s][1], v, O[ct]);
              O[ct] = mma(rp[s][0], v, O[ct]);
            }
          }
      }
      settle(O);
      load_p(c + 1);
      const __amdgpu_buffer_rsrc_t ro = os.next(c, last);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
          __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(short, __bf16(O[ct][e])), ro, o_off[ct],
                                                e * p.o_tok * 2, 0);
    }
  };

  // Whether the last state of this group's columns, and of any group's, is finite, for every wave of the block
  int* const verdict = reinterpret_cast<int*>(lds);       // (every wave is past its last read of LDS)
  const auto vote = [&](bool bad) {
    if (!helper && lane == 0) verdict[wave] = bad;
    lds_barrier();
    int mine = 0, all = 0;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const int x = verdict[4 * g] | verdict[4 * g + 1] | verdict[4 * g + 2] | verdict[4 * g + 3];
      all |= x;
      if (g == grp) mine = x;
    }
    if (uniform(all)) {                     // outputs will be written again, by another wave
      stores_done();
      lds_barrier();
    }
    return uniform(mine) != 0;
  };

  if constexpr (HELP) {
    if (helper) {                           // the same barriers as the state's waves, below
      if (chunks > 0) {
        load_k(0);
        load_q(0);
        load_p(0);
        put_k(0);
        load_k(1);
        lds_barrier();
      }
      for (int c = 0; c < chunks; ++c) {
        if constexpr (OUT) {
          bf16x8 sp[CT][SK][SP];
          get_s(sp);
          read_out(sp, dec[c & 1]);
          load_q(c + 1);
        }
        lds_barrier();
        put_k(c + 1);                       // (of nothing after the last chunk)
        load_k(c + 2);
        lds_barrier();
        write_out(c);
        lds_barrier();
      }
      if (kept.walk().last) vote(false);
      return;
    }
  }

  if (chunks > 0) {
    if constexpr (!HELP) {
      load_k(0);
      load_q(0);
    }
    load_v(0);
    load_t(0);
    if constexpr (!HELP) load_p(0);
    if constexpr (!DELTA) {
      if (wave < 2) make_decays(dec[wave], w.gate(a, wave), a.scale, lane);
      rg = w.gate(a, 2);
      lds_barrier();
      put_v(dec[0]);
    }
    if constexpr (!HELP) put_k(0);
    put_s();
    if constexpr (!HELP) load_k(1);
    lds_barrier();
  }

  // Without helpers, what the next state does not need stands behind what it does: a wave does it while
  // it would wait for the others.
  for (int c = 0; c < chunks; ++c) {
    const char* const K = lds + (DELTA ? (c & 1) * L::kK : 0);
    const Decays& d = DELTA ? dec[c & 1] : dec[c % 3];
    const bool more = c + 1 < chunks;
    if constexpr (!DELTA) {
      load_v(c + 1);
      if (wave == 0) make_decays(dec[(c + 2) % 3], rg, a.scale, lane);    // (it has one block of P, others two)
      rg = w.gate(a, c + 3);
    }
    bf16x8 sp[CT][SK][SP];
    get_s(sp);
    if constexpr (DELTA) {
      f32x4 X[CT];
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) X[ct] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < SK; ++s) {
        const bf16x8 k = sigma_unit<U>(K, m, n, 4 * s + q);
#pragma unroll
        for (int j = 2; j >= 0; --j)
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) X[ct] = mma(k, sp[ct][s][j], X[ct]);
      }
      const f32x4 ex = *reinterpret_cast<const f32x4*>(d.e + sigma(m, 4 * q));
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = fmaf(-ex[e], X[ct][e], __uint_as_float(uint32_t(rv[ct][e]) << 16));
        uint2 h3[3];
        half_planes(y, h3);
        put_half(lds + L::kY + (tile0 + ct) * 6144, m, lane, h3);
      }
      load_v(c + 1);
      if constexpr (!HELP) {
        read_out(sp, d);
        load_q(c + 1);
      }
      lds_barrier();                        // Y is whole
      const f32x4 er = *reinterpret_cast<const f32x4*>(d.er + sigma(m, 4 * q));
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        f32x4 u = {0, 0, 0, 0};
        const char* yb = lds + L::kY + (tile0 + ct) * 6144;
#pragma unroll
        for (int s = 0; s < 2; ++s)
          if (s == 0 || deep) {
            const bf16x8 y0 = get(yb, 3 * s, lane), y1 = get(yb, 3 * s + 1, lane), y2 = get(yb, 3 * s + 2, lane);
            u = mma(rt[s][2], y0, u);
            u = mma(rt[s][0], y2, u);
            u = mma(rt[s][1], y1, u);
            u = mma(rt[s][1], y0, u);
            u = mma(rt[s][0], y1, u);
            u = mma(rt[s][0], y0, u);
          }
        settle(u);
        uint2 h3[3];
        half_planes(u * er, h3);
        put_half(lds + L::kU + (tile0 + ct) * 6144, m, lane, h3);
        if constexpr (OUT) {
          uint2 h2[2];
          half_planes(u, h2);
          put_half(lds + L::kW + (tile0 + ct) * 4096, m, lane, h2);
        }
      }
      load_t(c + 1);
      lds_barrier();                        // U is whole
    } else if constexpr (OUT) {
      read_out(sp, d);
#pragma unroll
      for (int s = 0; s < 2; ++s)
        if (s == 0 || deep)
          make_p<DK>(d.G, a.scale, m, s, lane, [&](int x, int u) { return sigma_unit<U>(K, x, n, u); },
                     [&](int kk) { return rq[kk]; }, rp[s][0], rp[s][1]);
      load_q(c + 1);
    }

    // the state
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) decay_state(S[ct], d);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int t = 0; t < TW; ++t) {
        const int tt = TW * m + t;
        const bf16x8 k = columns<kStride<U> * 16>(K + k_col, 32 * s, 64 * (tt / 2) + 8 * (tt % 2));
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          const char* ub = lds + L::kU + (tile0 + ct) * 6144;
          S[ct][t] = mma(k, get(ub, 3 * s + 2, lane), S[ct][t]);
          S[ct][t] = mma(k, get(ub, 3 * s + 1, lane), S[ct][t]);
          S[ct][t] = mma(k, get(ub, 3 * s, lane), S[ct][t]);
        }
      }
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) settle(S[ct]);
    if constexpr (HELP) {
      put_s();                              // (for nobody after the last chunk)
    } else if constexpr (DELTA) {
      if (more) {
        put_s();
        put_k(c + 1);
      }
      load_k(c + 2);
    }
    if constexpr (!HELP) write_out(c);
    if constexpr (!DELTA) {
      if (more) {
        lds_barrier();                      // everybody is done with this chunk
        put_v(dec[(c + 1) % 3]);
        put_k(c + 1);
        put_s();
        load_k(c + 2);
      }
    }
    lds_barrier();                          // the next chunk's keys and state are whole
  }

  const ChunkArgs pe = arguments_again();
  const Walk we = kept.walk();
  if (we.last) {
    bool bad = false;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) bad |= !finite(S[ct]);
    if (vote(__any(bad))) {
      const int tile = we.cb * TILES + tile0 + m;
      if (m < CT && 16 * tile < pe.a.dv) walk_tokens<DK, 16, DELTA, OUT>(pe.a, we.i, we.h, 16 * tile, lane);
      return;
    }
  }
  float* to = we.end<DELTA, false>(pe, DK);
  if (to) {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
      if (col0 + 16 * ct < pe.a.dv) {
#pragma unroll
        for (int t = 0; t < TW; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            to[int64_t(sigma(TW * m + t, 4 * q + e)) * pe.a.dv + col0 + 16 * ct] = S[ct][t][e];
      }
  }
}

// ---- a wave per 16 columns ------------------------------------------------------------------------

template <int DK, int TILES, bool DELTA, bool OUT>
struct ColumnLayout {
  static constexpr int kRow = kRowsBytes<DK / 8>;
  static constexpr int kV = kRow * (OUT ? 2 : 1);
  static constexpr int kP = kV + kC * kVStride<2 * TILES> * 16;
  static constexpr int kT = kP + (OUT ? kPBytes : 0);
  static constexpr int kD = kT + (DELTA ? kTBytes : 0);
  static constexpr int kBytes = kD + int(sizeof(Decays)) * (DELTA ? 1 : 2);
};

// waves of a SIMD that the registers are to leave room for
template <int CT, bool DELTA, bool OUT>
constexpr int kWavesPerSimd = CT == 1 && !DELTA && !OUT ? 4 : 2;

// One block walks one request (delta) or one segment of one (plain) of a head over 16 CT NW columns, a wave
// on 16 CT.  A wave has the whole state of its columns and needs nothing of another's: K, Q, V, P and T lie
// in LDS for all of them.
// LOCAL: only what the segment adds to a state of zero, left in seg_state for the join.
template <int DK, int CT, int NW, bool DELTA, bool OUT, bool LOCAL>
__global__ __launch_bounds__(64 * NW, (kWavesPerSimd<CT, DELTA, OUT>)) void linear_columns_kernel(ChunkArgs p) {
  constexpr int NT = 64 * NW, KT = DK / 16, U = DK / 8, UV = 2 * CT * NW;
  using L = ColumnLayout<DK, CT * NW, DELTA, OUT>;
  __shared__ __attribute__((aligned(16))) char lds[L::kBytes];
  char* const K = lds;
  char* const Q = lds + L::kRow;
  char* const V = lds + L::kV;
  char* const P = lds + L::kP;
  char* const T = lds + L::kT;
  Decays* const dec = reinterpret_cast<Decays*>(lds + L::kD);

  const LinearArgs& a = p.a;
  const int tid = threadIdx.x, wave = uniform(tid / 64), lane = tid % 64, q = lane / 16, n = lane % 16;
  const Walk w = walk_of<DELTA, false>(p);
  if (w.chunks < 0) return;
  const Kept kept(w);
  const int k_col = key_column<U>(lane), v_col = value_column<UV>(lane);
  const int h = w.h, hk = h / a.rep, dv = a.dv, chunks = w.chunks;

  // the state: lane (q, n) holds channels sigma(t, 4 q + i) of column n of each tile
  const int tile0 = CT * (w.cb * NW + wave), col = 16 * tile0 + n;
  f32x4 S[CT][KT];
  {
    const float* from = w.start<DELTA, LOCAL>(p, DK);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          S[ct][t][e] = from && col + 16 * ct < dv
                            ? from[int64_t(sigma(t, 4 * q + e)) * dv + col + 16 * ct] : 0.0f;
  }

  // What a chunk takes from memory goes through registers a chunk ahead: 16-byte units of K, Q and V
  // rows and of the packet.  Rows come through buffer resources that end with the request's last row of
  // the chunk; what lies past it reads as zero.
  constexpr int kRowsPass = NT / U, kPasses = kC / kRowsPass;
  constexpr int kVRows = NT / UV, kVPasses = kC / kVRows;
  constexpr int kT = DELTA ? (kBlocks * 64 + NT - 1) / NT : 0;   // a lane's eight values of a block of T each
  u32x4 rk[kPasses], rq[OUT ? kPasses : 1], rv[kVPasses], rd;
  float rt[kT ? kT : 1][8];
  float rg = 0;
  const uint16_t* const kb = a.io.k + hk * a.io.k_head;
  const uint16_t* const qb = a.io.q + (OUT ? hk * a.io.q_head : 0);
  const uint16_t* const vb = a.io.v + h * a.io.v_head;
  uint16_t* const ob = a.io.o + (OUT ? h * a.io.o_head : 0);
  const int vcol = 16 * CT * NW * w.cb + 8 * (tid % UV);
  const int k_off = (tid / U * p.k_tok + 8 * (tid % U)) * 2;
  const int q_off = (tid / U * p.q_tok + 8 * (tid % U)) * 2;
  const int v_off = vcol < dv ? (tid / UV * p.v_tok + vcol) * 2 : kOutside;
  // columns that the join has marked: the request's first segment takes them by token
  bool left[CT];
  int o_off[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const bool in = col + 16 * ct < dv;
    left[ct] = !DELTA && OUT && p.seg_chunks && 16 * (tile0 + ct) < dv &&
               __any(marked(p, DK, w.i, h, tile0 + ct, lane));
    o_off[ct] = in && !left[ct] ? (8 * q * p.o_tok + col + 16 * ct) * 2 : kOutside;
  }
  const int last = chunks - 1;
  Stream ks = w.rows(kb, p.k_tok, DK), qs = w.rows(qb, p.q_tok, DK), vs = w.rows(vb, p.v_tok, dv),
         os = w.rows(ob, p.o_tok, dv), ps = w.packets<false>(p);
  const auto load = [&](int c) {
    const __amdgpu_buffer_rsrc_t k = ks.next(c, last), v = vs.next(c, last);
#pragma unroll
    for (int j = 0; j < kPasses; ++j)
      rk[j] = __builtin_bit_cast(u32x4, dasc_wy::ldf4(k, k_off, j * kRowsPass * p.k_tok * 2));
    if constexpr (OUT) {
      const __amdgpu_buffer_rsrc_t x = qs.next(c, last);
#pragma unroll
      for (int j = 0; j < kPasses; ++j)
        rq[j] = __builtin_bit_cast(u32x4, dasc_wy::ldf4(x, q_off, j * kRowsPass * p.q_tok * 2));
    }
#pragma unroll
    for (int j = 0; j < kVPasses; ++j)
      rv[j] = __builtin_bit_cast(u32x4, dasc_wy::ldf4(v, v_off, j * kVRows * p.v_tok * 2));
    if constexpr (DELTA) {
      const __amdgpu_buffer_rsrc_t r = ps.next(c, last);
      rd = __builtin_bit_cast(u32x4, dasc_wy::ldf4(r, tid < int(sizeof(Decays)) / 16 ? tid * 16 : kOutside, 0));
#pragma unroll
      for (int j = 0; j < kT; ++j) {
        const int x = j * NT + tid, off = x < kBlocks * 64 ? x * 16 : kOutside;
        const f32x4 lo = dasc_wy::ldf4(r, off, kPacketT), hi = dasc_wy::ldf4(r, off, kPacketT + kBlocks * 1024);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          rt[j][e] = lo[e];
          rt[j][4 + e] = hi[e];
        }
      }
    } else {
      rg = w.gate(a, c + 1);
    }
  };
  const auto stage = [&]() {
#pragma unroll
    for (int j = 0; j < kPasses; ++j) {
      const int r = j * kRowsPass + tid / U, at = row_at<U>(r) + tid % U * 16;
      *reinterpret_cast<u32x4*>(K + at) = rk[j];
      if (OUT) *reinterpret_cast<u32x4*>(Q + at) = rq[j];
    }
#pragma unroll
    for (int j = 0; j < kVPasses; ++j) {
      const int r = j * kVRows + tid / UV;
      *reinterpret_cast<u32x4*>(V + (r * kVStride<UV> + tid % UV) * 16) = rv[j];
    }
    if constexpr (DELTA) {
      if (tid < int(sizeof(Decays)) / 16) reinterpret_cast<u32x4*>(dec)[tid] = rd;
#pragma unroll
      for (int j = 0; j < kT; ++j) {
        const int x = j * NT + tid;
        bf16x8 t[3];
        planes<3>(rt[j], t);
        if (x < kBlocks * 64) {
#pragma unroll
          for (int y = 0; y < 3; ++y) *reinterpret_cast<bf16x8*>(T + y * kBlocks * 1024 + x * 16) = t[y];
        }
      }
    }
  };

  double log2_sum = 0;                      // LOCAL: the segment's decay
  if (chunks > 0) {
    load(0);
    if constexpr (!DELTA) {
      if (wave == NW - 1) make_decays(dec[0], w.gate(a, 0), a.scale, lane);
    }
    stage();
  }
  lds_barrier();

  for (int c = 0; c < chunks; ++c) {
    const Decays& d = DELTA ? dec[0] : dec[c & 1];
    const float g_next = rg;
    load(c + 1);
    if constexpr (OUT) {
      for (int b = wave; b < kBlocks; b += NW) {
        const int t = b < 2 ? b : 2 + (b - 2) / 2, s = b < 2 ? 0 : (b - 2) % 2;
        bf16x8 hi, lo;
        make_p<DK>(d.G, a.scale, t, s, lane, [&](int x, int u) { return sigma_unit<U>(K, x, n, u); },
                   [&](int kk) { return sigma_unit<U>(Q, t, n, 4 * kk + q); }, hi, lo);
        char* at = P + b * 1024 + lane * 16;
        *reinterpret_cast<bf16x8*>(at) = hi;
        *reinterpret_cast<bf16x8*>(at + kBlocks * 1024) = lo;
      }
    }
    if constexpr (!DELTA) {
      if (wave == NW - 1) make_decays(dec[(c + 1) & 1], g_next, a.scale, lane);
    }
    f32x4 O[CT][4], X[CT][4];
    bf16x8 v[CT][2];
    // what needs the state: Q S, K S
    if constexpr (OUT || DELTA) {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int t = 0; t < 4; ++t) O[ct][t] = X[ct][t] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < DK / 32; ++s) {
        bf16x8 b[CT][3];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) planes<3>(S[ct][2 * s], S[ct][2 * s + 1], b[ct]);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          if constexpr (DELTA) {
            const bf16x8 k = sigma_unit<U>(K, t, n, 4 * s + q);
#pragma unroll
            for (int j = 2; j >= 0; --j)
#pragma unroll
              for (int ct = 0; ct < CT; ++ct) X[ct][t] = mma(k, b[ct][j], X[ct][t]);
          }
          if constexpr (OUT) {
            const bf16x8 x = sigma_unit<U>(Q, t, n, 4 * s + q);
#pragma unroll
            for (int j = 1; j >= 0; --j)
#pragma unroll
              for (int ct = 0; ct < CT; ++ct) O[ct][t] = mma(x, b[ct][j], O[ct][t]);
          }
        }
      }
    }
    if constexpr (OUT) lds_barrier();       // P is whole
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int s = 0; s < 2; ++s) v[ct][s] = columns<kVStride<UV> * 16>(V + v_col, 32 * s, 32 * (wave * CT + ct));

    f32x4 Uf[CT][4];                        // U in fp32
    if constexpr (DELTA) {
      bf16x8 y[CT][2][3];
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          float x[8];
          widen8(v[ct][s], x);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            x[e] = fmaf(-d.e[32 * s + 8 * q + e], X[ct][2 * s + e / 4][e % 4], x[e]);
          planes<3>(x, y[ct][s]);
        }
#pragma unroll
      for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) Uf[ct][t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s <= t / 2; ++s) {
          const char* b = T + block_of(t, s) * 1024 + lane * 16;
          const bf16x8 t0 = *reinterpret_cast<const bf16x8*>(b);
          const bf16x8 t1 = *reinterpret_cast<const bf16x8*>(b + kBlocks * 1024);
          const bf16x8 t2 = *reinterpret_cast<const bf16x8*>(b + 2 * kBlocks * 1024);
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            f32x4 u = Uf[ct][t];
            u = mma(t2, y[ct][s][0], u);
            u = mma(t0, y[ct][s][2], u);
            u = mma(t1, y[ct][s][1], u);
            u = mma(t1, y[ct][s][0], u);
            u = mma(t0, y[ct][s][1], u);
            Uf[ct][t] = mma(t0, y[ct][s][0], u);
          }
        }
      }
    }

    if constexpr (OUT) {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const f32x4 eo = *reinterpret_cast<const f32x4*>(d.eo + sigma(t, 4 * q));
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) O[ct][t] *= eo;
      }
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        bf16x8 u[CT][2];
        if constexpr (DELTA) {
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) planes<2>(Uf[ct][2 * s], Uf[ct][2 * s + 1], u[ct]);
        }
#pragma unroll
        for (int t = 2 * s; t < 4; ++t) {
          const char* b = P + block_of(t, s) * 1024 + lane * 16;
          const bf16x8 p0 = *reinterpret_cast<const bf16x8*>(b);
          const bf16x8 p1 = *reinterpret_cast<const bf16x8*>(b + kBlocks * 1024);
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            if constexpr (DELTA) {
              O[ct][t] = mma(p0, u[ct][1], O[ct][t]);
              O[ct][t] = mma(p1, u[ct][0], O[ct][t]);
              O[ct][t] = mma(p0, u[ct][0], O[ct][t]);
            } else {
              O[ct][t] = mma(p1, v[ct][s], O[ct][t]);
              O[ct][t] = mma(p0, v[ct][s], O[ct][t]);
            }
          }
        }
      }
      const __amdgpu_buffer_rsrc_t ro = os.next(c, last);
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int ct = 0; ct < CT; ++ct)
            __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(short, __bf16(O[ct][t][e])), ro, o_off[ct],
                                                  (32 * (t / 2) + 4 * (t % 2) + e) * p.o_tok * 2, 0);
    }

    // the state
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) decay_state(S[ct], d);
    // (what a chunk has cleared no later growth brings back)
    if constexpr (LOCAL) log2_sum = d.G[kC - 1] < -1000.0 ? -1e30 : log2_sum + d.G[kC - 1];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      bf16x8 u[CT][3];
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        float x[8];
        if constexpr (!DELTA) widen8(v[ct][s], x);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          x[e] = (DELTA ? Uf[ct][2 * s + e / 4][e % 4] : x[e]) * d.er[32 * s + 8 * q + e];
        planes<3>(x, u[ct]);
      }
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        const bf16x8 k = columns<kStride<U> * 16>(K + k_col, 32 * s, 64 * (t / 2) + 8 * (t % 2));
#pragma unroll
        for (int j = 2; j >= 0; --j)
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) S[ct][t] = mma(k, u[ct][j], S[ct][t]);
      }
    }
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) settle(S[ct]);
    lds_barrier();                          // everybody is done with this chunk
    if (c + 1 < chunks) {
      stage();
      lds_barrier();
    }
  }

  const ChunkArgs pe = arguments_again();
  const Walk we = kept.walk();
  if (LOCAL && tid == 0 && we.cb == 0) pe.seg_log2[we.unit * pe.a.H + we.h] = log2_sum;
  float* to = we.end<DELTA, LOCAL>(pe, DK);
  const bool segment = !DELTA && pe.seg_chunks;
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    if (!LOCAL && !segment && we.last) left[ct] = __any(!finite(S[ct])) && 16 * (tile0 + ct) < pe.a.dv;
    if (left[ct]) {
      if (!segment || we.first) {
        stores_done();
        walk_tokens<DK, 16, DELTA, OUT>(pe.a, we.i, we.h, 16 * (tile0 + ct), lane);
      }
    } else if (to && col + 16 * ct < pe.a.dv) {
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) to[int64_t(sigma(t, 4 * q + e)) * pe.a.dv + col + 16 * ct] = S[ct][t][e];
    }
  }
}

// ---- plain rule: the segments of a request joined ------------------------------------------------------

// Segment j's start: its own from the request's first state, and what the segments before it add.
// Replaces the segments' sums by their starts; with no output to come (finish), leaves the last state in
// place of the first segment's sum.  Marks the columns whose last state is not finite: those the request's
// first segment takes token by token and the others leave out, or linear_finish_kernel does.
constexpr int kAhead = 8;

__global__ __launch_bounds__(256) void linear_join_kernel(ChunkArgs p, int dk, bool finish) {
  __shared__ int bad[16];
  const LinearArgs& a = p.a;
  const int64_t per = int64_t(dk) * a.dv;                              // a multiple of 1024
  const int64_t x = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 4;
  const int h = blockIdx.y, i = blockIdx.z;
  const int segs = segments(p, request_span(a, i).len);
  const int64_t u0 = first_segment(p, i);
  const float* from = slot_state(a, a.src, i, h, dk);
  f32x4 S[1] = {from ? *reinterpret_cast<const f32x4*>(from + x) : f32x4{0, 0, 0, 0}};
  const auto at = [&](int j) { return reinterpret_cast<f32x4*>(p.seg_state + ((u0 + j) * a.H + h) * per + x); };
  for (int j0 = 0; j0 < segs; j0 += kAhead) {       // what kAhead segments add, asked for together
    f32x4 add[kAhead];
    double end[kAhead];
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      const int j = j0 + e < segs ? j0 + e : segs - 1;
      add[e] = *at(j);
      end[e] = p.seg_log2[(u0 + j) * a.H + h];
    }
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      const int j = j0 + e;
      if (j >= segs) break;
      if (!finish) *at(j) = S[0];
      if (end[e] > -0.72) {
        const float m = expm1f(float(end[e] * 0.6931471805599453));
#pragma unroll
        for (int i = 0; i < 4; ++i) S[0][i] = fmaf(S[0][i], m, S[0][i]) + add[e][i];
      } else {
        S[0] = S[0] * dasc_wy::ex2(float(end[e])) + add[e];
      }
    }
  }
  if (finish) *at(0) = S[0];
  if (threadIdx.x < 16) bad[threadIdx.x] = 0;
  __syncthreads();
  if (!finite(S)) bad[x % a.dv / 16] = 1;
  __syncthreads();
  const int tiles = a.dv / 16;
  if (threadIdx.x < tiles)
    p.seg_bad[((int64_t(i) * a.H + h) * gridDim.x + blockIdx.x) * tiles + threadIdx.x] = bad[threadIdx.x];
}

// States alone: the last state from where the join left it, 16 columns a block; or token by token
template <int DK>
__global__ __launch_bounds__(4 * DK) void linear_finish_kernel(ChunkArgs p) {
  const LinearArgs& a = p.a;
  const int tiles = a.dv / 16, tile = blockIdx.x % tiles, h = blockIdx.x / tiles % a.H, i = blockIdx.x / tiles / a.H;
  if (__syncthreads_or(marked(p, DK, i, h, tile, threadIdx.x))) {
    if (threadIdx.x < 64) walk_tokens<DK, 16, false, false>(a, i, h, 16 * tile, threadIdx.x);
    return;
  }
  float* to = slot_state(a, a.dst, i, h, DK);
  if (!to) return;
  const int64_t x = threadIdx.x / 4 * a.dv + 16 * tile + threadIdx.x % 4 * 4;
  const float* S = p.seg_state + (first_segment(p, i) * a.H + h) * int64_t(DK) * a.dv;
  *reinterpret_cast<f32x4*>(to + x) = *reinterpret_cast<const f32x4*>(S + x);
}

// ---- delta rule: T, P and the decays of every chunk -----------------------------------------------------

constexpr int kTS = 68;                     // floats from row to row of a 64 x 64 matrix in LDS

// 16 x 16 blocks of a matrix in LDS on fp32 matrix instructions: c + x y
__device__ inline f32x4 block_mul(const float* x, const float* y, f32x4 c, int lane) {
  const int q = lane / 16, r = lane % 16;
#pragma unroll
  for (int k = 0; k < 4; ++k) c = mma32(x[r * kTS + 4 * k + q], y[(4 * k + q) * kTS + r], c);
  return c;
}
__device__ inline void block_put(float* x, f32x4 v, int lane) {
#pragma unroll
  for (int e = 0; e < 4; ++e) x[(4 * (lane / 16) + e) * kTS + lane % 16] = v[e];
}

// A wave per chunk and head, four of a block's waves on heads side by side, none waiting for another.
// For the split walk it is bound by the packets it writes: 128 chunks of 32 heads, 217 MB in 52 us, 4.2 TB/s.
// A and P have the same decays: both are formed transposed, block (t, s) at a time, whose lane (q, n)
// holds columns 32 s + 8 q .. + 7 of row sigma(t, n).  A is inverted in place in LDS, in fp32: the
// diagonal 16 x 16 blocks by substitution, a column per lane, all four at once; then the blocks (1, 0)
// and (3, 2); then the lower left 32 x 32.
template <int DK, bool OUT, bool PLANES>
__global__ __launch_bounds__(256) void linear_factor_kernel(ChunkArgs p, int64_t total) {
  constexpr int NW = 4, SK = DK / 32;
  constexpr bool kP = OUT && PLANES;
  struct Own {
    float A[kC * kTS];
    Decays d;
    float beta[kC];
  };
  __shared__ __attribute__((aligned(16))) Own own[NW];
  const LinearArgs& a = p.a;
  const int wave = uniform(int(threadIdx.x / 64)), lane = threadIdx.x % 64, q = lane / 16, n = lane % 16;
  const int64_t job = int64_t(blockIdx.x) * NW + wave;
  if (job >= total) return;
  const int h = int(job % a.H), hk = h / a.rep;
  const int64_t unit = p.u0 + job / a.H;
  const int i = uniform(unit_request(a, unit, kC));
  const Span sp = request_span(a, i);
  const int64_t c = unit - first_unit(a, i, kC);
  if (c < 0 || c * kC >= sp.len) return;
  const int64_t row0 = uniform(sp.begin + c * kC);
  const int len = uniform(sp.len - int(c) * kC);   // tokens from row0 to the request's end
  float* const A = own[wave].A;
  Decays& d = own[wave].d;
  float* const beta = own[wave].beta;
  char* const pk = p.packets + uniform(job * int64_t(kPacket<PLANES>));

  const __amdgpu_buffer_rsrc_t rk = chunk_rows(a.io.k + hk * a.io.k_head, p.k_tok, DK, row0, len);
  bf16x8 k[4][SK];
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int s = 0; s < SK; ++s)
      k[t][s] = __builtin_bit_cast(bf16x8, dasc_wy::ldf4(rk, (sigma(0, n) * p.k_tok + 8 * q) * 2,
                                                         (sigma(t, 0) * p.k_tok + 32 * s) * 2));
  {
    const int64_t r = row0 + (lane < len ? lane : len - 1);
    const float b = a.io.beta[r * a.io.beta_tok + h * a.io.beta_head];
    const float g = a.io.g[r * a.io.g_tok + h * a.io.g_head];
    beta[lane] = lane < len ? b : 0.0f;
    make_decays(d, lane < len ? g : 0.0f, a.scale, lane);
  }
  dasc_wy::wave_lds_sync();

#pragma unroll
  for (int t = 0; t < 4; ++t) {
    bf16x8 x[SK];
    if constexpr (kP) {
      const __amdgpu_buffer_rsrc_t rq = chunk_rows(a.io.q + hk * a.io.q_head, p.q_tok, DK, row0, len);
#pragma unroll
      for (int s = 0; s < SK; ++s)
        x[s] = __builtin_bit_cast(bf16x8, dasc_wy::ldf4(rq, (sigma(0, n) * p.q_tok + 8 * q) * 2,
                                                        (sigma(t, 0) * p.q_tok + 32 * s) * 2));
    }
    const int r = sigma(t, n);
    const double gr = d.G[r];
    const float br = beta[r];
#pragma unroll
    for (int s = 0; s <= t / 2; ++s) {
      f32x4 y[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}}, z[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
      for (int kk = 0; kk < SK; ++kk)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          y[j] = mma(k[2 * s + j][kk], k[t][kk], y[j]);
          if constexpr (kP) z[j] = mma(k[2 * s + j][kk], x[kk], z[j]);
        }
      const int c0 = 32 * s + 8 * q;
      float Pf[8];
      f32x4 Af[2];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float D = decay_of(gr, d.G[c0 + e]);
        Af[e / 4][e % 4] = c0 + e < r ? br * D * y[e / 4][e % 4] : 0.0f;
        if constexpr (kP) Pf[e] = c0 + e <= r ? a.scale * D * z[e / 4][e % 4] : 0.0f;
      }
      *reinterpret_cast<f32x4*>(A + r * kTS + c0) = Af[0];
      *reinterpret_cast<f32x4*>(A + r * kTS + c0 + 4) = Af[1];
      if constexpr (kP) {
        bf16x8 hi, lo;
        dasc_wy::split8(Pf, hi, lo);
        char* at = pk + kPacketP + block_of(t, s) * 1024 + lane * 16;
        *reinterpret_cast<bf16x8*>(at) = hi;
        *reinterpret_cast<bf16x8*>(at + kBlocks * 1024) = lo;
      }
    }
  }
  dasc_wy::wave_lds_sync();

  const auto block = [&](int x, int y) { return A + 16 * x * kTS + 16 * y; };
  const f32x4 zero = {0, 0, 0, 0};
  {
    float* const D = block(q, q);           // this lane: column n of diagonal block q
    float x[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float s[4] = {r == n ? 1.0f : 0.0f, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < r; ++j) s[j % 4] = fmaf(-D[r * kTS + j], x[j], s[j % 4]);
      x[r] = (s[0] + s[1]) + (s[2] + s[3]);
    }
    dasc_wy::wave_lds_sync();
#pragma unroll
    for (int r = 0; r < 16; ++r) D[r * kTS + n] = x[r];
  }
  dasc_wy::wave_lds_sync();
  {
    const f32x4 x = block_mul(block(1, 0), block(0, 0), zero, lane), y = block_mul(block(3, 2), block(2, 2), zero, lane);
    dasc_wy::wave_lds_sync();
    block_put(block(1, 0), -x, lane);
    block_put(block(3, 2), -y, lane);
    dasc_wy::wave_lds_sync();
    const f32x4 u = block_mul(block(1, 1), block(1, 0), zero, lane), v = block_mul(block(3, 3), block(3, 2), zero, lane);
    dasc_wy::wave_lds_sync();
    block_put(block(1, 0), u, lane);
    block_put(block(3, 2), v, lane);
    dasc_wy::wave_lds_sync();
  }
  {
    f32x4 x[2][2], y[2][2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      x[r][0] = block_mul(block(2 + r, 1), block(1, 0), block_mul(block(2 + r, 0), block(0, 0), zero, lane), lane);
      x[r][1] = block_mul(block(2 + r, 1), block(1, 1), zero, lane);
    }
    dasc_wy::wave_lds_sync();
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int j = 0; j < 2; ++j) block_put(block(2 + r, j), -x[r][j], lane);
    dasc_wy::wave_lds_sync();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      y[0][j] = block_mul(block(2, 2), block(2, j), zero, lane);
      y[1][j] = block_mul(block(3, 3), block(3, j), block_mul(block(3, 2), block(2, j), zero, lane), lane);
    }
    dasc_wy::wave_lds_sync();
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int j = 0; j < 2; ++j) block_put(block(2 + r, j), y[r][j], lane);
    dasc_wy::wave_lds_sync();
  }

#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int s = 0; s <= t / 2; ++s) {
      const int c0 = 32 * s + 8 * q;
      const float* row = A + sigma(t, n) * kTS + c0;
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = row[e] * beta[c0 + e];
      if constexpr (PLANES) {
        bf16x8 pl[3];
        planes<3>(x, pl);
#pragma unroll
        for (int j = 0; j < 3; ++j)
          *reinterpret_cast<bf16x8*>(pk + kPacketT + (j * kBlocks + block_of(t, s)) * 1024 + lane * 16) = pl[j];
      } else {
        f32x4* f = reinterpret_cast<f32x4*>(pk + kPacketT) + block_of(t, s) * 64 + lane;
        f[0] = f32x4{x[0], x[1], x[2], x[3]};
        f[kBlocks * 64] = f32x4{x[4], x[5], x[6], x[7]};
      }
    }
  for (int b = lane; b < int(sizeof(Decays)) / 16; b += 64)
    reinterpret_cast<u32x4*>(pk)[b] = reinterpret_cast<const u32x4*>(&d)[b];
}

// ---- launches --------------------------------------------------------------------------------------------

int64_t units_of(const ChunkPlan& c, int64_t tokens) { return c.n_tokens / tokens + c.n_req; }

constexpr int kCus = 256;                   // blocks that give every CU one

// columns that the walk with a wave per 16 takes in a block
constexpr int whole_tiles(int dk) { return dk == 64 ? 4 : 8; }

struct Segments {
  int chunks, each;                         // of a segment, 0: requests are not split; ChunkArgs::seg_each
  int64_t units;
};

// Segments of the plain rule's requests, for a block per CU at most: a block more on some CUs makes all
// wait (two share a CU's matrix units: 9.4 us per chunk against 4.7).  Equal numbers for every request
// suit requests alike, numbers by length suit others; the shorter segments are taken.  A split request
// costs 3.2 + 5.6 us per chunk of a segment and some 20 us for two launches more and the join, one that
// is not 1.8 (32 heads or fewer) or 2.7 us (64) per chunk.  us, split | whole:
//     dk = dv = 128:  4096 tokens x 32 heads  82 | 117    1536 x 32  46 | 48    1024 x 32  40 | 34
//                     16384 x 4  57 | 405     1024 x 4    24 | 30     640 x 4   22 | 21
//                     2 of 2048 x 32  79 | 86
//     dk = dv = 64:   4096 x 16  34 | 91      2048 x 16   25 | 48     1024 x 16  21 | 26
// The states of 64 segments are joined one after another in 17 us, hence no more.
constexpr int kMaxSegments = 64;

// Segments, a head's blocks each, that the chip has CUs for; no more are ever made
int64_t segment_room(const ChunkPlan& c) {
  const int64_t cols = 16 * whole_tiles(c.dk);
  return kCus / (c.H * ((c.dv + cols - 1) / cols));
}

int64_t longest(const ChunkPlan& c) {       // chunks of the longest request
  return ((c.max_len < c.n_tokens ? c.max_len : c.n_tokens) + kC - 1) / kC;
}

// Whether splitting pays for a request of `all` chunks in segments of `seg`, and for any of this length
bool split_pays(int64_t all, int64_t seg) { return 2 * all >= 5 * seg + 23; }
bool may_split(const ChunkPlan& c) { return !c.delta && segment_room(c) >= 2 && split_pays(longest(c), 1); }

Segments segments_of(const ChunkPlan& c) {
  const int64_t room = segment_room(c), all = longest(c);
  if (!may_split(c)) return {};
  const int64_t each = room / c.n_req;      // segments of every request, or numbers by length
  int64_t seg = each > 0 ? (all + each - 1) / each : all;
  const int64_t by_length = room > c.n_req ? c.n_tokens / kC / (room - c.n_req) + 1 : all;
  const bool alike = seg <= by_length;
  if (!alike) seg = by_length;
  if (seg < (all + kMaxSegments - 1) / kMaxSegments) seg = (all + kMaxSegments - 1) / kMaxSegments;
  if (!split_pays(all, seg)) return {};
  const int64_t n = (all + seg - 1) / seg;
  return {int(seg), alike ? int(n) : 0, alike ? n * c.n_req : units_of(c, seg * kC)};
}

// Column tiles of 16 that a block takes: the fewest that keep the blocks at one per CU, because a chunk
// takes a block the less time the fewer it has (four waves on one tile share a chunk's state; eight waves
// of a tile each share its keys).  us per chunk of 64 tokens, dk = dv = 128, delta rule, by heads:
//     heads              32     64    128    256
//     1 tile (split)    1.7    3.3    6.4   12.3
//     2 tiles (split)   2.6    3.0    6.1   11.6
//     4 tiles (split)   3.8    4.0    4.9    9.3
//     8 tiles           5.7    5.8    6.1    7.5
// The plain rule's segments, which fill the chip by themselves, take whole heads.
int tiles_of(int64_t heads, int dv, int most) {
  int t = 1;
  while (t < most && heads * ((dv + 16 * t - 1) / (16 * t)) > kCus) t *= 2;
  return t;
}

// The workspace's part for packets: 1 GiB (270000 tokens of 8 heads) bounds it, whatever the length.  It has
// room for packets with planes, whichever the call takes: fewer heads of the same tokens do take them.
constexpr int64_t kWindowBytes = int64_t(1) << 30;

int64_t packet_bytes(const ChunkPlan& c) {
  const int64_t all = units_of(c, kC), unit = c.H * int64_t(kPacket<true>), fit = kWindowBytes / unit;
  return (all <= fit ? all : fit > 0 ? fit : 1) * unit;
}

// Units of a window, of which a longer call has several and takes two launches for each
int64_t window_units(const ChunkPlan& c, int64_t packet) {
  const int64_t all = units_of(c, kC), fit = packet_bytes(c) / (c.H * packet);
  return all <= fit ? all : fit;
}

struct Launch {
  const ChunkPlan& c;
  ChunkArgs p;
  int64_t units;
  hipStream_t st;

  template <int DK, bool DELTA, bool OUT, bool LOCAL>
  void walk(int tiles) {
    p.col_blocks = (c.dv + 16 * tiles - 1) / (16 * tiles);
    const uint32_t grid = uint32_t(units * c.H * p.col_blocks);
    constexpr int kWhole = whole_tiles(DK);
    if (tiles == kWhole) {
      linear_columns_kernel<DK, 1, kWhole, DELTA, OUT, LOCAL><<<grid, 64 * kWhole, 0, st>>>(p);
    } else if constexpr (!LOCAL) {
      if (tiles == 1) linear_split_kernel<DK, 1, 1, DELTA, OUT><<<grid, kSplitThreads<1, 1, DELTA>, 0, st>>>(p);
      else if (tiles == 2) linear_split_kernel<DK, 1, 2, DELTA, OUT><<<grid, kSplitThreads<1, 2, DELTA>, 0, st>>>(p);
      else if constexpr (DK == 128) linear_split_kernel<DK, 2, 2, DELTA, OUT><<<grid, kSplitThreads<2, 2, DELTA>, 0, st>>>(p);
    }
  }

  template <int DK>
  void run(char* ws) {
    constexpr int kWhole = whole_tiles(DK);
    const bool out = p.a.io.o;
    if (c.delta) {
      units = c.n_req;
      const int tiles = tiles_of(units * c.H, c.dv, kWhole);
      const int64_t all = units_of(c, kC), step = window_units(c, tiles == kWhole ? kPacket<false> : kPacket<true>);
      float* const carry = reinterpret_cast<float*>(ws + packet_bytes(c));
      const int64_t carried = int64_t(c.H) * DK * c.dv;
      p.packets = ws;
      for (int64_t u = 0, j = 0; u < all; u += step, ++j) {
        p.u0 = u;
        p.u1 = u + step < all ? u + step : all;
        p.carry_in = carry + (j & 1) * carried;
        p.carry_out = carry + (1 - (j & 1)) * carried;
        const int64_t jobs = (p.u1 - p.u0) * c.H;
        const uint32_t grid = uint32_t((jobs + 3) / 4);
        if (tiles == kWhole) linear_factor_kernel<DK, false, false><<<grid, 256, 0, st>>>(p, jobs);
        else if (out) linear_factor_kernel<DK, true, true><<<grid, 256, 0, st>>>(p, jobs);
        else linear_factor_kernel<DK, false, true><<<grid, 256, 0, st>>>(p, jobs);
        if (out) walk<DK, true, true, false>(tiles);
        else walk<DK, true, false, false>(tiles);
      }
      return;
    }
    const Segments g = segments_of(c);
    p.seg_chunks = g.chunks;
    p.seg_each = g.each;
    if (p.seg_chunks == 0) {
      units = c.n_req;
      const int tiles = tiles_of(units * c.H, c.dv, kWhole);
      if (out) walk<DK, false, true, false>(tiles);
      else walk<DK, false, false, false>(tiles);
      return;
    }
    units = g.units;
    p.seg_state = reinterpret_cast<float*>(ws);
    p.seg_log2 = reinterpret_cast<double*>(ws + units * c.H * int64_t(DK) * c.dv * 4);
    p.seg_bad = reinterpret_cast<int32_t*>(p.seg_log2 + units * c.H);
    walk<DK, false, false, true>(kWhole);
    linear_join_kernel<<<dim3(DK * c.dv / 1024, c.H, c.n_req), 256, 0, st>>>(p, DK, !out);
    if (out) walk<DK, false, true, false>(kWhole);
    else linear_finish_kernel<DK><<<uint32_t(c.n_req * c.H * (c.dv / 16)), 4 * DK, 0, st>>>(p);
  }
};

}  // namespace

constexpr int64_t kMaxHeads = 1 << 21;      // of all requests: a grid counts threads in 32 bits

bool linear_chunk_supported(const ChunkPlan& c) {
  return (c.dk == 64 || c.dk == 128) && c.dv % 16 == 0 && c.n_tokens > 0 && int64_t(c.n_req) * c.H <= kMaxHeads;
}

// For this call and for every one with no more requests and tokens, none longer: a caller that allocates once,
// for its largest, has enough for all.  More requests alone may need less (they are not split, or too many
// for the chunked form), so what depends on their number is taken at its most.
int64_t linear_chunk_workspace(ChunkPlan c) {
  if (c.n_req * int64_t(c.H) > kMaxHeads) c.n_req = int32_t(kMaxHeads / c.H);
  if (c.n_req == 0 || !linear_chunk_supported(c)) return 0;
  if (c.delta) {
    const bool windows = window_units(c, kPacket<true>) < units_of(c, kC);
    return packet_bytes(c) + (windows ? 2 * int64_t(c.H) * c.dk * c.dv * 4 : 0);
  }
  const int64_t room = segment_room(c);     // segments, and so requests that are split
  const int64_t state = int64_t(c.dk) * c.dv * 4;
  return may_split(c) ? room * c.H * (state + 8 + state / 4096 * (c.dv / 16) * 4) : 0;
}

void launch_linear_chunks(const ChunkPlan& c, const LinearArgs& a, void* ws, hipStream_t st) {
  ChunkArgs p{};
  p.a = a;
  p.q_tok = int32_t(a.io.q_tok);
  p.k_tok = int32_t(a.io.k_tok);
  p.v_tok = int32_t(a.io.v_tok);
  p.o_tok = int32_t(a.io.o_tok);
  Launch l{c, p, 0, st};
  if (c.dk == 64) l.run<64>(static_cast<char*>(ws));
  else l.run<128>(static_cast<char*>(ws));
}

}  // namespace dasc

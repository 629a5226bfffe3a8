// Attention of new tokens over a paged cache.
//
// For the tokens of a request and a key head h, the rows of a tile are (token, query head of h's group), so a
// key is read once for the whole group.  Scores are formed transposed, S^T = K Q^T on 32 x 32 x 16 matrix
// instructions: a lane then holds 16 scores of one row, whose maximum and sum it takes by itself (and once
// across the two halves of the wave), and after exp2 the lane's weights are already the operand P^T of
//     O^T <- 2^(m - m') O^T + V^T P^T,
// for a product's operands may hold the keys in any order, if both hold the same one: half h of the
// wave has keys 16 s + 4 h + {0..3} and 16 s + 8 + 4 h + {0..3} of step s.  V^T comes from LDS through the
// transposing read.  The running maximum m and sum l are fp32 and in units of log2.
//
// The weights are rounded to the cache's type, as the matrix operand has to be; scores, maxima, sums and O are not,
// and the sum takes the weights unrounded.  Each is off by at most half a step, independently, so an output's error
// is that of its own rounding and about as much again: 0.0023 of its norm for bf16 and 0.00027 for fp16, where weights of
// 32 bits give 0.0017 and 0.0002.  A second operand for what the rounding left would double the products with V.
//
// Work.  A tile's keys may be split: the pieces of all requests are numbered in order, and every block finds
// its own from the device's lengths, so that a piece has about the same number of keys whatever the requests'
// lengths are.  Pieces of a split tile leave (m, l, O) in the workspace, and a second kernel joins them.
//
// What is not seen must not reach a result: its weight is 0, but 0 times an infinity or NaN is NaN.  Positions
// beyond a request or of no page are put into LDS as zeros.  A block that finds a value that is not finite where some
// of its rows see the position and some do not starts again, a token at a time, with what that one does not
// see as zeros: right, but slow.
//
// Measured.  Few rows: HBM bounds it; 64 tokens over 1500 to 10000 positions, 32 heads of 128 on 8 of keys, 1.64 GB in
// 300 us (5.4 TB/s, where a large copy runs at 4.8).  Many rows: 2048 tokens over 30011 positions, 16 heads of
// 256, 727 TFLOP/s; over 16048, 32 heads of 128, 917, and of 64, 654 (a large matrix product 1330).  Matrix instructions
// are busy 13 to 38% of the time, LDS as long as they: a wave has 32 rows, so each of its products, 32 cycles of its SIMD,
// reads 1 KB of K or V, and four SIMDs ask for the 128 bytes a cycle that LDS gives (conflicts, a fifth to a quarter of its
// cycles, come on top).  Reads that are not hidden under products cost matrix time one for one; beside them
// stand a step's waits, the exchange of a row's maximum across the wave, the barrier, the loads' addresses.

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "cache_common.h"
#include "launch_common.h"
#include "output_rows.h"
#include "wy_ops.h"

namespace dasc {
namespace {

using dasc_wy::f32x16;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ---- types ------------------------------------------------------------------------------------

using dasc_wy::f32x4;

struct Bf16 {
  typedef bf16x8 x8;
  __device__ static f32x4 mfma(x8 a, x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  typedef __bf16 elem;
  static constexpr uint32_t kExp = 0x7F807F80u;      // exponents of two elements
  static constexpr float kLift = 0.0f;               // see rebase()
  __device__ static f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
struct F16 {
  typedef f16x8 x8;
  __device__ static f32x4 mfma(x8 a, x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
  typedef _Float16 elem;
  static constexpr uint32_t kExp = 0x7C007C00u;
  static constexpr float kLift = 7.0f;
  __device__ static f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

// Whether one of eight elements is an infinity or NaN
template <typename T>
__device__ inline bool odd_value(u32x4 v) {
  constexpr uint32_t lo = T::kExp & 0xFFFFu, hi = T::kExp & 0xFFFF0000u;
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) odd |= (v[i] & lo) == lo || (v[i] & hi) == hi;
  return odd;
}

// See the note on waits in linear_chunk.hip: results of matrix instructions that cross a branch
__device__ inline void settle(f32x16& x) { asm volatile("s_nop 15\n\ts_nop 3" : "+v"(x)); }
__device__ inline void settle(f32x4& x) { asm volatile("s_nop 7\n\ts_nop 3" : "+v"(x)); }
template <typename V, int N>
__device__ inline void settle(V (&x)[N]) {
  settle(x[0]);
#pragma unroll
  for (int i = 1; i < N; ++i) asm volatile("" : "+v"(x[i]));
}

// ---- work -------------------------------------------------------------------------------------

struct Divisor {                          // n / d for 0 <= n < 2^31: (n * mul) >> 32 >> shift
  uint32_t mul, shift, d;
  __device__ uint32_t of(uint32_t n) const { return d == 1 ? n : __umulhi(n, mul) >> shift; }
};

struct AttnArgs {
  dasc_kv_cache c;
  dasc_attn_io io;
  Divisor group, page, heads;
  uint32_t k_page, k_tok, v_page, v_tok;  // the cache's strides of pages and tokens
  int64_t block0;                         // first block of this launch: piece * n_kv_heads + head
  int64_t pieces;                         // of a key head that there is room for
  int32_t target;                         // pieces of a key head to aim at
  int32_t split;                          // whether tiles may be split
  int32_t least;                          // steps that a piece has at least
  float scale2;                           // scale * log2 e
  int4* meta;                             // [pieces]: of a tile's first piece, request, first row, rows, splits
  float* ml;                              // [pieces, n_kv_heads, rows of a tile, 2]
  float* part;                            // [pieces, n_kv_heads, rows of a tile, D]
};

struct Piece {
  int32_t req, row0, rows, tok0, len, kv; // rows of the tile, the request's first token, tokens and positions
  int32_t index, splits;
};

// Blocks are numbered by piece, then by head: the long pieces of all heads come first, and heads that are a
// multiple of eight apart share the L2 of an XCD.
__device__ inline void block_of(const AttnArgs& a, int& head, int& index) {
  if (a.block0 == 0) {
    index = int(a.heads.of(blockIdx.x));
    head = int(blockIdx.x) - index * a.c.n_kv_heads;
  } else {
    const int64_t x = a.block0 + blockIdx.x;
    index = int(x / a.c.n_kv_heads);
    head = int(x % a.c.n_kv_heads);
  }
}

// How request r is cut: its tiles of ROWS rows, and the keys of its last one in steps of KEYS
struct Cut { int32_t tok0, len, kv, tiles, steps; };

template <int ROWS, int KEYS>
__device__ inline Cut cut_of(const AttnArgs& a, int r) {
  Cut c = {0, 0, 0, 0, 0};
  if (r >= a.io.n_req) return c;
  const int n = int(a.io.n_tokens);
  int lo = a.io.cu_seqlens[r], hi = a.io.cu_seqlens[r + 1];
  lo = lo < 0 ? 0 : lo > n ? n : lo;
  hi = hi < lo ? lo : hi > n ? n : hi;
  const int most = a.io.table_width * a.c.page_size;
  int kv = a.io.kv_lens[r];
  kv = kv < 0 ? 0 : kv > most ? most : kv;
  c.tok0 = lo;
  c.len = hi - lo;
  c.kv = kv;
  c.tiles = int((int64_t(c.len) * a.group.d + ROWS - 1) / ROWS);
  int64_t keys = kv;
  if (a.io.window > 0) {                  // what the rows of a tile can see
    const int64_t span = int64_t(a.io.window) + ROWS / a.group.d + 1;
    if (a.io.causal && span < keys) keys = span;
  }
  c.steps = int((keys + KEYS - 1) / KEYS);
  if (c.steps == 0) c.steps = 1;
  return c;
}

// Piece `index` of the call, for every lane of the wave alike; false if there is none.
template <int ROWS, int KEYS>
__device__ inline bool locate(const AttnArgs& a, int index, Piece& p) {
  const int lane = threadIdx.x % 64;
  const Cut first = cut_of<ROWS, KEYS>(a, lane);
  int64_t per = int64_t(1) << 40;         // steps of a piece
  if (a.split) {
    uint64_t all = 0;
    for (int r0 = 0; r0 < a.io.n_req; r0 += 64) {
      const Cut c = r0 ? cut_of<ROWS, KEYS>(a, r0 + lane) : first;
      all += uint64_t(c.tiles) * uint64_t(c.steps);
    }
#pragma unroll
    for (int s = 1; s < 64; s *= 2) all += __shfl_xor((unsigned long long)all, s);
    per = int64_t((all + a.target - 1) / a.target);
    if (per < a.least) per = a.least;
  }
  const auto take = [&](const Cut& c, int splits, int r0, int at, int rest) {
    const auto of = [&](int x) { return __builtin_amdgcn_readlane(x, at); };
    const int tiles = of(c.tiles);
    p.splits = of(splits);
    const int tile = tiles - 1 - rest / p.splits;          // the longest first
    p.index = rest % p.splits;
    p.req = r0 + at;
    p.tok0 = of(c.tok0);
    p.len = of(c.len);
    p.kv = of(c.kv);
    p.row0 = tile * ROWS;
    const int left = p.len * int(a.group.d) - p.row0;
    p.rows = left < ROWS ? left : ROWS;
  };
  if (!a.split && a.io.n_req <= 64) {     // whole tiles: the longest request's first
    const Cut& c = first;
    int64_t before = 0;
    for (int j = 0; j < a.io.n_req; ++j) {
      const int steps = __builtin_amdgcn_readlane(c.steps, j), tiles = __builtin_amdgcn_readlane(c.tiles, j);
      before += steps > c.steps || (steps == c.steps && j < lane) ? tiles : 0;
    }
    const uint64_t in = __ballot(before <= index && index < before + c.tiles);
    if (!in) return false;
    const int at = __builtin_ctzll(in);
    take(c, 1, 0, at, __builtin_amdgcn_readlane(int(index - before), at));
    return true;
  }
  int64_t before = 0;
  for (int r0 = 0; r0 < a.io.n_req; r0 += 64) {
    const Cut c = r0 ? cut_of<ROWS, KEYS>(a, r0 + lane) : first;
    const int splits = a.split ? int((c.steps + per - 1) / per) : 1;
    const int64_t mine = int64_t(c.tiles) * splits;
    int64_t upto = mine;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const int64_t y = __shfl_up((long long)upto, s);
      if (lane >= s) upto += y;
    }
    const uint64_t past = __ballot(before + upto > index);
    if (past) {
      const int at = __builtin_ctzll(past);
      take(c, splits, r0, at, __builtin_amdgcn_readlane(int(index - (before + upto - mine)), at));
      return true;
    }
    before += __shfl((long long)upto, 63);
  }
  return false;
}

// ---- what the kernels share -----------------------------------------------------------------------

// Tiles of many rows: WQ waves of 32 rows each, steps of KW keys; D: head_dim rounded up
template <int D, int WQ, int KW>
struct Form {
  static constexpr int kThreads = 64 * WQ, kRows = 32 * WQ, kKeys = KW;
  static constexpr int kChunks = D / 8;                       // 16 bytes each, of a row
  static constexpr int kLoads = kKeys * kChunks / kThreads;   // of a thread, keys and values each
  static constexpr int kRowBytes = 2 * D;
  static constexpr int kKv = kKeys * kRowBytes;
};

// Tiles of many rows: waves of 32 rows each, waves of a SIMD, keys of a step.  Heads of 128 (2048 tokens over 16048,
// us): eight waves and 64 keys 550, four waves twice on a CU with 32 keys 651, eight with 32 keys 705.  Heads of 64:
// four waves twice on a CU 386, eight 405, three times four 380 with spills (a window of 1000 over 4097 tokens 45, 107
// and 56).  Heads of 256: a wave has 128 registers of O and 64 of Q, so it has a SIMD to itself (two: 2730 to 4380 us with
// spills, one: 1433).
constexpr int wide_wq(int D) { return D == 128 ? 8 : 4; }
constexpr int wide_simd(int D) { return D == 256 ? 1 : 2; }
constexpr int wide_keys(int D) { return D == 256 ? 32 : 64; }
// Of few rows: waves of a SIMD, which are blocks of a CU.  Heads of 256 have 128 or 64 registers of loads on their way.
constexpr int few_simd(int form, int D) { return D == 256 && form < 2 ? 1 : 2; }

// Where 16-byte chunk c of row r lies: lanes of a read that take the same chunk of many rows (keys), or a few
// chunks of four rows (values), are spread over the banks (two cycles of conflicts a product are left, of its eight of LDS)
__device__ inline int key_chunk(int r, int c) { return c ^ (r & 7); }
template <int D>
__device__ inline int value_chunk(int r, int c) {
  return c ^ (D == 64 ? (r >> 1 & 1) << 2 : (r & 3) << 2) ^ (r >> 2 & 1) << 1;
}

// The positions that token t of the request sees: lo .. hi
struct Sight { int lo, hi; };
__device__ inline Sight sight(const AttnArgs& a, const Piece& p, int t) {
  const int64_t here = int64_t(p.kv) - p.len + t;
  const int64_t hi = a.io.causal && here < p.kv - 1 ? here : p.kv - 1;
  const int64_t lo = a.io.window > 0 && here - a.io.window >= 0 ? here - a.io.window + 1 : 0;
  return {int(lo > INT32_MAX ? INT32_MAX : lo), int(hi < -1 ? -1 : hi)};
}

// A lane's row of a tile
struct Row {
  bool real;               // not one that pads the tile
  int tok;                 // token of the request
  int64_t qh;              // query head
  int lo, hi;              // positions that it sees (a row that pads the tile: all)
  int all_lo, all_hi;      // positions that every row of the wave sees
};
template <int R = 32>
__device__ inline Row row_of(const AttnArgs& a, const Piece& p, int head, int r) {
  Row x;
  const int row = p.row0 + r, G = a.group.d;
  x.real = r < p.rows;
  x.tok = x.real ? int(a.group.of(row)) : 0;
  x.qh = int64_t(head) * G + (x.real ? row - x.tok * G : 0);
  const Sight s = sight(a, p, x.tok);
  x.lo = x.real ? s.lo : 0;
  x.hi = x.real ? s.hi : INT32_MAX;
  x.all_lo = x.lo;
  x.all_hi = x.hi;
#pragma unroll
  for (int i = 1; i < R; i *= 2) {
    const int lo = __shfl_xor(x.all_lo, i), hi = __shfl_xor(x.all_hi, i);
    x.all_lo = lo > x.all_lo ? lo : x.all_lo;
    x.all_hi = hi < x.all_hi ? hi : x.all_hi;
  }
  x.all_lo = __builtin_amdgcn_readfirstlane(x.all_lo);
  x.all_hi = __builtin_amdgcn_readfirstlane(x.all_hi);
  return x;
}

// The operand Q of a lane's row: channels 16 s + 8 half + {0..7} of each step s
template <typename T, int D>
__device__ inline void load_query(const AttnArgs& a, const Piece& p, const Row& row, int half, typename T::x8 (&q)[D / 16]) {
  const auto* at = static_cast<const typename T::elem*>(a.io.q) + (int64_t(p.tok0) + row.tok) * a.io.q_tok + row.qh * a.io.q_head;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    const int c = 16 * s + 8 * half;
    u32x4 v = {0, 0, 0, 0};
    if (row.real && c < a.c.head_dim) v = *reinterpret_cast<const u32x4*>(at + c);
    q[s] = __builtin_bit_cast(typename T::x8, v);
  }
}

// Key of element e of the scores, from the wave's first
__device__ inline int key_at(int e, int half) { return 8 * (e / 4) + 4 * half + e % 4; }

// A lane's places in LDS.  Chunk 2 i + half of row n lies at key[i % 4] + (i / 4) * 128, and of the rows that step
// 16 u of the keys takes the columns of tile i at value[i % 4] + (i / 4) * 256 (D = 64: value[i]), for rows
// that are multiples of 32 (keys) and 16 (values) apart swap the same chunks.
struct Places { int key[4], value[4]; };
template <int D>
__device__ inline Places places_of(int lane) {
  Places x;
  const int n = lane % 32, half = lane / 32, r = 4 * half + lane % 16 / 4;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x.key[i] = n * 2 * D + key_chunk(n, 2 * i + half) * 16;
    const int c = i * 32 + lane % 32 / 16 * 16 + lane % 4 * 4;
    x.value[i] = r * 2 * D + value_chunk<D>(r, c / 8) * 16 + c % 8 * 2;
  }
  return x;
}

// Nothing moves across.  Left alone, the compiler waits for each operand right before its product, an LDS access's
// time each; so the order of reads, products and arithmetic in the inner loops is the one that is written.
__device__ inline void hold() { __builtin_amdgcn_sched_barrier(0); }

// S^T = K Q^T of 32 keys, four operands on their way
template <typename T, int D>
__device__ inline void scores(const char* lk, const Places& at, const typename T::x8 (&q)[D / 16], f32x16& s) {
  constexpr int kSteps = D / 16, kAhead = 4;
  const auto read = [&](int i) {
    return *reinterpret_cast<const typename T::x8*>(lk + at.key[i % 4] + i / 4 * 128);
  };
  typename T::x8 k[kAhead];
#pragma unroll
  for (int j = 0; j < kAhead; ++j) k[j] = read(j);
#pragma unroll
  for (int e = 0; e < 16; ++e) s[e] = 0;
  hold();
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    s = T::mfma(k[j % kAhead], q[j], s);
    if (j + kAhead < kSteps) k[j % kAhead] = read(j + kAhead);
    hold();
  }
}

// Scores that are not seen become -inf.  have: the 32 positions that have a page, a bit each.
__device__ inline void hide(f32x16& s, int half, int key0, uint32_t have, const Row& row) {
  if (have == 0xFFFFFFFFu && key0 >= row.all_lo && key0 + 31 <= row.all_hi) return;
  settle(s);
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int i = key_at(e, half);
    s[e] = (have >> i & 1) && key0 + i >= row.lo && key0 + i <= row.hi ? s[e] : -__builtin_inff();
  }
}

// A base is a finite number, so that none less another is NaN.  A row without a score yet has -kLargest, and weights
// 2^-inf = 0; one with a score of +inf has kLargest, and the weight 2^inf = inf there: its sum and log-sum are +inf, its
// output inf / inf = NaN.
constexpr float kLargest = 0x1.fffffep127f;

// A wave that has a SIMD to itself has 256 accumulation registers beside its others, which products read and write
// directly.  O stays there if it is put there wherever it was last touched by other arithmetic; else the compiler
// moves all of it there and back in every step.
template <bool ACC, typename V, int N>
__device__ inline void in_acc(V (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
    if constexpr (ACC) asm volatile("" : "+a"(x[i]));
}
// The row's running base m of the weights 2^(s - m), sum l (of this half's keys) and output O, before scores with
// maximum `top` (of this half's, unscaled) join them.  The base follows the maximum only where that has left it by more
// than 2^8 in some row: most steps leave O alone.  It stands kLift below the maximum then, so a weight is at most
// 2^(kLift + 8): in fp16, whose numbers end at 2^16 and lose bits below 2^-14, the largest is 2^7 to 2^15, and what has
// less than 2^-21 of it is off by up to 2^-32 of it.
template <typename T, bool ACC, typename V, int NO>
__device__ inline void rebase(float top, float scale2, float& m, float& l, V (&o)[NO]) {
  constexpr int kE = sizeof(V) / 4;
  constexpr float kMost = T::kLift + 8.0f;
  top = fmaxf(top, __shfl_xor(top, 32));
  if (__any(fmaf(top, scale2, -m) > kMost)) {
    float next = fmaxf(m, fmaf(top, scale2, -T::kLift));
    // (scores from 2^26 on: a base rounded down may leave more than the largest weight above it)
    if (fmaf(top, scale2, -next) > kMost) next += fabsf(next) * 0x1p-23f;
    next = fminf(next, kLargest);
    const float shrink = __builtin_amdgcn_exp2f(m - next);
    m = next;
    l *= shrink;
    settle(o);
#pragma unroll
    for (int i = 0; i < NO; ++i)
#pragma unroll
      for (int e = 0; e < kE; ++e) o[i][e] *= shrink;
    in_acc<ACC>(o);
  }
}
template <typename T, bool ACC, int NO>
__device__ inline void rebase(f32x16& s, float scale2, float& m, float& l, f32x16 (&o)[NO]) {
  settle(s);
  float top = -__builtin_inff();
#pragma unroll
  for (int e = 0; e < 16; ++e) top = fmaxf(top, s[e]);
  rebase<T, ACC>(top, scale2, m, l, o);
}

// V^T of 16 keys from row r0 (a multiple of 16) of lv, columns 32 i ..
template <typename T, int D>
__device__ inline typename T::x8 value_operand(const char* lv, const Places& at, int r0, int i) {
  union { s16x4 h[2]; typename T::x8 v; } x;
  const char* p = lv + at.value[i % 4] + r0 * 2 * D + i / 4 * 256;
  x.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p));
  x.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 16 * D));
  return x.v;
}

// A row's result: to the workspace if its tile is split, else to the output.  g: the lane's part of the row, columns
// 4 g + {0..3} of each 8 (of 32 rows), or of each 16.
template <typename T, int D, typename V, int N>
__device__ inline void write_row(const AttnArgs& a, const Piece& p, const Row& row, int64_t slot, int g, float m, float l,
                                 const V (&o)[N]) {
  if (!row.real) return;
  constexpr int kFours = D / N == 32 ? 4 : 1, kWidth = D / N == 32 ? 8 : 16;
  if (p.splits > 1) {
    if (g == 0) {
      a.ml[slot * 2] = m;
      a.ml[slot * 2 + 1] = l;
    }
    float* out = a.part + slot * D;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int b = 0; b < kFours; ++b)
        *reinterpret_cast<float4*>(out + (i * kFours + b) * kWidth + 4 * g) =
            make_float4(o[i][4 * b], o[i][4 * b + 1], o[i][4 * b + 2], o[i][4 * b + 3]);
    return;
  }
  typedef typename T::elem elem;
  typedef elem e4 __attribute__((ext_vector_type(4)));
  const int64_t t = int64_t(p.tok0) + row.tok;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  elem* out = static_cast<elem*>(a.io.o) + t * a.io.o_tok + row.qh * a.io.o_head;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int b = 0; b < kFours; ++b) {
      const int c = (i * kFours + b) * kWidth + 4 * g;
      e4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = elem(o[i][4 * b + e] * inv);
      if (c < a.c.head_dim) *reinterpret_cast<e4*>(out + c) = x;
    }
  if (a.io.lse && g == 0) a.io.lse[t * a.io.lse_tok + row.qh * a.io.lse_head] = m * 0.69314718056f + logf(l);
}

// The block's piece; false if there is none.  The first block of a split tile says so to those that join.  (Requests
// whose rows overlap, which are not allowed, may have more pieces than there is room for: a tile that ends beyond is
// left out.)
template <int ROWS, int KEYS>
__device__ inline bool take_piece(const AttnArgs& a, int head, int index, Piece& p) {
  const bool any = locate<ROWS, KEYS>(a, index, p) && int64_t(index) - p.index + p.splits <= a.pieces;
  if (a.split && head == 0 && threadIdx.x == 0)
    a.meta[index] =
        any && p.index == 0 && p.splits > 1 ? make_int4(p.req, p.row0, p.rows, p.splits) : make_int4(0, 0, 0, 0);
  return any;
}

// The steps of KEYS positions of a piece, and the positions that every row of its tile sees
struct Steps { int begin, end, all_lo, all_hi; };
template <int KEYS>
__device__ inline Steps steps_of(const AttnArgs& a, const Piece& p) {
  const Sight first = sight(a, p, int(a.group.of(p.row0))), last = sight(a, p, int(a.group.of(p.row0 + p.rows - 1)));
  const int64_t begin = first.lo / KEYS, end = last.hi < first.lo ? begin : last.hi / KEYS + 1;
  return {int(begin + (end - begin) * p.index / p.splits), int(begin + (end - begin) * (p.index + 1) / p.splits),
          last.lo, first.hi};
}

// A token that is taken alone, and the positions that it sees.  tok: -1: none is
struct Alone { int tok, lo, hi; };
// Whether the pass sees position `key`
__device__ inline bool taken(const Alone& x, int key) { return x.tok < 0 || (key >= x.lo && key <= x.hi); }
// After a pass over a tile: whether another has to follow, over the next of its tokens alone
__device__ inline bool next_alone(const AttnArgs& a, const Piece& p, bool odd, Alone& x) {
  if (x.tok < 0) {
    if (!odd) return false;
    x.tok = int(a.group.of(p.row0));
  } else if (++x.tok > int(a.group.of(p.row0 + p.rows - 1))) {
    return false;
  }
  const Sight s = sight(a, p, x.tok);
  x.lo = s.lo;
  x.hi = s.hi;
  return true;
}

// ---- few rows -------------------------------------------------------------------------------------

// A tile of 32 keys and 16 rows, on 16 x 16 x 32 products: lane (g, n) = (lane / 16, lane % 16) has keys
// 4 g + {0..3} of each 16 of row n, so both tiles of S^T again form the operand P^T, keys 4 g + {0..3} and
// 16 + 4 g + {0..3} of a product.
template <typename T, int D, bool ACC>
struct Tile {
  static constexpr int kO = D / 16, kQ = D / 32;
  typedef typename T::x8 x8;
  x8 q[kQ];
  f32x4 o[kO];
  float m, l;
  int key_place[2], value_place[8];

  __device__ void start(const AttnArgs& a, const Piece& p, const Row& row, int lane) {
    const int n = lane % 16, g = lane / 16;
#pragma unroll
    for (int i = 0; i < 2; ++i) key_place[i] = n * 2 * D + key_chunk(n, 4 * i + g) * 16;
    const int r = 4 * g + n / 4;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = i * 16 + lane % 4 * 4;
      value_place[i] = r * 2 * D + value_chunk<D>(r, c / 8) * 16 + c % 8 * 2;
    }
    const auto* at = static_cast<const typename T::elem*>(a.io.q) + (int64_t(p.tok0) + row.tok) * a.io.q_tok + row.qh * a.io.q_head;
#pragma unroll
    for (int i = 0; i < kQ; ++i) {
      const int c = (4 * i + g) * 8;
      u32x4 v = {0, 0, 0, 0};
      if (row.real && c < a.c.head_dim) v = *reinterpret_cast<const u32x4*>(at + c);
      q[i] = __builtin_bit_cast(x8, v);
    }
    m = -kLargest;
    l = 0;
#pragma unroll
    for (int i = 0; i < kO; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][e] = 0;
    in_acc<ACC>(o);
  }
  __device__ x8 key_operand(const char* lk, int j) const {      // of product j: keys 16 (j / kQ) .., channels j % kQ
    const int t = j / kQ, i = j % kQ;
    return *reinterpret_cast<const x8*>(lk + key_place[i % 2] + i / 2 * 128 + t * 32 * D);
  }
  __device__ x8 value_operand(const char* lv, int i) const {    // columns 16 i ..
    union { s16x4 h[2]; x8 v; } x;
    const char* p = lv + value_place[i % 8] + i / 8 * 256;
    x.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p));
    x.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 32 * D));
    return x.v;
  }
  // S^T, hidden where it is not seen, the base, and O^T += V^T P^T
  __device__ void step(const char* lk, const char* lv, int lane, int key0, uint64_t have, const Row& row, float scale2) {
    constexpr int kAll = 2 * kQ, kAhead = 4;
    x8 k[kAhead];
    f32x4 s[2];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) k[j] = key_operand(lk, j);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[t][e] = 0;
    hold();
#pragma unroll
    for (int j = 0; j < kAll; ++j) {
      s[j / kQ] = T::mfma(k[j % kAhead], q[j % kQ], s[j / kQ]);
      if (j + kAhead < kAll) k[j % kAhead] = key_operand(lk, j + kAhead);
      hold();
    }
    settle(s);
    if (have != (uint64_t(1) << 32) - 1 || key0 < row.all_lo || key0 + 31 > row.all_hi) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 16 * t + 4 * (lane / 16) + e;
          s[t][e] = (have >> i & 1) && key0 + i >= row.lo && key0 + i <= row.hi ? s[t][e] : -__builtin_inff();
        }
    }
    float top = -__builtin_inff();
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) top = fmaxf(top, s[t][e]);
    rebase<T, ACC>(fmaxf(top, __shfl_xor(top, 16)), scale2, m, l, o);
    x8 v[kAhead], w;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) v[j] = value_operand(lv, j);
    float sum[2] = {0, 0};
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = __builtin_amdgcn_exp2f(fmaf(s[t][e], scale2, -m));
        w[t * 4 + e] = typename T::elem(x);
        sum[e % 2] += x;
      }
    l += sum[0] + sum[1];
    hold();
#pragma unroll
    for (int j = 0; j < kO; ++j) {
      o[j] = T::mfma(v[j % kAhead], w, o[j]);
      if (j + kAhead < kO) v[j % kAhead] = value_operand(lv, j + kAhead);
      hold();
    }
  }
};

// Four waves: WQ on 16 rows each with the same keys, the others with keys of their own, 32 a wave and step.  Each group
// of WQ waves has its place in LDS; one that is alone needs no barrier.  Keys and values of the next step are on
// their way in registers meanwhile, the pages of the one after too.
template <typename T, int D, int WQ, int SIMD, bool ONE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(SIMD, SIMD))) void attn_few_kernel(AttnArgs a) {
  constexpr int R = 16, WK = 4 / WQ, kKeys = 32 * WK, kRows = R * WQ, kRowBytes = 2 * D, kKv = 32 * kRowBytes;
  constexpr int kChunks = D / 8, kWaveRows = 64 / kChunks, kLoads = 32 / WQ / kWaveRows;   // rows of a load; loads of a wave
  constexpr int kMerge = (WK - 1) * WQ * R * (D + 2) * 4;
  typedef typename T::elem elem;
  __shared__ __attribute__((aligned(16))) char lds[2 * WK * kKv > kMerge ? 2 * WK * kKv : kMerge];
  __shared__ int odd_flag;
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64), wq = wave % WQ, wk = wave / WQ;
  int head, index;
  block_of(a, head, index);
  Piece p;
  if (!take_piece<kRows, kKeys>(a, head, index, p)) return;
  if (tid == 0) odd_flag = 0;
  __syncthreads();
  const Row row = row_of<R>(a, p, head, wq * R + lane % R);
  const Steps steps = steps_of<kKeys>(a, p);
  const int d = a.c.head_dim;

  const int32_t* table = a.io.block_table + int64_t(p.req) * a.io.table_req;
  const elem* const kc = static_cast<const elem*>(a.c.k) + head * a.c.k_head;
  const elem* const vc = static_cast<const elem*>(a.c.v) + head * a.c.v_head;
  Alone alone = {-1, 0, 0};
  // Lane r (and r + 32) knows where row r of its group's keys lies; see the kernel for many rows
  int entry, inside;
  const int stand_in = ONE ? (p.kv - 1) & -kWaveRows : p.kv - 1;   // for positions beyond the last, its page's too
  const auto ask = [&](int step) {
    int key = (step < steps.end ? step : steps.end - 1) * kKeys + wk * 32 + lane % 32;
    key = key < p.kv ? key : stand_in;
    const int at = a.page.of(key);
    entry = table[at];
    inside = key - at * int(a.page.d);
  };
  const auto there = [&](int step) {
    const int key = step * kKeys + wk * 32 + lane;
    return __ballot(lane < 32 && step < steps.end && key < p.kv && entry >= 0 && entry < a.c.n_pages && taken(alone, key));
  };
  const auto rows_at = [&](uint32_t page_stride, uint32_t tok_stride) {
    const uint32_t b = entry >= 0 && entry < a.c.n_pages ? entry : 0;
    return uint64_t(b) * page_stride + uint64_t(uint32_t(inside)) * tok_stride;
  };
  constexpr uint64_t kAll = (uint64_t(1) << 32) - 1;
  const int chunk = lane % kChunks, column = chunk * 8 < d ? chunk * 8 : 0, first_row = wq * (32 / WQ);
  const uint32_t k_lane = 2 * ((ONE ? lane / kChunks : 0) * a.k_tok + column);     // bytes
  const uint32_t v_lane = 2 * ((ONE ? lane / kChunks : 0) * a.v_tok + column);
  const auto load = [&](const elem* base, uint64_t rows, uint32_t lane_off, u32x4 (&x)[kLoads]) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      uint64_t where;
      if constexpr (ONE) {
        const int r = first_row + i * kWaveRows;
        where = uint32_t(__builtin_amdgcn_readlane(int(uint32_t(rows)), r)) |
                uint64_t(uint32_t(__builtin_amdgcn_readlane(int(uint32_t(rows >> 32)), r))) << 32;
      } else {
        where = __shfl((unsigned long long)rows, first_row + i * kWaveRows + lane / kChunks);
      }
      x[i] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(base + where) + lane_off);
    }
  };
  char* const lk = lds + wk * 2 * kKv;
  char* const lv = lk + kKv;
  // Where load i goes: rows eight apart swap the same chunks
  constexpr int kPlaces = kWaveRows >= 8 ? 1 : 8 / kWaveRows;
  int k_place[kPlaces], v_place[kPlaces];
#pragma unroll
  for (int i = 0; i < kPlaces; ++i) {
    const int r = first_row + i * kWaveRows + lane / kChunks;
    k_place[i] = r * kRowBytes + key_chunk(r, chunk) * 16;
    v_place[i] = r * kRowBytes + value_chunk<D>(r, chunk) * 16;
  }
  const auto store = [&](char* to, const int (&place)[kPlaces], uint64_t have, u32x4 (&x)[kLoads]) {
    if (have != kAll || d < D) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        if (!(have >> (first_row + i * kWaveRows + lane / kChunks) & 1) || chunk * 8 >= d) x[i] = u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      *reinterpret_cast<u32x4*>(to + place[i % kPlaces] + i / kPlaces * kPlaces * kWaveRows * kRowBytes) = x[i];
  };
  const auto watch = [&](int step, const u32x4 (&x)[kLoads]) {
    const int key0 = step * kKeys + wk * 32;
    if (alone.tok >= 0 || (key0 >= steps.all_lo && key0 + 31 <= steps.all_hi)) return;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) odd |= odd_value<T>(x[i]);
    if (odd) odd_flag = 1;
  };
  const bool alike = a.k_page == a.v_page && a.k_tok == a.v_tok;
  u32x4 kr[kLoads], vr[kLoads];
  const auto load_both = [&] {
    const uint64_t k_rows = rows_at(a.k_page, a.k_tok);
    load(kc, k_rows, k_lane, kr);
    load(vc, alike ? k_rows : rows_at(a.v_page, a.v_tok), v_lane, vr);
  };

  Tile<T, D, SIMD == 1> t;
  const bool busy = steps.begin < steps.end;
  do {
    uint64_t have = 0;
    if (busy) {
      ask(steps.begin);
      have = there(steps.begin);
      load_both();
      ask(steps.begin + 1);
    }
    t.start(a, p, row, lane);
    if (busy) {
      store(lk, k_place, have, kr);
      store(lv, v_place, have, vr);
      watch(steps.begin, vr);
      // (else the first product of every step would wait for the queries' loads, and so for all that came after)
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        u32x4 x = __builtin_bit_cast(u32x4, t.q[i]);
        asm volatile("" : "+v"(x));
        t.q[i] = __builtin_bit_cast(typename T::x8, x);
      }
      for (int step = steps.begin; step < steps.end; ++step) {
        const uint64_t next = there(step + 1);
        if (step + 1 < steps.end) load_both();
        ask(step + 2);
        if constexpr (WQ > 1) __syncthreads();
        t.step(lk, lv, lane, step * kKeys + wk * 32, have, row, a.scale2);
        if constexpr (WQ > 1) __syncthreads();
        if (step + 1 < steps.end) {
          store(lk, k_place, next, kr);
          store(lv, v_place, next, vr);
          watch(step + 1, vr);
        }
        have = next;
      }
    }
    settle(t.o);
    t.l += __shfl_xor(t.l, 16);
    t.l += __shfl_xor(t.l, 32);

    // waves that share rows meet in LDS
    __syncthreads();
    const bool odd = odd_flag;
    if constexpr (WK > 1) {
      const auto part = [&](int w) { return reinterpret_cast<float*>(lds) + ((w - 1) * WQ + wq) * R * (D + 2); };
      if (wk > 0) {
        float* const mine = part(wk);
        if (lane < R) {
          mine[lane * 2] = t.m;
          mine[lane * 2 + 1] = t.l;
        }
#pragma unroll
        for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4*>(mine + 2 * R + (i * 64 + lane) * 4) = t.o[i];
      }
      __syncthreads();
      if (wk == 0) {
#pragma unroll 1
        for (int w = 1; w < WK; ++w) {
          const float* const other = part(w);
          const float om = other[lane % R * 2], ol = other[lane % R * 2 + 1];
          const float both = fmaxf(t.m, om);
          const float f = __builtin_amdgcn_exp2f(t.m - both), g = __builtin_amdgcn_exp2f(om - both);
          t.m = both;
          t.l = t.l * f + ol * g;
#pragma unroll
          for (int i = 0; i < D / 16; ++i) {
            const f32x4 x = *reinterpret_cast<const f32x4*>(other + 2 * R + (i * 64 + lane) * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) t.o[i][e] = t.o[i][e] * f + x[e] * g;
          }
        }
      }
    }
    if (wk == 0 && (alone.tok < 0 ? !odd : row.tok == alone.tok))
      write_row<T, D>(a, p, row, (int64_t(index) * a.c.n_kv_heads + head) * kRows + wq * R + lane % R, lane / R, t.m, t.l, t.o);
    if (!next_alone(a, p, odd, alone)) return;
    __syncthreads();                                 // LDS is free again
  } while (true);
}

// ---- many rows --------------------------------------------------------------------------------------

// From the scores S(u) of 32 keys to the next: the products of S(u + 1) run while the weights of S(u) are formed, and
// the products of those while S(u + 1)'s maximum is taken.  lk: keys of u + 1, lv: values of u.  `mask` hides what
// is not seen of S(u + 1).
template <typename T, int D, typename M>
__device__ inline void advance(const char* lk, const char* lv, const Places& at, const typename T::x8 (&q)[D / 16],
                               float scale2, f32x16& s, float& m, float& l, f32x16 (&o)[D / 32], const M& mask) {
  constexpr int kSteps = D / 16, kDt = D / 32, kSlice = 16 / kSteps, kMax = 16 / (2 * kDt - 2) + 1;
  const auto read_k = [&](int j) { return *reinterpret_cast<const typename T::x8*>(lk + at.key[j % 4] + j / 4 * 128); };
  const auto read_v = [&](int j) { return value_operand<T, D>(lv, at, j / kDt * 16, j % kDt); };
  typename T::x8 k[4], v[4], w[2];
  f32x16 next;
  const float base = m;
  float part[2] = {0, 0};
#pragma unroll
  for (int j = 0; j < 4; ++j) k[j] = read_k(j);
#pragma unroll
  for (int e = 0; e < 16; ++e) next[e] = 0;
  hold();
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    next = T::mfma(k[j % 4], q[j], next);
    if (j + 4 < kSteps) k[j % 4] = read_k(j + 4);
#pragma unroll
    for (int e = j * kSlice; e < (j + 1) * kSlice; ++e) {
      const float x = __builtin_amdgcn_exp2f(fmaf(s[e], scale2, -base));
      w[e / 8][e % 8] = typename T::elem(x);
      part[e % 2] += x;
    }
    // (else the weights would move to where they are used, past the branch)
    if ((j + 1) * kSlice % 8 == 0) {
      u32x4 x = __builtin_bit_cast(u32x4, w[((j + 1) * kSlice - 1) / 8]);
      asm volatile("" : "+v"(x));
      w[((j + 1) * kSlice - 1) / 8] = __builtin_bit_cast(typename T::x8, x);
    }
    asm volatile("" : "+v"(part[0]), "+v"(part[1]));
    hold();
  }
  l += part[0] + part[1];
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = read_v(j);
  mask(next);
  float top = -__builtin_inff();
  hold();
#pragma unroll
  for (int j = 0; j < 2 * kDt; ++j) {
    o[j % kDt] = T::mfma(v[j % 4], w[j / kDt], o[j % kDt]);
    if (j + 4 < 2 * kDt) v[j % 4] = read_v(j + 4);
    // two products later the next scores are there, whichever way the branch before went
    if (j == 1) asm volatile("" : "+v"(next));
    if (j >= 2) {
#pragma unroll
      for (int e = (j - 2) * kMax; e < (j - 1) * kMax && e < 16; ++e) top = fmaxf(top, next[e]);
    }
    hold();
  }
  rebase<T, D == 256>(top, scale2, m, l, o);
  s = next;
}

// WQ waves of 32 rows each go over the keys together, 32 at a time, a product ahead (advance()).  Keys are in LDS
// two steps ahead and values one, so the block meets once a step; the loads of both are issued at a step's
// start and stored at its end.  No wave may still read what another stores before they meet: between two meetings
// the present and the next step's keys are read (the present one's before the loop too, for the first scores) and those
// of the step after them are stored, so keys have three buffers whatever a step's size; values, of which the
// present step's are read and the next one's stored, have two.  ONE: a load's rows always lie in one page, whose address is
// then the same for a wave.
template <typename T, int D, int WQ, int SIMD, bool ONE>
__global__ __launch_bounds__(64 * WQ) __attribute__((amdgpu_waves_per_eu(SIMD, SIMD))) void attn_wide_kernel(AttnArgs a) {
  constexpr int KW = wide_keys(D), NS = KW / 32;
  typedef Form<D, WQ, KW> F;
  typedef typename T::elem elem;
  constexpr int kKeyBuffers = 3;
  __shared__ __attribute__((aligned(16))) char lds[(kKeyBuffers + 2) * F::kKv];
  char* const lds_v = lds + kKeyBuffers * F::kKv;
  const int tid = threadIdx.x, lane = tid % 64, n = lane % 32, half = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  int head, index;
  block_of(a, head, index);
  Piece p;
  if (!take_piece<F::kRows, F::kKeys>(a, head, index, p)) return;
  const Steps steps = steps_of<F::kKeys>(a, p);
  const Places at = places_of<D>(lane);
  const Row row = row_of(a, p, head, wave * 32 + n);
  // the steps that some row of the wave sees something of
  const int w0 = wave * 32, r0 = w0 < p.rows ? w0 : p.rows - 1, r1 = w0 + 31 < p.rows ? w0 + 31 : p.rows - 1;
  const int first = sight(a, p, int(a.group.of(p.row0 + r0))).lo / F::kKeys;
  const int end_hi = sight(a, p, int(a.group.of(p.row0 + r1))).hi, last = end_hi < 0 ? -1 : end_hi / F::kKeys;
  Alone alone = {-1, 0, 0};
  // A pass over the tile, of all its rows or for the token that is taken alone; whether a value was met that calls
  // for the latter.  (Two copies, so that the first has no register to spare for the others' loop.)
  const auto pass = [&](auto single) -> bool {
    constexpr bool kAlone = decltype(single)::value;
    const int d = a.c.head_dim;

    const int32_t* table = a.io.block_table + int64_t(p.req) * a.io.table_req;
    const elem* const kc = static_cast<const elem*>(a.c.k) + head * a.c.k_head;
    const elem* const vc = static_cast<const elem*>(a.c.v) + head * a.c.v_head;
    // Lane r of a wave knows where row r of a step lies.  Its entry of the table is asked for a step ahead, and looked
    // at when it is there.  Loads have no branch: what is not there is loaded from page 0 and put into LDS as zeros.
    struct Place { int entry, inside; };             // the entry, the place in the page
    constexpr int kRow = F::kThreads / F::kChunks, kWaveRows = 64 / F::kChunks;   // rows of a load of the block, of a wave
    // for positions beyond the last (with ONE, where the rows after it are of its page too)
    const int stand_in = ONE ? (p.kv - 1) & -kWaveRows : p.kv - 1;
    const auto ask = [&](int step) {
      int key = (step < steps.end ? step : steps.end - 1) * F::kKeys + lane % KW;
      key = key < p.kv ? key : stand_in;
      const int at = a.page.of(key);
      return Place{table[at], key - at * int(a.page.d)};
    };
    const auto is_page = [&](const Place& x) { return x.entry >= 0 && x.entry < a.c.n_pages; };
    const auto there = [&](int step, const Place& x) {   // the positions of the step that have a page
      const int key = step * F::kKeys + lane;
      return __ballot(lane < KW && step < steps.end && key < p.kv && is_page(x) && (!kAlone || taken(alone, key)));
    };
    const auto k_rows_at = [&](const Place& x) {
      return uint64_t(uint32_t(is_page(x) ? x.entry : 0)) * a.k_page + uint64_t(uint32_t(x.inside)) * a.k_tok;
    };
    const bool alike = a.k_page == a.v_page && a.k_tok == a.v_tok;
    const auto v_rows_at = [&](const Place& x, uint64_t k_rows) {
      return alike ? k_rows : uint64_t(uint32_t(is_page(x) ? x.entry : 0)) * a.v_page + uint64_t(uint32_t(x.inside)) * a.v_tok;
    };
    constexpr uint64_t kAll = KW == 64 ? ~uint64_t(0) : (uint64_t(1) << 32) - 1;
    const int chunk = tid % F::kChunks, column = chunk * 8 < d ? chunk * 8 : 0;
    const uint32_t k_lane = 2 * ((ONE ? lane / F::kChunks : 0) * a.k_tok + column);   // bytes
    const uint32_t v_lane = 2 * ((ONE ? lane / F::kChunks : 0) * a.v_tok + column);
    const auto load = [&](const elem* base, uint64_t rows, uint32_t lane_off, u32x4 (&x)[F::kLoads]) {
#pragma unroll
      for (int i = 0; i < F::kLoads; ++i) {
        uint64_t at;
        if constexpr (ONE) {                         // the rows of a wave's load follow the first, in its page
          const int r = i * kRow + wave * kWaveRows;
          at = uint32_t(__builtin_amdgcn_readlane(int(uint32_t(rows)), r)) |
               uint64_t(uint32_t(__builtin_amdgcn_readlane(int(uint32_t(rows >> 32)), r))) << 32;
        } else {
          at = __shfl((unsigned long long)rows, i * kRow + tid / F::kChunks);
        }
        x[i] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(base + at) + lane_off);
      }
    };
    const int row_in = tid / F::kChunks;             // (kRow is a multiple of eight: loads swap the same chunks)
    const int k_place = row_in * F::kRowBytes + key_chunk(row_in, chunk) * 16;
    const int v_place = row_in * F::kRowBytes + value_chunk<D>(row_in, chunk) * 16;
    const auto store = [&](char* to, uint64_t have, u32x4 (&x)[F::kLoads]) {
      if (have != kAll || d < D) {
#pragma unroll
        for (int i = 0; i < F::kLoads; ++i)
          if (!(have >> (i * kRow + row_in) & 1) || chunk * 8 >= d) x[i] = u32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int i = 0; i < F::kLoads; ++i) *reinterpret_cast<u32x4*>(to + i * kRow * F::kRowBytes) = x[i];
    };
    // Whether the values of a step have to be watched: some row of the block does not see some of its positions, and
    // a value is not finite.  The block meets.
    const auto meet = [&](int step, const u32x4 (&x)[F::kLoads]) {
      if (kAlone || step >= steps.end ||
          (step * F::kKeys >= steps.all_lo && step * F::kKeys + F::kKeys - 1 <= steps.all_hi)) {
        __syncthreads();
        return false;
      }
      bool odd = false;
#pragma unroll
      for (int i = 0; i < F::kLoads; ++i) odd |= odd_value<T>(x[i]);
      return __syncthreads_or(odd) != 0;
    };

    typename T::x8 q[D / 16];
    load_query<T, D>(a, p, row, half, q);
    f32x16 o[D / 32], s;
    float m = -kLargest, l = 0;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[i][e] = 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = -__builtin_inff();
    in_acc<D == 256>(o);
    bool watch = false;
    if (steps.begin < steps.end) {
      u32x4 kr[F::kLoads], vr[F::kLoads];
      // the first two steps' pages, keys and values at once: a block's start is a chain of loads
      const Place p0 = ask(steps.begin), p1 = ask(steps.begin + 1);
      Place next = ask(steps.begin + 2);             // of the keys to be loaded next
      u32x4 k1[F::kLoads];
      uint64_t have = there(steps.begin, p0), have1 = there(steps.begin + 1, p1), have2;   // of the present step, of those after
      uint64_t k_rows = k_rows_at(p0);
      load(kc, k_rows, k_lane, kr);
      load(vc, v_rows_at(p0, k_rows), v_lane, vr);
      k_rows = k_rows_at(p1);
      load(kc, k_rows, k_lane, k1);
      uint64_t v_rows = v_rows_at(p1, k_rows);       // of the values to be loaded next
      store(lds + k_place, have, kr);
      store(lds_v + v_place, have, vr);
      store(lds + F::kKv + k_place, have1, k1);
      watch = meet(steps.begin, vr);
      if (!watch) {
        scores<T, D>(lds, at, q, s);
        hide(s, half, steps.begin * F::kKeys, uint32_t(have), row);
        rebase<T, D == 256>(s, a.scale2, m, l, o);
      }
      const auto mask_of = [&](int step, uint64_t all, int t) {
        return [&, step, all, t](f32x16& x) {
          hide(x, half, step * F::kKeys + t * 32, uint32_t(all >> (32 * t)), row);
        };
      };
      int kb = 0;                                    // the buffer of the present step's keys
      for (int step = steps.begin; step < steps.end && !watch; ++step) {
        const char* const lv = lds_v + ((step - steps.begin) & 1) * F::kKv;
        const int kb1 = kb + 1 == kKeyBuffers ? 0 : kb + 1, kb2 = kb1 + 1 == kKeyBuffers ? 0 : kb1 + 1;
        have2 = there(step + 2, next);
        k_rows = k_rows_at(next);
        load(kc, k_rows, k_lane, kr);
        load(vc, v_rows, v_lane, vr);
        v_rows = v_rows_at(next, k_rows);
        next = ask(step + 3);
        if (step + 1 >= first && step <= last) {     // else nothing of this step or the next is seen by the wave
          if constexpr (NS == 2)
            advance<T, D>(lds + kb * F::kKv + 32 * F::kRowBytes, lv, at, q, a.scale2, s, m, l, o, mask_of(step, have, 1));
          advance<T, D>(lds + kb1 * F::kKv, lv + (NS - 1) * 32 * F::kRowBytes, at, q, a.scale2, s, m, l, o,
                        mask_of(step + 1, have1, 0));
        }
        store(lds + kb2 * F::kKv + k_place, have2, kr);
        store(lds_v + ((step + 1 - steps.begin) & 1) * F::kKv + v_place, have1, vr);
        watch = meet(step + 1, vr);
        have = have1;
        have1 = have2;
        kb = kb1;
      }
    }
    settle(o);
    l += __shfl_xor(l, 32);
    if (kAlone ? row.tok == alone.tok : !watch)
      write_row<T, D>(a, p, row, (int64_t(index) * a.c.n_kv_heads + head) * F::kRows + wave * 32 + n, half, m, l, o);
    return watch;
  };
  const bool odd = pass(std::false_type{});
  if (!odd) return;
#pragma unroll 1
  while (next_alone(a, p, odd, alone)) {
    __syncthreads();                               // LDS is free again
    (void)pass(std::true_type{});
  }
}

// The pieces of a split tile: o = sum 2^(m_i - m) O_i / sum 2^(m_i - m) l_i.  A wave has a row, lane i the weight of
// piece i (of 64 at a time).
constexpr int kJoinRows = 16;                    // of a block
template <typename T, int D, int ROWS>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a) {
  typedef typename T::elem elem;
  constexpr int V = D / 64;                      // columns of a lane
  typedef float fv __attribute__((ext_vector_type(V)));
  typedef elem ev __attribute__((ext_vector_type(V)));
  int head, index;
  block_of(a, head, index);
  const int heads = a.c.n_kv_heads, lane = threadIdx.x % 64;
  const int4 t = a.meta[index];                  // request, first row, rows, pieces
  if (t.w < 2) return;
  const int c = lane * V, n = int(a.io.n_tokens), G = a.group.d;
  int tok0 = a.io.cu_seqlens[t.x];
  tok0 = tok0 < 0 ? 0 : tok0 > n ? n : tok0;
  const int end = int(blockIdx.y + 1) * kJoinRows < t.z ? (blockIdx.y + 1) * kJoinRows : t.z;
  for (int r = blockIdx.y * kJoinRows + threadIdx.x / 64; r < end; r += 4) {
    const auto slot = [&](int i) { return (int64_t(index + i) * heads + head) * ROWS + r; };
    const auto stats = [&](int i) { return *reinterpret_cast<const float2*>(a.ml + slot(i) * 2); };   // m, l
    float2 own = lane < t.w ? stats(lane) : make_float2(-__builtin_inff(), 0.0f);
    float m = own.x;
    for (int i = 64 + lane; i < t.w; i += 64) m = fmaxf(m, stats(i).x);
#pragma unroll
    for (int s = 1; s < 64; s *= 2) m = fmaxf(m, __shfl_xor(m, s));
    float l = 0;
    fv o = 0;
    for (int i0 = 0; i0 < t.w; i0 += 64) {
      if (i0 > 0) own = i0 + lane < t.w ? stats(i0 + lane) : make_float2(-__builtin_inff(), 0.0f);
      const float f = __builtin_amdgcn_exp2f(own.x - m);
      l += f * own.y;
      const int some = t.w - i0 < 64 ? t.w - i0 : 64;
      const auto piece = [&](int i) { return *reinterpret_cast<const fv*>(a.part + slot(i0 + i) * D + c); };
      const auto weight = [&](int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), i)); };
      int i = 0;
      for (; i + 4 <= some; i += 4) {
        const fv x0 = piece(i), x1 = piece(i + 1), x2 = piece(i + 2), x3 = piece(i + 3);
        o += weight(i) * x0;
        o += weight(i + 1) * x1;
        o += weight(i + 2) * x2;
        o += weight(i + 3) * x3;
      }
      for (; i < some; ++i) o += weight(i) * piece(i);
    }
#pragma unroll
    for (int s = 1; s < 64; s *= 2) l += __shfl_xor(l, s);
    const int tok = int(a.group.of(t.y + r)), qh = head * G + t.y + r - tok * G;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const int64_t at = int64_t(tok0) + tok;
    ev x;
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = elem(o[e] * inv);
    if (c < a.c.head_dim)
      *reinterpret_cast<ev*>(static_cast<elem*>(a.io.o) + at * a.io.o_tok + qh * a.io.o_head + c) = x;
    if (a.io.lse && lane == 0) a.io.lse[at * a.io.lse_tok + qh * a.io.lse_head] = m * 0.69314718056f + logf(l);
  }
}

// ---- launches -----------------------------------------------------------------------------------

// How a call runs: the form by the rows of its longest request, pieces by the tiles that it can have
struct Launch {
  int form;                      // 0: up to 16 rows, 1: 32, 2: 64, 3: many
  int rows, keys;                // of a tile and a step
  int64_t pieces;                // of a key head, at most
  bool split;
  int target;
};

constexpr float kLog2e = 1.44269504089f;
constexpr int kWide = 3;         // the form of many rows
constexpr int kUnits = 256;      // compute units
constexpr int64_t kMostTok = int64_t(1) << 27;   // eight tokens' bytes fit into 32 bits
constexpr int kMostPieces = 16;  // of a tile of many rows

// Blocks of a compute unit
constexpr int wide_blocks(int D) { return 4 * wide_simd(D) / wide_wq(D); }

int dim_of(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }

constexpr int least_steps(int form) { return form == kWide ? 4 : 1; }

// Pieces of few rows that a call aims at: two for each place that a block has
int few_target(int form, int D, int n_kv_heads) {
  const int x = 2 * kUnits * few_simd(form, D) / n_kv_heads;
  return x < 1 ? 1 : x;
}

void shape_of(Launch& x, int D) {
  if (x.form == kWide) {
    x.rows = 32 * wide_wq(D);
    x.keys = wide_keys(D);
  } else {
    x.rows = 16 << x.form;
    x.keys = 128 >> x.form;
  }
}

Launch launch_of(int n_req, int64_t n_tokens, int group, int n_kv_heads, int head_dim, int max_len, int max_kv,
                 int64_t window) {
  Launch x;
  const int64_t most = n_tokens < max_len ? n_tokens : max_len;
  const int64_t rows = most * group;
  x.form = rows <= 16 ? 0 : rows <= 32 ? 1 : rows <= 64 ? 2 : kWide;
  shape_of(x, dim_of(head_dim));
  const int64_t tiles = n_tokens * group / x.rows + n_req;
  const int64_t steps = (int64_t(max_kv) + x.keys - 1) / x.keys;
  x.target = 1;
  x.split = false;
  if (x.form == kWide) {
    // Blocks go over the chip in rounds: a tile is cut into as many pieces as leave least of the last one empty.
    // (Requests end inside a tile, each in the middle of one on average.)
    const int64_t about = (n_tokens * group + (n_req - 1) * int64_t(x.rows / 2) + x.rows - 1) / x.rows * n_kv_heads;
    const int64_t slots = kUnits * wide_blocks(dim_of(head_dim));
    const int64_t reach = window > 0 && window + x.rows / group + 1 < max_kv ? window + x.rows / group + 1 : max_kv;
    const double length = double(reach) / x.keys;            // steps of a tile
    double best = 1e30;
    int at = 1;
    for (int n = 1; n <= kMostPieces && (n == 1 || n * least_steps(kWide) <= length) && (n == 1 || about < 2 * slots); ++n) {
      // a piece's start and end cost as much as four steps, and its part of the join as much again
      const double time = double((about * n + slots - 1) / slots) * (length / n + (n > 1 ? 8 : 4));
      if (time < best) best = time, at = n;
    }
    x.split = at > 1;
    x.target = int(x.split ? (about * at + n_kv_heads - 1) / n_kv_heads : 1);
  } else {
    x.target = few_target(x.form, dim_of(head_dim), n_kv_heads);
    x.split = tiles < 2 * x.target && steps > least_steps(x.form);
  }
  x.pieces = x.split ? tiles + x.target : tiles;
  return x;
}

template <typename T, int D, int FORM>
void launch_form(AttnArgs a, const Launch& x, hipStream_t st) {
  constexpr int64_t kMost = int64_t(1) << 22;     // a grid counts threads in 32 bits
  const int64_t blocks = x.pieces * a.c.n_kv_heads;
  for (a.block0 = 0; a.block0 < blocks; a.block0 += kMost) {
    const uint32_t g = uint32_t(blocks - a.block0 < kMost ? blocks - a.block0 : kMost);
    const bool one = a.page.d % (512 / D) == 0;   // the rows of a wave's load are of one page
    if constexpr (FORM < kWide) {
      constexpr int WQ = 1 << FORM;
      if (one) attn_few_kernel<T, D, WQ, few_simd(FORM, D), true><<<g, 256, 0, st>>>(a);
      else attn_few_kernel<T, D, WQ, few_simd(FORM, D), false><<<g, 256, 0, st>>>(a);
    } else if (one)
      attn_wide_kernel<T, D, wide_wq(D), wide_simd(D), true><<<g, 64 * wide_wq(D), 0, st>>>(a);
    else attn_wide_kernel<T, D, wide_wq(D), wide_simd(D), false><<<g, 64 * wide_wq(D), 0, st>>>(a);
  }
  constexpr int kRows = FORM == kWide ? 32 * wide_wq(D) : 16 << FORM;
  a.block0 = 0;
  if (x.split)                                    // few pieces
    attn_join_kernel<T, D, kRows><<<dim3(uint32_t(blocks), (kRows + kJoinRows - 1) / kJoinRows), 256, 0, st>>>(a);
}

template <typename T, int D>
void launch_rows(const AttnArgs& a, const Launch& x, hipStream_t st) {
  switch (x.form) {
    case 0: launch_form<T, D, 0>(a, x, st); break;
    case 1: launch_form<T, D, 1>(a, x, st); break;
    case 2: launch_form<T, D, 2>(a, x, st); break;
    default: launch_form<T, D, kWide>(a, x, st); break;
  }
}

template <typename T>
void launch_dim(const AttnArgs& a, const Launch& x, hipStream_t st) {
  switch (dim_of(a.c.head_dim)) {
    case 64: launch_rows<T, 64>(a, x, st); break;
    case 128: launch_rows<T, 128>(a, x, st); break;
    default: launch_rows<T, 256>(a, x, st); break;
  }
}

Divisor divisor(uint32_t d) {              // exact for n < 2^31
  Divisor x = {0, 0, d};
  if (d == 1) return x;
  uint32_t s = 0;
  while ((uint64_t(1) << s) < d) ++s;      // 2^(s - 1) < d <= 2^s
  x.shift = s - 1;
  x.mul = uint32_t(((uint64_t(1) << (31 + s)) + d - 1) / d);
  return x;
}

int check_sizes(int32_t n_req, int64_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim) {
  if (head_dim < 8 || head_dim > 256 || head_dim % 8 || n_kv_heads < 1 || n_q_heads < 1 || n_q_heads > 65535 ||
      n_q_heads % n_kv_heads || n_tokens < 0 || n_tokens > INT32_MAX ||
      n_tokens * (n_q_heads / n_kv_heads) > INT32_MAX)
    return DASC_E_SHAPE;
  return n_req < 1 ? DASC_E_INVAL : DASC_OK;
}

}  // namespace
}  // namespace dasc

extern "C" int dasc_cache_attn_workspace_bytes(int32_t n_req, int64_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads,
                                               int32_t head_dim, int32_t max_len, int32_t max_kv, size_t* bytes) {
  using namespace dasc;
  if (!bytes || max_len < 0 || max_kv < 0) return DASC_E_INVAL;
  const int rc = check_sizes(n_req, n_tokens, n_q_heads, n_kv_heads, head_dim);
  if (rc != DASC_OK) return rc;
  *bytes = 0;
  // the largest need of any smaller call: each form at its most tiles
  const int group = n_q_heads / n_kv_heads;
  const int64_t D = dim_of(head_dim);
  for (int form = 0; form <= kWide; ++form) {
    if (form > 0 && int64_t(max_len) * group <= (8 << form)) continue;    // no request that takes it
    Launch x;
    x.form = form;
    shape_of(x, int(D));
    // (a tile is cut only where there are few tiles)
    const int64_t tiles = n_tokens * group / x.rows + n_req, target = few_target(form, int(D), n_kv_heads);
    const int64_t most = form == kWide ? 2 * (2 * kUnits * wide_blocks(int(D)) / n_kv_heads + 2) : 2 * target;
    const int64_t pieces = (tiles < most ? tiles : most) * (form == kWide ? kMostPieces + 1 : 1) +
                           (form == kWide ? 2 * kMostPieces : target);
    const int64_t need = pieces * 16 + pieces * n_kv_heads * x.rows * (D + 2) * 4;
    if (max_kv > least_steps(form) * x.keys && size_t(need) > *bytes) *bytes = size_t(need);
  }
  return DASC_OK;
}

extern "C" int dasc_cache_attn(const dasc_kv_cache* given, const dasc_attn_io* attn, void* workspace,
                               size_t workspace_bytes, dasc_stream_t stream) {
  using namespace dasc;
  if (!given || !attn) return DASC_E_INVAL;
  AttnArgs a;
  a.c = *given;
  a.io = *attn;
  drop_unused(a.c);
  drop_unused(a.io.n_tokens, {&a.io.q_tok, &a.io.o_tok, &a.io.lse_tok});
  drop_unused(a.io.n_q_heads, {&a.io.q_head, &a.io.o_head, &a.io.lse_head});
  drop_unused(a.io.n_req, {&a.io.table_req});
  const dasc_kv_cache* const cache = &a.c;
  const dasc_attn_io* const io = &a.io;
  int rc = check_cache(cache, 16);
  if (rc != DASC_OK) return rc;
  rc = check_sizes(io->n_req, io->n_tokens, io->n_q_heads, cache->n_kv_heads, cache->head_dim);
  if (rc != DASC_OK) return rc;
  if (io->table_width < 0 || io->max_len < 0 || io->max_kv < 0 || io->window < 0 || io->table_req < 0 ||
      (io->causal != 0 && io->causal != 1) || !std::isfinite(io->scale * kLog2e) || !(io->scale >= 0x1p-126f))
    return DASC_E_INVAL;
  if (int64_t(io->table_width) * cache->page_size > INT32_MAX) return DASC_E_SHAPE;
  if (!io->cu_seqlens || !io->kv_lens || (io->table_width > 0 && !io->block_table) ||
      !aligned_to(io->cu_seqlens, 4) || !aligned_to(io->kv_lens, 4) || !aligned_to(io->block_table, 4) ||
      !aligned_to(io->lse, 4))
    return DASC_E_INVAL;
  if (io->q_tok < 0 || io->q_head < 0 || io->q_tok % 8 || io->q_head % 8 || io->o_tok % 8 || io->o_head % 8)
    return DASC_E_INVAL;
  if (!rows_apart(io->n_tokens, io->o_tok, io->n_q_heads, io->o_head, cache->head_dim) ||
      (io->lse && !rows_apart(io->n_tokens, io->lse_tok, io->n_q_heads, io->lse_head, 1)))
    return DASC_E_INVAL;
  if (io->n_tokens == 0) return DASC_OK;
  if (!io->q || !io->o || !aligned16(io->q) || !aligned16(io->o)) return DASC_E_INVAL;
  const int group = io->n_q_heads / cache->n_kv_heads;
  const int most = io->table_width * cache->page_size;
  const Launch x = launch_of(io->n_req, io->n_tokens, group, cache->n_kv_heads, cache->head_dim, io->max_len,
                             io->max_kv < most ? io->max_kv : most, io->window);
  if (cache->k_page > UINT32_MAX || cache->v_page > UINT32_MAX || cache->k_tok >= kMostTok || cache->v_tok >= kMostTok)
    return DASC_E_UNSUPPORTED;
  a.k_page = uint32_t(cache->k_page);
  a.k_tok = uint32_t(cache->k_tok);
  a.v_page = uint32_t(cache->v_page);
  a.v_tok = uint32_t(cache->v_tok);
  a.group = divisor(group);
  a.heads = divisor(cache->n_kv_heads);
  a.page = divisor(cache->page_size);
  a.pieces = x.pieces;
  a.target = x.target;
  a.split = x.split;
  a.least = least_steps(x.form);
  a.scale2 = io->scale * kLog2e;
  a.meta = nullptr;
  a.ml = a.part = nullptr;
  if (x.split) {
    const int64_t rows = x.pieces * cache->n_kv_heads * x.rows, D = dim_of(cache->head_dim);
    const size_t need = size_t(x.pieces * 16 + rows * (D + 2) * 4);
    if (workspace_bytes < need || !workspace) return DASC_E_WORKSPACE;
    if (!aligned16(workspace)) return DASC_E_INVAL;
    a.meta = static_cast<int4*>(workspace);
    a.part = reinterpret_cast<float*>(a.meta + x.pieces);
    a.ml = a.part + rows * D;
  }
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (cache->dtype == DASC_DTYPE_BF16) launch_dim<Bf16>(a, x, st);
  else launch_dim<F16>(a, x, st);
  return launch_status();
}

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
// Work.  A tile's keys may be split: the pieces of all requests are numbered in order, and every block finds
// its own from the device's lengths, so that a piece has about the same number of keys whatever the requests'
// lengths are.  Pieces of a split tile leave (m, l, O) in the workspace, and a second kernel joins them.
//
// What is not seen must not reach a result: its weight is 0, but 0 times an infinity or NaN is NaN.  Positions
// beyond a request or of no page are put into LDS as zeros; where a tile's mask cuts through its positions
// and a value in it is not finite, the products are made one by one (careful()).

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

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

struct Bf16 {
  typedef bf16x8 x8;
  typedef __bf16 elem;
  static constexpr uint32_t kExp = 0x7F807F80u;      // exponents of two elements
  __device__ static f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
struct F16 {
  typedef f16x8 x8;
  typedef _Float16 elem;
  static constexpr uint32_t kExp = 0x7C007C00u;
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

// ---- work -------------------------------------------------------------------------------------

struct Divisor {                          // n / d for 0 <= n < 2^31: (n * mul) >> 32 >> shift
  uint32_t mul, shift, d;
  __device__ uint32_t of(uint32_t n) const { return d == 1 ? n : __umulhi(n, mul) >> shift; }
};

struct AttnArgs {
  dasc_kv_cache c;
  dasc_attn_io io;
  Divisor group, page;
  int32_t index0;                         // first piece of this launch
  int32_t target;                         // pieces of a key head to aim at
  int32_t split;                          // whether tiles may be split
  float scale2;                           // scale * log2 e
  int4* meta;                             // [pieces]: of a tile's first piece, request, first row, rows, splits
  float* ml;                              // [pieces, n_kv_heads, rows of a tile, 2]
  float* part;                            // [pieces, n_kv_heads, rows of a tile, D]
};

struct Piece {
  int32_t req, row0, rows, tok0, len, kv; // rows of the tile, the request's first token, tokens and positions
  int32_t index, splits;
};

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
  int64_t per = int64_t(1) << 40;         // steps of a piece
  if (a.split) {
    uint64_t all = 0;
    for (int r0 = 0; r0 < a.io.n_req; r0 += 64) {
      const Cut c = cut_of<ROWS, KEYS>(a, r0 + lane);
      all += uint64_t(c.tiles) * uint64_t(c.steps);
    }
#pragma unroll
    for (int s = 1; s < 64; s *= 2) all += __shfl_xor((unsigned long long)all, s);
    per = int64_t((all + a.target - 1) / a.target);
    if (per < kMinSteps) per = kMinSteps;
  }
  int64_t before = 0;
  for (int r0 = 0; r0 < a.io.n_req; r0 += 64) {
    const Cut c = cut_of<ROWS, KEYS>(a, r0 + lane);
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
      const auto of = [&](int x) { return __builtin_amdgcn_readlane(x, at); };
      const int rest = of(int(index - (before + upto - mine)));
      const int tiles = of(c.tiles);
      p.splits = of(splits);
      const int tile = tiles - 1 - rest / p.splits;        // the longest first
      p.index = rest % p.splits;
      p.req = r0 + at;
      p.tok0 = of(c.tok0);
      p.len = of(c.len);
      p.kv = of(c.kv);
      p.row0 = tile * ROWS;
      const int left = p.len * int(a.group.d) - p.row0;
      p.rows = left < ROWS ? left : ROWS;
      return true;
    }
    before += __shfl((long long)upto, 63);
  }
  return false;
}

// ---- the kernel ---------------------------------------------------------------------------------

// WQ waves of 32 rows each, WK of them on the same rows with KW keys each; D: head_dim rounded up
template <typename T, int D, int WQ, int WK, int KW>
struct Form {
  static constexpr int kWaves = WQ * WK, kThreads = 64 * kWaves;
  static constexpr int kRows = 32 * WQ, kKeys = KW * WK;      // of a step
  static constexpr int kChunks = D / 8;                       // 16 bytes each, of a row
  static constexpr int kLoads = kKeys * kChunks / kThreads;   // of a thread, keys and values each
  static constexpr int kRowBytes = 2 * D;
  static constexpr int kKv = kKeys * kRowBytes;
  static constexpr int kScratch = kWaves * 16 * 32 * 4;       // weights of 16 keys a wave
  static constexpr int kMerge = WK > 1 ? (WK - 1) * WQ * 32 * (D + 2) * 4 : 0;
  static constexpr int kLds = 2 * kKv + kScratch > kMerge ? 2 * kKv + kScratch : kMerge;
};

// Where 16-byte chunk c of row r lies: lanes of a read that take the same chunk of many rows (keys), or a few
// chunks of four rows (values), meet different banks
__device__ inline int key_chunk(int r, int c) { return c ^ (r & 7); }
template <int D>
__device__ inline int value_chunk(int r, int c) {
  return D == 64 ? c ^ ((r >> 1 & 1) << 2) : c ^ ((r & 3) << 2);
}

template <typename T, int D, int WQ, int WK, int KW>
__global__ __launch_bounds__(64 * WQ * WK) void attn_kernel(AttnArgs a) {
  typedef Form<T, D, WQ, WK, KW> F;
  typedef typename T::x8 x8;
  typedef typename T::elem elem;
  constexpr int kSub = KW / 32;                  // tiles of 32 keys of a wave
  constexpr int kDt = D / 32, kSteps = D / 16;
  __shared__ __attribute__((aligned(16))) char lds[F::kLds];
  char* const lk = lds;
  char* const lv = lds + F::kKv;
  const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64, n = lane % 32, half = lane / 32;
  const int wq = wave % WQ, wk = wave / WQ;
  const int head = blockIdx.y, index = a.index0 + blockIdx.x;
  Piece p;
  const bool any = locate<F::kRows, F::kKeys>(a, index, p);
  if (a.split && head == 0 && tid == 0)
    a.meta[index] = any && p.index == 0 && p.splits > 1 ? make_int4(p.req, p.row0, p.rows, p.splits) : make_int4(0, 0, 0, 0);
  if (!any) return;
  const int d = a.c.head_dim, G = a.group.d;

  // the row of this lane: its token, its query head, the keys it sees
  const int row = p.row0 + wq * 32 + n;
  const bool real = row < p.row0 + p.rows;
  const int tok = real ? int(a.group.of(row)) : 0;
  const int64_t qh = int64_t(head) * G + (real ? row - tok * G : 0);
  const auto seen = [&](int t, int64_t& lo, int64_t& hi) {    // by token t of the request
    const int64_t here = int64_t(p.kv) - p.len + t;
    hi = a.io.causal && here < p.kv - 1 ? here : p.kv - 1;
    lo = a.io.window > 0 && here - a.io.window >= 0 ? here - a.io.window + 1 : 0;
  };
  int64_t lo64, hi64, first_lo, first_hi, last_lo, last_hi;
  seen(tok, lo64, hi64);
  seen(int(a.group.of(p.row0)), first_lo, first_hi);
  seen(int(a.group.of(p.row0 + p.rows - 1)), last_lo, last_hi);
  // rows that pad the tile see everything and are not written
  const int lo = real ? int(lo64 > INT32_MAX ? INT32_MAX : lo64) : 0;
  const int hi = real ? int(hi64 < -1 ? -1 : hi64) : INT32_MAX;
  int all_lo = lo, all_hi = hi;                  // what every row of the wave sees
#pragma unroll
  for (int s = 1; s < 32; s *= 2) {
    const int x = __shfl_xor(all_lo, s), y = __shfl_xor(all_hi, s);
    all_lo = x > all_lo ? x : all_lo;
    all_hi = y < all_hi ? y : all_hi;
  }
  all_lo = __builtin_amdgcn_readfirstlane(all_lo);
  all_hi = __builtin_amdgcn_readfirstlane(all_hi);
  // this piece's steps: of the tile's range, the part `index`
  const int64_t begin = first_lo / F::kKeys, end = last_hi < first_lo ? begin : last_hi / F::kKeys + 1;
  const int step0 = int(begin + (end - begin) * p.index / p.splits);
  const int step1 = int(begin + (end - begin) * (p.index + 1) / p.splits);

  x8 q[kSteps];
  const elem* qrow = static_cast<const elem*>(a.io.q) + (int64_t(p.tok0) + tok) * a.io.q_tok + qh * a.io.q_head;
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int at = 16 * s + 8 * half;
    u32x4 v = {0, 0, 0, 0};
    if (real && at < d) v = *reinterpret_cast<const u32x4*>(qrow + at);
    q[s] = __builtin_bit_cast(x8, v);
  }
  f32x16 o[kDt];
#pragma unroll
  for (int i = 0; i < kDt; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0;
  float m = -__builtin_inff(), l = 0;

  const int32_t* table = a.io.block_table + int64_t(p.req) * a.io.table_req;
  const auto page_of = [&](int key) {            // -1: none
    if (key >= p.kv) return -1;
    const int b = table[a.page.of(key)];
    return b >= 0 && b < a.c.n_pages ? b : -1;
  };
  const elem* const kc = static_cast<const elem*>(a.c.k) + head * a.c.k_head;
  const elem* const vc = static_cast<const elem*>(a.c.v) + head * a.c.v_head;

  for (int step = step0; step < step1; ++step) {
    const int key0 = step * F::kKeys;
    u32x4 kr[F::kLoads], vr[F::kLoads];
    bool odd = false;
#pragma unroll
    for (int i = 0; i < F::kLoads; ++i) {
      const int at = i * F::kThreads + tid, r = at / F::kChunks, c = at % F::kChunks, key = key0 + r;
      const int64_t b = page_of(key), off = key - int(a.page.of(key) * a.page.d);
      kr[i] = u32x4{0, 0, 0, 0};
      vr[i] = u32x4{0, 0, 0, 0};
      if (b >= 0 && c * 8 < d) {
        kr[i] = *reinterpret_cast<const u32x4*>(kc + b * a.c.k_page + off * a.c.k_tok + c * 8);
        vr[i] = *reinterpret_cast<const u32x4*>(vc + b * a.c.v_page + off * a.c.v_tok + c * 8);
      }
      odd |= odd_value<T>(vr[i]);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < F::kLoads; ++i) {
      const int at = i * F::kThreads + tid, r = at / F::kChunks, c = at % F::kChunks;
      *reinterpret_cast<u32x4*>(lk + r * F::kRowBytes + key_chunk(r, c) * 16) = kr[i];
      *reinterpret_cast<u32x4*>(lv + r * F::kRowBytes + value_chunk<D>(r, c) * 16) = vr[i];
    }
    // whether some row of the block does not see some position of the step
    const bool cut = key0 < last_lo || key0 + F::kKeys - 1 > first_hi;
    const bool watch = __syncthreads_or(odd) && cut;

    const int wkey = key0 + wk * KW;             // this wave's keys
    const uint64_t have = __ballot(lane < KW && page_of(wkey + lane) >= 0);
    const bool masked = have != (KW == 64 ? ~uint64_t(0) : (uint64_t(1) << KW) - 1) || wkey < all_lo ||
                        wkey + KW - 1 > all_hi;
    f32x16 s[kSub];
#pragma unroll
    for (int t = 0; t < kSub; ++t) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[t][e] = 0;
      const int r = wk * KW + t * 32 + n;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const x8 k = *reinterpret_cast<const x8*>(lk + r * F::kRowBytes + key_chunk(r, 2 * i + half) * 16);
        s[t] = T::mfma(k, q[i], s[t]);
      }
    }
#pragma unroll
    for (int t = 0; t < kSub; ++t) settle(s[t]);
    const auto visible = [&](int t, int e) {     // key of element e of s[t]
      const int i = t * 32 + 8 * (e / 4) + 4 * half + e % 4;
      return (have >> i & 1) && wkey + i >= lo && wkey + i <= hi;
    };
    if (masked) {
#pragma unroll
      for (int t = 0; t < kSub; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[t][e] = visible(t, e) ? s[t][e] : -__builtin_inff();
    }
    float top = -__builtin_inff();
#pragma unroll
    for (int t = 0; t < kSub; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, s[t][e]);
    top = fmaxf(top, __shfl_xor(top, 32));
    const float next = fmaxf(m, top * a.scale2);
    const float base = next > -__builtin_inff() ? next : 0.0f;
    const float shrink = __builtin_amdgcn_exp2f(m - base);
    m = next;
    float sum = 0;
#pragma unroll
    for (int t = 0; t < kSub; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[t][e] = __builtin_amdgcn_exp2f(fmaf(s[t][e], a.scale2, -base));
        sum += s[t][e];
      }
    l = l * shrink + sum;
#pragma unroll
    for (int i = 0; i < kDt; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[i][e] *= shrink;
    if (watch) {
      // the products one by one, 16 keys at a time, without those that are not seen (weight -1)
      float* const w = reinterpret_cast<float*>(lds + 2 * F::kKv) + wave * 16 * 32;
#pragma unroll
      for (int t = 0; t < kSub; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          dasc_wy::wave_lds_sync();
#pragma unroll
          for (int e = 0; e < 8; ++e)
            w[(8 * (e / 4) + 4 * half + e % 4) * 32 + n] = visible(t, 8 * u + e) ? s[t][8 * u + e] : -1.0f;
          dasc_wy::wave_lds_sync();
          for (int k = 0; k < 16; ++k) {
            const float x = w[k * 32 + n];
            const int r = wk * KW + t * 32 + u * 16 + k;
            if (!(x < 0.0f))
#pragma unroll
              for (int i = 0; i < kDt; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                  const int c = i * 32 + 8 * (e / 4) + 4 * half + e % 4;
                  const elem v = *reinterpret_cast<const elem*>(lv + r * F::kRowBytes + value_chunk<D>(r, c / 8) * 16 + c % 8 * 2);
                  o[i][e] = fmaf(x, float(v), o[i][e]);
                }
          }
        }
    } else {
#pragma unroll
      for (int t = 0; t < kSub; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          x8 w;
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e] = elem(s[t][8 * u + e]);
          // rows of the transposing read: this lane's place in four keys of 16 columns
          const int r = wk * KW + t * 32 + u * 16 + 4 * half + lane % 16 / 4;
#pragma unroll
          for (int i = 0; i < kDt; ++i) {
            const int c = i * 32 + lane % 32 / 16 * 16 + lane % 4 * 4;
            union { s16x4 h[2]; x8 v; } x;
            x.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lv + r * F::kRowBytes + value_chunk<D>(r, c / 8) * 16 + c % 8 * 2));
            x.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lv + (r + 8) * F::kRowBytes + value_chunk<D>(r + 8, c / 8) * 16 + c % 8 * 2));
            o[i] = T::mfma(x.v, w, o[i]);
          }
        }
    }
#pragma unroll
    for (int i = 0; i < kDt; ++i) settle(o[i]);
  }
  l += __shfl_xor(l, 32);

  // waves that share rows meet in LDS
  if constexpr (WK > 1) {
    __syncthreads();
    float* const mine = reinterpret_cast<float*>(lds) + ((wk - 1) * WQ + wq) * 32 * (D + 2);
    if (wk > 0) {
      if (half == 0) {
        mine[n * 2] = m;
        mine[n * 2 + 1] = l;
      }
#pragma unroll
      for (int i = 0; i < kDt; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) mine[64 + (i * 16 + e) * 64 + lane] = o[i][e];
    }
    __syncthreads();
    if (wk > 0) return;
    for (int w = 1; w < WK; ++w) {
      const float* const other = reinterpret_cast<const float*>(lds) + ((w - 1) * WQ + wq) * 32 * (D + 2);
      const float om = other[n * 2], ol = other[n * 2 + 1];
      const float next = fmaxf(m, om), base = next > -__builtin_inff() ? next : 0.0f;
      const float f = __builtin_amdgcn_exp2f(m - base), g = __builtin_amdgcn_exp2f(om - base);
      m = next;
      l = l * f + ol * g;
#pragma unroll
      for (int i = 0; i < kDt; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] = o[i][e] * f + other[64 + (i * 16 + e) * 64 + lane] * g;
    }
  }
  if (!real) return;
  if (p.splits > 1) {
    const int64_t slot = (int64_t(index) * gridDim.y + head) * F::kRows + wq * 32 + n;
    if (half == 0) {
      a.ml[slot * 2] = m;
      a.ml[slot * 2 + 1] = l;
    }
    float* out = a.part + slot * D;
#pragma unroll
    for (int i = 0; i < kDt; ++i)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int c = i * 32 + 8 * b + 4 * half;
        *reinterpret_cast<float4*>(out + c) = make_float4(o[i][4 * b], o[i][4 * b + 1], o[i][4 * b + 2], o[i][4 * b + 3]);
      }
    return;
  }
  const int64_t t = int64_t(p.tok0) + tok;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  elem* out = static_cast<elem*>(a.io.o) + t * a.io.o_tok + qh * a.io.o_head;
  typedef elem e4 __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int i = 0; i < kDt; ++i)
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int c = i * 32 + 8 * b + 4 * half;
      e4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = elem(o[i][4 * b + e] * inv);
      if (c < d) *reinterpret_cast<e4*>(out + c) = x;
    }
  if (a.io.lse && half == 0)
    a.io.lse[t * a.io.lse_tok + qh * a.io.lse_head] = m * 0.69314718056f + logf(l);
}

// The pieces of a split tile: o = sum 2^(m_i - m) O_i / sum 2^(m_i - m) l_i
template <typename T, int D, int ROWS>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a) {
  typedef typename T::elem elem;
  constexpr int kLanes = D / 4;                  // of a row
  const int index = a.index0 + blockIdx.x, head = blockIdx.y, heads = gridDim.y;
  const int4 t = a.meta[index];                  // request, first row, rows, pieces
  if (t.w < 2) return;
  const int c = threadIdx.x % kLanes * 4, n = int(a.io.n_tokens), G = a.group.d;
  int tok0 = a.io.cu_seqlens[t.x];
  tok0 = tok0 < 0 ? 0 : tok0 > n ? n : tok0;
  for (int r = threadIdx.x / kLanes; r < t.z; r += 256 / kLanes) {
    const auto slot = [&](int i) { return (int64_t(index + i) * heads + head) * ROWS + r; };
    float m = -__builtin_inff(), l = 0;
    for (int i = 0; i < t.w; ++i) m = fmaxf(m, a.ml[slot(i) * 2]);
    const float base = m > -__builtin_inff() ? m : 0.0f;
    float4 o = make_float4(0, 0, 0, 0);
    for (int i = 0; i < t.w; ++i) {
      const float f = __builtin_amdgcn_exp2f(a.ml[slot(i) * 2] - base);
      const float4 x = *reinterpret_cast<const float4*>(a.part + slot(i) * D + c);
      l += f * a.ml[slot(i) * 2 + 1];
      o.x = fmaf(f, x.x, o.x);
      o.y = fmaf(f, x.y, o.y);
      o.z = fmaf(f, x.z, o.z);
      o.w = fmaf(f, x.w, o.w);
    }
    const int tok = int(a.group.of(t.y + r)), qh = head * G + t.y + r - tok * G;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    typedef elem e4 __attribute__((ext_vector_type(4)));
    const e4 x = {elem(o.x * inv), elem(o.y * inv), elem(o.z * inv), elem(o.w * inv)};
    const int64_t at = int64_t(tok0) + tok;
    if (c < a.c.head_dim)
      *reinterpret_cast<e4*>(static_cast<elem*>(a.io.o) + at * a.io.o_tok + qh * a.io.o_head + c) = x;
    if (a.io.lse && c == 0) a.io.lse[at * a.io.lse_tok + qh * a.io.lse_head] = m * 0.69314718056f + logf(l);
  }
}

// ---- launches -----------------------------------------------------------------------------------

// How a call runs: the form by the rows of its longest request, pieces by the tiles that it can have
struct Launch {
  int rows, keys;                // of a tile and a step
  int64_t pieces;                // of a key head, at most
  bool split;
  int target;
};

constexpr float kLog2e = 1.44269504089f;
constexpr int kBlocks = 512;     // that a split call aims at

Launch launch_of(int n_req, int64_t n_tokens, int group, int n_kv_heads, int head_dim, int max_len, int max_kv) {
  Launch x;
  const int64_t most = n_tokens < max_len ? n_tokens : max_len;
  const int64_t rows = most * group;
  x.rows = rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
  const int wk = x.rows == 32 ? (head_dim > 128 ? 2 : 4) : x.rows == 64 ? 2 : 1;
  x.keys = wk * (x.rows == 128 && head_dim <= 128 ? 64 : 32);
  const int64_t tiles = n_tokens * group / x.rows + n_req;
  x.target = kBlocks / n_kv_heads;
  if (x.target < 1) x.target = 1;
  x.split = tiles < 2 * x.target && max_kv > kMinSteps * x.keys;
  x.pieces = x.split ? tiles + x.target : tiles;
  return x;
}

int dim_of(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }

template <typename T, int D, int WQ, int WK, int KW>
void launch_form(AttnArgs a, const Launch& x, hipStream_t st) {
  constexpr int64_t kMost = int64_t(1) << 21;     // a grid counts threads in 32 bits
  const auto grid = [&](int64_t i) {
    a.index0 = int32_t(i);
    return dim3(uint32_t(x.pieces - i < kMost ? x.pieces - i : kMost), a.c.n_kv_heads);
  };
  for (int64_t i = 0; i < x.pieces; i += kMost) {
    const dim3 g = grid(i);
    attn_kernel<T, D, WQ, WK, KW><<<g, 64 * WQ * WK, 0, st>>>(a);
  }
  if (x.split) attn_join_kernel<T, D, 32 * WQ><<<grid(0), 256, 0, st>>>(a);   // few pieces
}

template <typename T, int D>
void launch_rows(const AttnArgs& a, const Launch& x, hipStream_t st) {
  if (x.rows == 32) launch_form<T, D, 1, D == 256 ? 2 : 4, 32>(a, x, st);
  else if (x.rows == 64) launch_form<T, D, 2, 2, 32>(a, x, st);
  else launch_form<T, D, 4, 1, D == 256 ? 32 : 64>(a, x, st);
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
  int target = kBlocks / n_kv_heads;
  if (target < 1) target = 1;
  for (const int rows : {32, 64, 128}) {
    if (int64_t(rows) / 2 >= int64_t(max_len) * group && rows > 32) continue;   // no request fills it
    int64_t tiles = n_tokens * group / rows + n_req;
    if (tiles > 2 * target) tiles = 2 * target;
    const int64_t pieces = tiles + target;
    const int64_t need = pieces * 16 + pieces * n_kv_heads * rows * (D + 2) * 4;
    if (size_t(need) > *bytes) *bytes = size_t(need);
  }
  if (max_kv <= kMinSteps * 32) *bytes = 0;
  return DASC_OK;
}

extern "C" int dasc_cache_attn(const dasc_kv_cache* cache, const dasc_attn_io* io, void* workspace,
                               size_t workspace_bytes, dasc_stream_t stream) {
  using namespace dasc;
  if (!io) return DASC_E_INVAL;
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
                             io->max_kv < most ? io->max_kv : most);
  AttnArgs a;
  a.c = *cache;
  a.io = *io;
  a.group = divisor(group);
  a.page = divisor(cache->page_size);
  a.target = x.target;
  a.split = x.split;
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

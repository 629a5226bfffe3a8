// Beam search: the best continuations over beams and vocabulary, and pool slots reordered after them.
//
// A candidate's score is its beam's score plus the logit less the row's log-sum of exponentials, in 64-bit
// arithmetic: the order of two candidates of different beams then does not hang on how a sum was rounded.
// Within a row the order is that of the logits, so a row's tiles each give their n_out best logits and
// their part of the sum, and one block per request merges them: first each beam's lists, then the beams'.
//
// The best n of a tile (logit and token in one 64-bit key, all different) without sorting it: every lane takes its
// largest logit; n lanes of a wave have one at or above the n-th largest of those, so at least n of the tile lie at
// or above it.  That is found bit by bit with ballots; what is at or above the largest of the waves' is
// gathered in LDS, a few times n as a rule, and ranked by comparing all with all.
//
// Measured: 16 requests of eight beams over 131071 bf16 tokens, 16 of each: 33 us for the rows, of which the 64-bit
// exponentials are about half (34 MB would take 7), and 13.5 for the merge, a chain of short loops in one block a request.
// Slots: HBM bounds them; eight states of 2 MB in each of 16 groups, 109 MB
// read and 268 written in 88 us (4.3 TB/s).

#include <hip/hip_runtime.h>

#include <cstdint>

#include "cache_common.h"
#include "launch_common.h"
#include "row_io.h"
#include "wy_ops.h"

namespace dasc {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = kThreads * 16;      // tokens of a block
constexpr int kMaxBeams = 64, kMaxOut = 64;
constexpr int64_t kMaxVocab = int64_t(1) << 24;
constexpr int64_t kMaxRows = int64_t(1) << 24;
constexpr int kPickWaves = 8, kPickKeys = 10;   // waves of a request's block, keys of a lane

struct BeamArgs {
  const void* logits;
  int64_t logits_req, logits_beam;
  const float* scores;
  const int32_t* slots;
  float* out_scores;
  int32_t *out_tokens, *out_parents, *out_slots;
  double* sums;          // [rows, tiles]: of e^(x - max), NaN if the tile holds NaN or +inf
  float* tops;           // [rows, tiles]: max
  uint64_t* keys;        // [rows, tiles, n_out], descending, 0: none
  int64_t row0;          // first row (scan), or request (pick), of a launch
  int32_t n_req, beams, vocab, n_out, tiles;
};

// Whole numbers in the order of the floats; 0 is below all of them.  -0 counts as 0.
__device__ inline uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float unordered(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}
__device__ inline uint64_t key_of(float x, uint32_t token) { return (uint64_t(ordered(x)) << 32) | (0xFFFFFFFFu - token); }
__device__ inline uint32_t token_of(uint64_t key) { return 0xFFFFFFFFu - uint32_t(key); }

// The largest number that at least n of the wave's keys reach (0 if fewer than n are not 0), bit by bit; of
// different keys just n reach it.
__device__ inline uint32_t reached_by(uint32_t key, int n) {
  if (__popcll(__ballot(key != 0)) < n) return 0;
  uint32_t all = key, any = key;
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    all &= uint32_t(__shfl_xor(int(all), s));
    any |= uint32_t(__shfl_xor(int(any), s));
  }
  const uint32_t differ = all ^ any;      // from the first bit in which they differ
  if (differ == 0) return all;
  int bit = 31 - __builtin_clz(differ);
  uint32_t t = bit < 31 ? any >> (bit + 1) << (bit + 1) : 0;
  for (; bit >= 0; --bit) {
    const uint32_t x = t | (1u << bit);
    const int c = __popcll(__ballot(key >= x));
    if (c >= n) t = x;
    if (c == n) break;
  }
  return t;
}
__device__ inline uint64_t reached_by(uint64_t key, int n) {
  const uint32_t hi = uint32_t(key >> 32), t = reached_by(hi, n);
  if (t == 0) return 0;
  const int above = __popcll(__ballot(hi > t));           // the lower half decides between those that are equal
  const uint32_t lo = reached_by(hi == t ? uint32_t(key) : 0u, n - above);
  return (uint64_t(t) << 32) | (__popcll(__ballot(hi >= t)) == n ? 0u : lo);
}

// e^x for x <= 0 in 64 bits, to 2^-36: 2^n e^r with r at most ln 2 / 2, the exponential's series to r^9 / 9!
// (the first term left out is below 2^-36 of the sum, and n ln 2 good to 2^-43)
__device__ inline double exp64(double x) {
  const double n = rint(x * 1.4426950408889634074);
  const double r = fma(n, -0.69314718055994530942, x);
  double p = 1.0 / 362880.0;
  p = fma(p, r, 1.0 / 40320.0);
  p = fma(p, r, 1.0 / 5040.0);
  p = fma(p, r, 1.0 / 720.0);
  p = fma(p, r, 1.0 / 120.0);
  p = fma(p, r, 1.0 / 24.0);
  p = fma(p, r, 1.0 / 6.0);
  p = fma(p, r, 0.5);
  p = fma(p, r, 1.0);
  p = fma(p, r, 1.0);
  return __builtin_amdgcn_ldexp(p, n > -2000.0 ? int(n) : -2000);
}

constexpr int kRanked = 512;             // keys that are ranked at most

// The block's n-th largest key, bit by bit, the block counting: for tiles with many equal logits, or with the large
// ones in a few lanes.  keys: of this thread, all different.
template <int N>
__device__ inline uint64_t block_reached_by(const uint64_t (&keys)[N], int n, int* count) {
  uint64_t t = 0;
  for (int bit = 63; bit >= 0; --bit) {
    const uint64_t x = t | (uint64_t(1) << bit);
    __syncthreads();
    if (threadIdx.x == 0) *count = 0;
    __syncthreads();
    int some = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) some += __popcll(__ballot(keys[i] >= x));
    if (threadIdx.x % 64 == 0 && some) atomicAdd(count, some);
    __syncthreads();
    const int c = *count;
    if (c >= n) t = x;
    if (c == n) break;
  }
  return t;
}

// A tile of a row: its largest logit, the sum of exponentials against it, its n_out best keys.
template <typename T>
__global__ __launch_bounds__(kThreads) void beam_scan_kernel(BeamArgs a) {
  __shared__ uint64_t list[kRanked];
  __shared__ uint32_t limit[kThreads / 64];
  __shared__ float top[kThreads / 64];
  __shared__ double part[kThreads / 64];
  __shared__ int count;
  const int tid = threadIdx.x, wave = tid / 64;
  const int64_t r = a.row0 + blockIdx.y;
  const T* row = static_cast<const T*>(a.logits) + r / a.beams * a.logits_req + r % a.beams * a.logits_beam;
  const int base = blockIdx.x * kTile + tid * 8;
  float x[16];
  load_vec<8>(row, base, a.vocab, x);
  load_vec<8>(row, base + kTile / 2, a.vocab, x + 8);
  const float inf = __builtin_inff();
  bool bad = false;
  float m = -inf;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int token = base + i % 8 + i / 8 * (kTile / 2);
    if (token >= a.vocab) x[i] = -inf;
    bad |= !(x[i] < inf);                              // +inf and NaN
    if (!(x[i] < inf)) x[i] = -inf;
    m = fmaxf(m, x[i]);
  }
  // n_out lanes of a wave have a logit at or above its floor, so the block has n_out at or above each
  const uint32_t t = reached_by(m > -inf ? ordered(m) : 0u, a.n_out);
  float wm = m;
#pragma unroll
  for (int s = 1; s < 64; s *= 2) wm = fmaxf(wm, __shfl_xor(wm, s));
  if (tid % 64 == 0) limit[wave] = t, top[wave] = wm;
  if (tid == 0) count = 0;
  __syncthreads();
  uint32_t low = ordered(-inf) + 1;
  float bm = -inf;
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) {
    low = limit[i] > low ? limit[i] : low;
    bm = fmaxf(bm, top[i]);
  }
  if (ordered(m) >= low) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (ordered(x[i]) >= low) {
        const int at = atomicAdd(&count, 1);
        if (at < kRanked) list[at] = key_of(x[i], base + i % 8 + i / 8 * (kTile / 2));
      }
  }
  double sum = bad ? __longlong_as_double(0x7FF8000000000000) : 0.0;
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (x[i] > -inf) sum += exp64(double(x[i]) - double(bm));
#pragma unroll
  for (int s = 1; s < 64; s *= 2) sum += __shfl_xor(sum, s);
  if (tid % 64 == 0) part[wave] = sum;
  __syncthreads();
  const int64_t at = r * a.tiles + blockIdx.x;
  if (tid == 0) {
    double all = 0;
    for (int i = 0; i < kThreads / 64; ++i) all += part[i];
    a.sums[at] = all;
    a.tops[at] = bm;
  }
  int c = count;
  uint64_t* out = a.keys + at * a.n_out;
  if (c > kRanked) {                       // more than fit: the n_out best alone
    uint64_t keys[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) keys[i] = x[i] > -inf ? key_of(x[i], base + i % 8 + i / 8 * (kTile / 2)) : 0;
    const uint64_t last = block_reached_by(keys, a.n_out, &count);
    __syncthreads();
    if (tid == 0) count = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (keys[i] >= last) list[atomicAdd(&count, 1)] = keys[i];
    __syncthreads();
    c = count;
  }
  for (int i = tid; i < c; i += kThreads) {
    const uint64_t key = list[i];
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < c; ++j) rank += list[j] > key;
    if (rank < a.n_out) out[rank] = key;
  }
  for (int i = c + tid; i < a.n_out; i += kThreads) out[i] = 0;
}

__device__ inline uint64_t ordered64(double x) {
  const uint64_t b = uint64_t(__double_as_longlong(x + 0.0));
  return b >> 63 ? ~b : b | (uint64_t(1) << 63);
}
__device__ inline double unordered64(uint64_t k) {
  return __longlong_as_double(k >> 63 ? int64_t(k & ~(uint64_t(1) << 63)) : int64_t(~k));
}

__global__ __launch_bounds__(kPickWaves * 64) void beam_pick_kernel(BeamArgs a) {
  __shared__ uint64_t list[kPickWaves][64 * kPickKeys], top[kPickWaves][64];
  __shared__ uint64_t score[kMaxBeams * kMaxOut], logit[kMaxBeams * kMaxOut];   // of each beam's best
  const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64, n = a.n_out;
  const int r = int(a.row0) + blockIdx.x;                  // the request
  for (int b = wave; b < a.beams; b += kPickWaves) {
    const int64_t row = int64_t(r) * a.beams + b;
    // the row's log-sum
    const float* tops = a.tops + row * a.tiles;
    const double* sums = a.sums + row * a.tiles;
    float m = -__builtin_inff();
    for (int i = lane; i < a.tiles; i += 64) m = fmaxf(m, tops[i]);
#pragma unroll
    for (int s = 1; s < 64; s *= 2) m = fmaxf(m, __shfl_xor(m, s));
    double sum = 0;
    for (int i = lane; i < a.tiles; i += 64)
      sum += sums[i] * (tops[i] > -__builtin_inff() ? exp64(double(tops[i]) - double(m)) : 1.0);
#pragma unroll
    for (int s = 1; s < 64; s *= 2) sum += __shfl_xor(sum, s);
    const double lse = double(m) + log(sum);
    const double start = double(a.scores[row]);
    // the n best of its tiles' lists, carried from step to step in the wave's list
    uint64_t* mine = list[wave];
    const uint64_t* keys = a.keys + row * a.tiles * n;
    const int total = a.tiles * n;
    uint64_t carried = 0;
    for (int at = 0; at < total; at += 64 * (kPickKeys - 1)) {
      uint64_t k[kPickKeys], best = carried;
      k[0] = carried;
#pragma unroll
      for (int i = 1; i < kPickKeys; ++i) {
        const int j = at + (i - 1) * 64 + lane;
        k[i] = j < total ? keys[j] : 0;
        best = k[i] > best ? k[i] : best;
      }
      uint64_t t = reached_by(best, n);
      if (t == 0) t = 1;
      int c = 0;
#pragma unroll
      for (int i = 0; i < kPickKeys; ++i) {
        const uint64_t in = __ballot(k[i] >= t);
        if (k[i] >= t) mine[c + __popcll(in & ((uint64_t(1) << lane) - 1))] = k[i];
        c += __popcll(in);
      }
      dasc_wy::wave_lds_sync();
      for (int i = lane; i < c; i += 64) {          // ranked, a key a lane
        const uint64_t key = mine[i];
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < c; ++j) rank += mine[j] > key;
        if (rank < n) top[wave][rank] = key;
      }
      dasc_wy::wave_lds_sync();
      carried = lane < n && lane < c ? top[wave][lane] : 0;
    }
    const bool live = start > -__builtin_inf() && start < __builtin_inf() && lse == lse;
    if (lane < n) {
      const double s = start + (double(unordered(uint32_t(carried >> 32))) - lse);
      const bool ok = live && carried != 0;
      score[b * n + lane] = ok ? ordered64(s) : 0;
      logit[b * n + lane] = ok ? carried : 0;
    }
  }
  __syncthreads();
  // all beams' best, ranked: by score, then the lower beam, then by logit and token
  const int total = a.beams * n;
  int valid = 0;
  int parts = 1;                                   // threads that share a candidate's comparisons
  while (parts < 16 && total * parts * 2 <= kPickWaves * 64) parts *= 2;
  for (int i0 = 0; i0 < total; i0 += kPickWaves * 64 / parts) {
    const int i = i0 + tid / parts, part = tid % parts;
    const uint64_t s = i < total ? score[i] : 0;
    int rank = 0;
    if (s != 0) {
#pragma unroll 8
      for (int j = part; j < total; j += parts) {
        const uint64_t o = score[j];
        if (o > s || (o == s && j < i)) ++rank;    // a beam's list is in order of logit and token
      }
    }
    for (int m = 1; m < parts; m *= 2) rank += __shfl_xor(rank, m);
    if (s != 0 && part == 0 && rank < n) {
      const int64_t out = int64_t(r) * n + rank;
      const int b = i / n;
      a.out_scores[out] = float(unordered64(s));
      a.out_tokens[out] = int32_t(token_of(logit[i]));
      a.out_parents[out] = b;
      if (a.out_slots) a.out_slots[out] = a.slots[int64_t(r) * a.beams + b];
    }
  }
  // places left over
  for (int j = lane; j < total; j += 64) valid += score[j] != 0;
#pragma unroll
  for (int s = 1; s < 64; s *= 2) valid += __shfl_xor(valid, s);
  if (tid < n && tid >= valid) {
    const int64_t out = int64_t(r) * n + tid;
    a.out_scores[out] = -__builtin_inff();
    a.out_tokens[out] = a.out_parents[out] = -1;
    if (a.out_slots) a.out_slots[out] = -1;
  }
}

constexpr int kRowsPerLaunch = 32768;   // a grid's second dimension

template <typename T>
void launch_scan(BeamArgs a, hipStream_t st) {
  const int64_t rows = int64_t(a.n_req) * a.beams;
  for (a.row0 = 0; a.row0 < rows; a.row0 += kRowsPerLaunch) {
    const int64_t left = rows - a.row0;
    beam_scan_kernel<T><<<dim3(a.tiles, uint32_t(left < kRowsPerLaunch ? left : kRowsPerLaunch)), kThreads, 0, st>>>(a);
  }
}

// ---- slots ------------------------------------------------------------------------------------

struct MoveArgs {
  char* pool;
  int64_t n_slots, stride, words;      // words of V in a slot
  const int32_t *src, *dst;
  int64_t src_group, dst_group;
  int32_t m;
};

// A thread has one word of every slot of a group: it loads all of them, then stores all of them, so no order
// of the moves matters.  The indices are the same for a wave, so that the addresses take no vector registers.
template <typename V, int M>
__global__ __launch_bounds__(256) void move_kernel(MoveArgs a) {
  const uint32_t w = blockIdx.x * 256 + threadIdx.x;
  if (w >= a.words) return;
  typedef const __attribute__((address_space(4))) int32_t* list_t;
  const list_t src = list_t(uintptr_t(a.src + blockIdx.y * a.src_group)), dst = list_t(uintptr_t(a.dst + blockIdx.y * a.dst_group));
  const auto moved = [&](int j) {
    const int s = src[j], d = dst[j];
    return s >= 0 && s < a.n_slots && d >= 0 && d < a.n_slots && s != d;
  };
  V x[M];
#pragma unroll
  for (int j = 0; j < M; ++j)
    if (j < a.m && moved(j)) x[j] = reinterpret_cast<const V*>(a.pool + src[j] * a.stride)[w];
#pragma unroll
  for (int j = 0; j < M; ++j)
    if (j < a.m && moved(j)) __builtin_nontemporal_store(x[j], reinterpret_cast<V*>(a.pool + dst[j] * a.stride) + w);
}

template <typename V, int M>
void launch_move(MoveArgs a, int64_t bytes, int groups, hipStream_t st) {
  constexpr int64_t kBlocks = int64_t(1) << 20;
  const int64_t words = bytes / int64_t(sizeof(V));
  char* pool = a.pool;
  for (int64_t w0 = 0; w0 < words; w0 += kBlocks * 256) {
    a.pool = pool + w0 * int64_t(sizeof(V));
    a.words = words - w0 < kBlocks * 256 ? words - w0 : kBlocks * 256;
    move_kernel<V, M><<<dim3(uint32_t((a.words + 255) / 256), groups), 256, 0, st>>>(a);
  }
}

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

int64_t tiles_of(int64_t vocab) { return (vocab + kTile - 1) / kTile; }

bool beam_shape(int64_t n_req, int64_t beams, int64_t vocab, int64_t n_out) {
  return n_req >= 0 && beams >= 1 && beams <= kMaxBeams && n_out >= 1 && n_out <= kMaxOut && vocab >= 1 &&
         vocab <= kMaxVocab && n_req * beams <= kMaxRows;
}

}  // namespace
}  // namespace dasc

extern "C" int dasc_beam_select_workspace_bytes(int32_t n_req, int32_t beams, int64_t vocab, int32_t n_out,
                                                size_t* bytes) {
  using namespace dasc;
  if (!bytes) return DASC_E_INVAL;
  if (!beam_shape(n_req, beams, vocab, n_out)) return DASC_E_SHAPE;
  *bytes = size_t(n_req) * beams * tiles_of(vocab) * (n_out * sizeof(uint64_t) + sizeof(double) + sizeof(float));
  return DASC_OK;
}

extern "C" int dasc_beam_select(int32_t n_req, int32_t beams, int64_t vocab, int32_t n_out, int32_t dtype,
                                const void* logits, int64_t logits_req, int64_t logits_beam, const float* scores,
                                const int32_t* slots, float* out_scores, int32_t* out_tokens, int32_t* out_parents,
                                int32_t* out_slots, void* workspace, size_t workspace_bytes, dasc_stream_t stream) {
  using namespace dasc;
  if (dtype != DASC_DTYPE_BF16 && dtype != DASC_DTYPE_F16 && dtype != DASC_DTYPE_F32) return DASC_E_INVAL;
  if (!beam_shape(n_req, beams, vocab, n_out)) return DASC_E_SHAPE;
  if (n_req == 0) return DASC_OK;
  if (!logits || !scores || !out_scores || !out_tokens || !out_parents) return DASC_E_INVAL;
  if ((slots != nullptr) != (out_slots != nullptr)) return DASC_E_INVAL;
  if (!aligned_to(logits, dtype == DASC_DTYPE_F32 ? 4 : 2) || logits_req < 0 || logits_beam < 0) return DASC_E_INVAL;
  for (const void* p : {static_cast<const void*>(scores), static_cast<const void*>(slots),
                        static_cast<const void*>(out_scores), static_cast<const void*>(out_tokens),
                        static_cast<const void*>(out_parents), static_cast<const void*>(out_slots)})
    if (!aligned_to(p, 4)) return DASC_E_INVAL;
  size_t need = 0;
  (void)dasc_beam_select_workspace_bytes(n_req, beams, vocab, n_out, &need);
  if (workspace_bytes < need || !workspace) return DASC_E_WORKSPACE;
  if (!aligned_to(workspace, 16)) return DASC_E_INVAL;
  BeamArgs a;
  a.logits = logits;
  a.logits_req = logits_req;
  a.logits_beam = logits_beam;
  a.scores = scores;
  a.slots = slots;
  a.out_scores = out_scores;
  a.out_tokens = out_tokens;
  a.out_parents = out_parents;
  a.out_slots = out_slots;
  a.n_req = n_req;
  a.beams = beams;
  a.vocab = int32_t(vocab);
  a.n_out = n_out;
  a.tiles = int32_t(tiles_of(vocab));
  a.row0 = 0;
  const int64_t tiles = int64_t(n_req) * beams * a.tiles;
  a.keys = static_cast<uint64_t*>(workspace);
  a.sums = reinterpret_cast<double*>(a.keys + tiles * n_out);
  a.tops = reinterpret_cast<float*>(a.sums + tiles);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  switch (dtype) {
    case DASC_DTYPE_BF16: launch_scan<bf16_t>(a, st); break;
    case DASC_DTYPE_F16: launch_scan<f16_t>(a, st); break;
    default: launch_scan<float>(a, st); break;
  }
  constexpr int kReqPerLaunch = 1 << 20;   // a grid counts threads in 32 bits
  for (a.row0 = 0; a.row0 < n_req; a.row0 += kReqPerLaunch)
    beam_pick_kernel<<<n_req - a.row0 < kReqPerLaunch ? uint32_t(n_req - a.row0) : kReqPerLaunch, kPickWaves * 64, 0, st>>>(a);
  return launch_status();
}

extern "C" int dasc_move_slots(void* pool, int64_t n_slots, int64_t slot_bytes, int64_t slot_stride,
                               const int32_t* src, int64_t src_group, const int32_t* dst, int64_t dst_group,
                               int32_t groups, int32_t m, dasc_stream_t stream) {
  using namespace dasc;
  if (groups < 0 || groups > 65535 || m < 0 || m > kMaxBeams) return DASC_E_SHAPE;
  if (n_slots < 1 || slot_bytes < 16 || slot_bytes % 16 || slot_stride % 16 || slot_stride < slot_bytes ||
      src_group < 0 || dst_group < 0)
    return DASC_E_INVAL;
  if (groups == 0 || m == 0) return DASC_OK;
  if (!pool || !src || !dst || !aligned16(pool) || !aligned_to(src, 4) || !aligned_to(dst, 4)) return DASC_E_INVAL;
  MoveArgs a{static_cast<char*>(pool), n_slots, slot_stride, 0, src, dst, src_group, dst_group, m};
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (m <= 4) launch_move<u32x4, 4>(a, slot_bytes, groups, st);
  else if (m <= 8) launch_move<u32x4, 8>(a, slot_bytes, groups, st);
  else if (m <= 16) launch_move<u32x4, 16>(a, slot_bytes, groups, st);
  else if (m <= 32) launch_move<u32x2, 32>(a, slot_bytes, groups, st);
  else launch_move<uint32_t, 64>(a, slot_bytes, groups, st);
  return launch_status();
}

// Verification of drafted tokens: which of a request's drafts the target accepts, and the token
// drawn in place of the first that it does not (or after the last).
//
// The accept test reads two probabilities per draft; the draw needs one row of the target and
// one of the draft model, whose weights are whole numbers (floor(min(w, 1) 2^36)), so that a
// row is summed in any order with the same result.  A weight is held as two 18-bit halves,
// whose sums over a tile of 2048 stay in 32 bits.
//
// Two launches: every tile of a row sums its weights (and finds out for itself which row it is), then one
// block per request finds the tile that the drawn level falls in, and the token in the tile.  One block
// that does all of a request is slower even for 64 of them (34 us against 20: a compute unit alone reads
// its 512 KB at 15 GB/s).
//
// Measured: 64 requests x 131071 bf16 tokens, one row of each model: 12.7 + 4.5 us, the 34 MB at 2.6 TB/s; a
// request of 32000 fp32 tokens 5.2 + 3.4, two chains of dependent loads and a launch.

#include <hip/hip_runtime.h>

#include <cstdint>

#include "dasc/ops.h"
#include "launch_common.h"
#include "row_io.h"

namespace dasc {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = kThreads * 8;
constexpr int kTiles = 4;                  // of a block that sums
constexpr int64_t kMaxVocab = int64_t(1) << 24;
constexpr int kMaxDraft = 1023;

struct VerifyArgs {
  const void *target, *draft;
  int64_t target_req, target_pos, draft_req, draft_pos;
  const int32_t *tokens, *n_draft;
  const float *u_accept, *u_sample;
  int32_t *out, *emitted;
  uint64_t* sums;        // [n_req, tiles, 2]: of w, of p_a
  int32_t* kept;         // [n_req]: a
  int32_t max_draft, vocab, tiles, req0;
};

__device__ inline int drafts_of(const VerifyArgs& a, int r) {
  const int n = a.n_draft ? a.n_draft[r] : a.max_draft;
  return n < a.max_draft ? n : a.max_draft;
}

// drafts accepted before the first that is not; the same in every thread.  A draft and its number are
// asked for before n is known.
template <typename T>
__device__ inline int accepted(const VerifyArgs& a, int r, int& n) {
  __shared__ int first;
  const int tid = threadIdx.x;
  const int64_t row = int64_t(r) * a.max_draft;
  int x = -1;
  float u = 0;
  if (tid < a.max_draft) {
    x = a.tokens[row + tid];
    u = a.u_accept[row + tid];
  }
  n = drafts_of(a, r);
  if (tid == 0) first = n;
  __syncthreads();
  const T* p = static_cast<const T*>(a.target) + r * a.target_req;
  const T* q = a.draft ? static_cast<const T*>(a.draft) + r * a.draft_req : nullptr;
  for (int i = tid; i < n; i += kThreads) {
    if (i != tid) {
      x = a.tokens[row + i];
      u = a.u_accept[row + i];
    }
    bool ok = x >= 0 && x < a.vocab;
    if (ok) {
      const float qx = q ? widen(q[i * a.draft_pos + x]) : 1.0f;
      ok = __fmul_rn(u, qx) < widen(p[i * a.target_pos + x]);
    }
    if (!ok) atomicMin(&first, i);
  }
  __syncthreads();
  return first;
}

struct Halves { uint32_t hi, lo; };   // a weight is hi 2^18 + lo

__device__ inline Halves whole(float w) {
  w = w > 0.0f ? fminf(w, 1.0f) : 0.0f;              // NaN counts as nothing
  const float f = w * 262144.0f;                     // 2^18
  const uint32_t hi = uint32_t(f);
  return {hi, uint32_t((f - float(hi)) * 262144.0f)};
}

__device__ inline uint64_t value(Halves h) { return (uint64_t(h.hi) << 18) + h.lo; }

// the weights of tokens c .. c + 7 of request r, whose first `kept` drafts are kept
template <typename T>
__device__ inline void weights(const VerifyArgs& a, int r, int n, int kept, int c, bool residual,
                               float (&p)[8], float (&w)[8]) {
  const T* row = static_cast<const T*>(a.target) + r * a.target_req + kept * a.target_pos;
  load_vec<8>(row, c, a.vocab, p);
  if (!residual || kept >= n) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = p[i];
  } else if (a.draft) {
    const T* q = static_cast<const T*>(a.draft) + r * a.draft_req + kept * a.draft_pos;
    load_vec<8>(q, c, a.vocab, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = p[i] - w[i];
  } else {
    const int x = a.tokens[int64_t(r) * a.max_draft + kept];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = c + i == x ? 0.0f : p[i];
  }
}

template <int CTRL, int ROWS>
__device__ inline uint32_t add_lane(uint32_t x) {
  return x + uint32_t(__builtin_amdgcn_update_dpp(0, int(x), CTRL, ROWS, 0xF, true));
}
// the wave's sum, in lane 63
__device__ inline uint32_t wave_sum(uint32_t x) {
  x = add_lane<0x111, 0xF>(x);             // the lanes before it in a row of 16
  x = add_lane<0x112, 0xF>(x);
  x = add_lane<0x114, 0xF>(x);
  x = add_lane<0x118, 0xF>(x);
  x = add_lane<0x142, 0xA>(x);             // the last lane of the row before
  return add_lane<0x143, 0xC>(x);          // the last lane of the first half
}

template <typename T>
__global__ __launch_bounds__(kThreads) void verify_sums_kernel(VerifyArgs a) {
  const int r = a.req0 + blockIdx.y, tile0 = blockIdx.x * kTiles;
  int n;
  const int kept = accepted<T>(a, r, n);
  if (n < 0) return;
  if (tile0 == 0 && threadIdx.x == 0) a.kept[r] = kept;
  float p[kTiles][8], w[kTiles][8];
#pragma unroll
  for (int v = 0; v < kTiles; ++v)
    weights<T>(a, r, n, kept, (tile0 + v) * kTile + threadIdx.x * 8, true, p[v], w[v]);
  __shared__ uint32_t part[kThreads / 64][kTiles * 4];
#pragma unroll
  for (int v = 0; v < kTiles; ++v) {
    uint32_t s[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const Halves x = whole(w[v][i]), y = whole(p[v][i]);
      s[0] += x.hi;
      s[1] += x.lo;
      s[2] += y.hi;
      s[3] += y.lo;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      s[j] = wave_sum(s[j]);
      if (threadIdx.x % 64 == 63) part[threadIdx.x / 64][v * 4 + j] = s[j];
    }
  }
  __syncthreads();
  if (threadIdx.x < 2 * kTiles) {          // (tile, of w or of p)
    const int v = threadIdx.x / 2, j = 2 * threadIdx.x;
    Halves h = {0, 0};
#pragma unroll
    for (int i = 0; i < kThreads / 64; ++i) {
      h.hi += part[i][j];
      h.lo += part[i][j + 1];
    }
    if (tile0 + v < a.tiles) a.sums[(int64_t(r) * a.tiles + tile0) * 2 + threadIdx.x] = value(h);
  }
}

// inclusive prefix sum over the block; total: the block's
__device__ inline uint64_t block_scan(uint64_t x, uint64_t& total) {
  __shared__ uint64_t part[kThreads / 64];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  unsigned long long v = x;
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    const unsigned long long y = __shfl_up(v, m);
    if (lane >= m) v += y;
  }
  __syncthreads();                       // part may still be read from a scan before
  if (lane == 63) part[wave] = v;
  __syncthreads();
  total = 0;
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) {
    if (i < wave) v += part[i];
    total += part[i];
  }
  return v;
}

// floor(all R / 2^24) with R = floor(u 2^24) in [0, 2^24 - 1]
__device__ inline uint64_t level_of(uint64_t all, float u) {
  const uint64_t R = u > 0.0f ? (u < 1.0f ? uint64_t(u * 16777216.0f) : 16777215u) : 0u;
  return (all >> 24) * R + (((all & 0xFFFFFFu) * R) >> 24);
}

// the token among c .. c + 7 whose weight the level falls in, `at` the sum before c; else -1
__device__ inline int token_of(const float (&w)[8], int c, uint64_t at, uint64_t level) {
  int token = -1;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint64_t x = value(whole(w[i]));
    if (at <= level && at + x > level) token = c + i;
    at += x;
  }
  return token;
}

__device__ inline void write_tokens(const VerifyArgs& a, int r, int kept, int token, int threads) {
  int32_t* out = a.out + int64_t(r) * (a.max_draft + 1);
  for (int i = threadIdx.x; i <= a.max_draft; i += threads)
    out[i] = i < kept ? a.tokens[int64_t(r) * a.max_draft + i] : i == kept ? token : -1;
  if (threadIdx.x == 0) a.emitted[r] = kept + 1;
}

// a request that is left out
__device__ inline void write_nothing(const VerifyArgs& a, int r, int threads) {
  write_tokens(a, r, 0, -1, threads);
  if (threadIdx.x == 0) a.emitted[r] = 0;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void verify_pick_kernel(VerifyArgs a) {
  __shared__ uint64_t level_s;
  __shared__ int tile_s, token_s;
  const int r = a.req0 + blockIdx.x, tid = threadIdx.x;
  const int n = drafts_of(a, r);
  if (n < 0) return write_nothing(a, r, kThreads);
  const int kept = a.kept[r];
  const uint64_t* sums = a.sums + int64_t(r) * a.tiles * 2;
  if (tid == 0) tile_s = token_s = -1;
  // the sum of w, or of p if that is 0; of up to 256 tiles the scan is kept
  bool residual = true;
  uint64_t all = 0, upto = 0, mine = 0;
  for (int which = 0; which < 2 && all == 0; ++which) {
    residual = which == 0;
    mine = 0;
    if (a.tiles <= kThreads) {
      if (tid < a.tiles) mine = sums[2 * tid + which];
    } else {
      for (int i = tid; i < a.tiles; i += kThreads) mine += sums[2 * i + which];
    }
    upto = block_scan(mine, all);
  }
  const uint64_t level = level_of(all, a.u_sample[r]);
  uint64_t before = 0;
  for (int t0 = 0; t0 < a.tiles; t0 += kThreads) {      // the tile, 256 at a time
    uint64_t total = all;
    if (a.tiles > kThreads) {
      mine = t0 + tid < a.tiles ? sums[2 * (t0 + tid) + (residual ? 0 : 1)] : 0;
      upto = before + block_scan(mine, total);
    }
    if (upto > level && upto - mine <= level) {         // one thread at most
      tile_s = t0 + tid;
      level_s = level - (upto - mine);
    }
    before += total;
    if (before > level) break;
  }
  __syncthreads();
  if (tile_s >= 0) {
    float p[8], w[8];
    const int c = tile_s * kTile + tid * 8;
    weights<T>(a, r, n, kept, c, residual, p, w);
    uint64_t sum = 0, total;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += value(whole(w[i]));
    const uint64_t at = block_scan(sum, total) - sum;
    if (at <= level_s && at + sum > level_s) token_s = token_of(w, c, at, level_s);
  }
  __syncthreads();
  write_tokens(a, r, kept, token_s, kThreads);
}

constexpr int kReqPerLaunch = 32768;   // a grid's second dimension

template <typename T>
void launch_verify(VerifyArgs a, int n_req, hipStream_t st) {
  for (int r0 = 0; r0 < n_req; r0 += kReqPerLaunch) {
    const int n = n_req - r0 < kReqPerLaunch ? n_req - r0 : kReqPerLaunch;
    a.req0 = r0;
    verify_sums_kernel<T><<<dim3((a.tiles + kTiles - 1) / kTiles, n), kThreads, 0, st>>>(a);
    verify_pick_kernel<T><<<n, kThreads, 0, st>>>(a);
  }
}

bool aligned_to(const void* p, int n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

int64_t tiles_of(int64_t vocab) { return (vocab + kTile - 1) / kTile; }

}  // namespace
}  // namespace dasc

extern "C" int dasc_verify_drafts_workspace_bytes(int32_t n_req, int64_t vocab, size_t* bytes) {
  if (!bytes || n_req < 0 || vocab < 1) return DASC_E_INVAL;
  if (vocab > dasc::kMaxVocab) return DASC_E_SHAPE;
  *bytes = size_t(n_req) * (dasc::tiles_of(vocab) * 2 * sizeof(uint64_t) + sizeof(int32_t));
  return DASC_OK;
}

extern "C" int dasc_verify_drafts(int32_t n_req, int32_t max_draft, int64_t vocab, int32_t dtype,
                                  const void* target, int64_t target_req, int64_t target_pos,
                                  const void* draft, int64_t draft_req, int64_t draft_pos,
                                  const int32_t* draft_tokens, const int32_t* n_draft,
                                  const float* u_accept, const float* u_sample,
                                  int32_t* out_tokens, int32_t* n_emitted, void* workspace,
                                  size_t workspace_bytes, dasc_stream_t stream) {
  using dasc::aligned_to;
  if (n_req < 0 || max_draft < 0) return DASC_E_INVAL;
  if (dtype != DASC_DTYPE_BF16 && dtype != DASC_DTYPE_F16 && dtype != DASC_DTYPE_F32) return DASC_E_INVAL;
  if (vocab < 1 || vocab > dasc::kMaxVocab || max_draft > dasc::kMaxDraft) return DASC_E_SHAPE;
  if (n_req == 0) return DASC_OK;
  if (!target || !u_sample || !out_tokens || !n_emitted) return DASC_E_INVAL;
  if (max_draft > 0 && (!draft_tokens || !u_accept)) return DASC_E_INVAL;
  const int e = dtype == DASC_DTYPE_F32 ? 4 : 2;
  if (!aligned_to(target, e) || !aligned_to(draft, e)) return DASC_E_INVAL;
  for (const void* p : {static_cast<const void*>(draft_tokens), static_cast<const void*>(n_draft),
                        static_cast<const void*>(u_accept), static_cast<const void*>(u_sample),
                        static_cast<const void*>(out_tokens), static_cast<const void*>(n_emitted)})
    if (!aligned_to(p, 4)) return DASC_E_INVAL;
  if (target_req < 0 || target_pos < 0 || (draft && (draft_req < 0 || draft_pos < 0))) return DASC_E_INVAL;
  size_t need = 0;
  const int rc = dasc_verify_drafts_workspace_bytes(n_req, vocab, &need);
  if (rc != DASC_OK) return rc;
  if (workspace_bytes < need || (need > 0 && !workspace)) return DASC_E_WORKSPACE;
  if (need > 0 && !aligned_to(workspace, 16)) return DASC_E_INVAL;
  dasc::VerifyArgs a;
  a.target = target;
  a.draft = max_draft > 0 ? draft : nullptr;
  a.target_req = target_req;
  a.target_pos = target_pos;
  a.draft_req = draft_req;
  a.draft_pos = draft_pos;
  a.tokens = draft_tokens;
  a.n_draft = n_draft;
  a.u_accept = u_accept;
  a.u_sample = u_sample;
  a.out = out_tokens;
  a.emitted = n_emitted;
  a.sums = static_cast<uint64_t*>(workspace);
  a.kept = reinterpret_cast<int32_t*>(a.sums + int64_t(n_req) * 2 * dasc::tiles_of(vocab));
  a.max_draft = max_draft;
  a.vocab = int32_t(vocab);
  a.tiles = int32_t(dasc::tiles_of(vocab));
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  switch (dtype) {
    case DASC_DTYPE_BF16: dasc::launch_verify<dasc::bf16_t>(a, n_req, st); break;
    case DASC_DTYPE_F16: dasc::launch_verify<dasc::f16_t>(a, n_req, st); break;
    default: dasc::launch_verify<float>(a, n_req, st); break;
  }
  return dasc::launch_status();
}

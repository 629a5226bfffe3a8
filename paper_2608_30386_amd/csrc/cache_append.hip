// Append to a paged cache: new queries and keys turned by their positions, keys and values written to
// their slots.
//
// A pair (x, y) of a head turns by angle = pos * inv_freq: (x cos - y sin, x sin + y cos).  The angle of a far
// position needs more than 24 bits, so its quarter turns are counted in 64-bit arithmetic, and the rest, at
// most an eighth of a turn, goes through the series of sine and cosine in fp32.
//
// A block takes a token: its threads first form the cosines and sines of the token's pairs, once for all heads,
// in LDS, then move the heads in units of eight elements (two of them for pairs that lie apart).
//
// HBM bounds it: 8192 tokens of 32 + 8 + 8 heads of 128, 201 MB in 39.5 us (5.1 TB/s), where every call has other inputs;
// 30.6 us on one set, part of which stays in the last-level cache.  One block for a token and 1024 units.
// A few tokens take 4.3 us, three dependent loads and a launch.

#include <hip/hip_runtime.h>

#include <cstdint>

#include "cache_common.h"
#include "launch_common.h"
#include "output_rows.h"
#include "row_io.h"

namespace dasc {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxHalf = 128;            // pairs of a head

struct AppendArgs {
  dasc_kv_cache c;
  dasc_append_io io;
  int64_t tok0;                          // first token of a launch
  int32_t parts;                         // blocks that share a token's heads
};

// cos and sin of the angle pos * freq.  Its quarter turns are pos (hi + lo) with hi + lo = freq 2 / pi to 100 bits, so
// that what is left of them is good to 2^-50 for any position.
__device__ inline void turn(double pos, double freq, float& c, float& s) {
  const double hi = freq * 0.6366197723675814;
  const double lo = fma(freq, 0.6366197723675814, -hi) + freq * -3.935735335036497e-17;
  const double n = rint(pos * hi);
  const float z = float(fma(pos, hi, -n) + pos * lo) * 1.57079632679f;     // at most pi / 4
  const float w = z * z;
  // Taylor series about 0: the first terms left out are below 2e-9
  float sn = fmaf(w, 2.7557319e-6f, -1.9841270e-4f);
  sn = fmaf(w, sn, 8.3333333e-3f);
  sn = fmaf(w, sn, -1.6666667e-1f);
  sn = fmaf(z * w, sn, z);
  float cs = fmaf(w, -2.7557319e-7f, 2.4801587e-5f);
  cs = fmaf(w, cs, -1.3888889e-3f);
  cs = fmaf(w, cs, 4.1666667e-2f);
  cs = fmaf(w, cs, -0.5f);
  cs = fmaf(w, cs, 1.0f);
  const double q = n - 4.0 * floor(0.25 * n);                // the quadrant
  const bool odd = q == 1.0 || q == 3.0;
  c = odd ? sn : cs;
  s = odd ? cs : sn;
  if (q == 1.0 || q == 2.0) c = -c;
  if (q >= 2.0) s = -s;
}

template <typename T, int VEC, bool ADJ>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a) {
  __shared__ float cosine[kMaxHalf], sine[kMaxHalf];
  __shared__ int64_t place[2];                               // page and place in it; page -1: none
  const dasc_append_io& io = a.io;
  const int tid = threadIdx.x, half = io.rot / 2, d = a.c.head_dim;
  const int64_t tok = a.tok0 + blockIdx.x;
  if (tid == 0) {
    const int64_t slot = io.slots[tok];
    const bool in = slot >= 0 && slot / a.c.page_size < a.c.n_pages;
    place[0] = in ? slot / a.c.page_size : -1;
    place[1] = in ? slot % a.c.page_size : 0;
  }
  for (int p = tid; p < half; p += kThreads) {
    const int axis = io.pair_axis ? io.pair_axis[p] : 0;
    float c = 1.0f, s = 0.0f;
    if (axis >= 0 && axis < io.n_axes)
      turn(double(io.pos[tok * io.pos_tok + axis * io.pos_axis]), double(io.inv_freq[p]), c, s);
    cosine[p] = c;
    sine[p] = s;
  }
  __syncthreads();
  // units of a head of q or k: those of pairs, then those of elements that stay; of v: elements
  const int turned = ADJ ? io.rot / (2 * VEC) : half / VEC;
  const int units = turned + (d - io.rot) / VEC, plain = d / VEC;
  const int hq = io.q ? io.n_q_heads : 0, hk = a.c.n_kv_heads;
  const int per = (hq + hk) * units + hk * plain;
  const int64_t page = place[0], off = place[1];
  for (int i = blockIdx.y * kThreads + tid; i < per; i += a.parts * kThreads) {
    int u = i;
    const T* src;
    T* dst;
    bool v = false;
    if (u < hq * units) {
      const int h = u / units;
      u -= h * units;
      src = static_cast<const T*>(io.q) + tok * io.q_tok + h * io.q_head;
      dst = static_cast<T*>(io.q_out) + tok * io.qo_tok + h * io.qo_head;
    } else {
      if (page < 0) continue;
      u -= hq * units;
      v = u >= hk * units;
      if (v) u -= hk * units;
      const int per_head = v ? plain : units, h = u / per_head;
      u -= h * per_head;
      src = v ? static_cast<const T*>(io.v) + tok * io.v_tok + h * io.v_head
              : static_cast<const T*>(io.k) + tok * io.k_tok + h * io.k_head;
      dst = v ? static_cast<T*>(a.c.v) + page * a.c.v_page + off * a.c.v_tok + h * a.c.v_head
              : static_cast<T*>(a.c.k) + page * a.c.k_page + off * a.c.k_tok + h * a.c.k_head;
    }
    typedef Vec<T, VEC> V;
    if (v || u >= turned) {
      const int at = v ? u * VEC : io.rot + (u - turned) * VEC;
      *reinterpret_cast<V*>(dst + at) = *reinterpret_cast<const V*>(src + at);
      continue;
    }
    const int p = u * VEC;                                   // the first pair
    const int x0 = ADJ ? 2 * p : p, y0 = ADJ ? 2 * p + VEC : p + half;
    V x = *reinterpret_cast<const V*>(src + x0), y = *reinterpret_cast<const V*>(src + y0);
    float f[2 * VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) f[e] = widen(x.e[e]);
#pragma unroll
    for (int e = 0; e < VEC; ++e) f[VEC + e] = widen(y.e[e]);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const int lo = ADJ ? 2 * e : e, hi = ADJ ? 2 * e + 1 : e + VEC;
      const float c = cosine[p + e], s = sine[p + e], g = f[lo], h = f[hi];
      f[lo] = fmaf(g, c, -(h * s));
      f[hi] = fmaf(g, s, h * c);
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) narrow(f[e], x.e[e]);
#pragma unroll
    for (int e = 0; e < VEC; ++e) narrow(f[VEC + e], y.e[e]);
    *reinterpret_cast<V*>(dst + x0) = x;
    *reinterpret_cast<V*>(dst + y0) = y;
  }
}

template <typename T, int VEC, bool ADJ>
void launch(AppendArgs a, hipStream_t st) {
  constexpr int64_t kBlocks = int64_t(1) << 20;
  const int heads = (a.io.q ? a.io.n_q_heads : 0) + 2 * a.c.n_kv_heads;
  const int work = heads * a.c.head_dim / VEC;
  a.parts = (work + 4 * kThreads - 1) / (4 * kThreads);
  if (a.parts > 32) a.parts = 32;
  for (; a.tok0 < a.io.n_tokens; a.tok0 += kBlocks) {
    const int64_t left = a.io.n_tokens - a.tok0;
    append_kernel<T, VEC, ADJ><<<dim3(uint32_t(left < kBlocks ? left : kBlocks), a.parts), kThreads, 0, st>>>(a);
  }
}

template <typename T>
void launch_type(const AppendArgs& a, hipStream_t st) {
  const bool adj = a.io.adjacent != 0;
  const int rot = a.io.rot;
  if (rot % 16 == 0) adj ? launch<T, 8, true>(a, st) : launch<T, 8, false>(a, st);
  else adj ? launch<T, 1, true>(a, st) : launch<T, 1, false>(a, st);
}

}  // namespace
}  // namespace dasc

extern "C" int dasc_cache_append(const dasc_kv_cache* cache, const dasc_append_io* append, dasc_stream_t stream) {
  using namespace dasc;
  if (!cache || !append) return DASC_E_INVAL;
  AppendArgs a = {};
  a.c = *cache;
  a.io = *append;
  drop_unused(a.c);
  drop_unused(a.io.n_tokens, {&a.io.q_tok, &a.io.qo_tok, &a.io.k_tok, &a.io.v_tok, &a.io.pos_tok});
  drop_unused(a.io.n_q_heads, {&a.io.q_head, &a.io.qo_head});
  drop_unused(a.c.n_kv_heads, {&a.io.k_head, &a.io.v_head});
  drop_unused(a.io.n_axes, {&a.io.pos_axis});
  const dasc_kv_cache& c = a.c;
  const dasc_append_io* const io = &a.io;
  const int rc = check_cache(&c, 2);
  if (rc != DASC_OK) return rc;
  if (io->rot < 0 || io->rot % 2 || io->rot > c.head_dim || io->n_axes < 1 || io->n_axes > 8 || io->n_tokens < 0 ||
      io->n_tokens > INT32_MAX || (io->q && (io->n_q_heads < 1 || io->n_q_heads > 65536)))
    return DASC_E_SHAPE;
  if (io->adjacent != 0 && io->adjacent != 1) return DASC_E_INVAL;
  if (!rows_apart3(c.n_pages, c.k_page, c.page_size, c.k_tok, c.n_kv_heads, c.k_head, c.head_dim) ||
      !rows_apart3(c.n_pages, c.v_page, c.page_size, c.v_tok, c.n_kv_heads, c.v_head, c.head_dim))
    return DASC_E_INVAL;
  if (io->n_tokens == 0) return DASC_OK;
  if (!io->k || !io->v || !io->slots || (io->q != nullptr) != (io->q_out != nullptr)) return DASC_E_INVAL;
  if (io->rot > 0 && (!io->pos || !io->inv_freq)) return DASC_E_INVAL;
  if (!aligned_to(io->q, 2) || !aligned_to(io->q_out, 2) || !aligned_to(io->k, 2) || !aligned_to(io->v, 2) ||
      !aligned_to(io->slots, 8) || !aligned_to(io->pos, 4) || !aligned_to(io->inv_freq, 4) ||
      !aligned_to(io->pair_axis, 4))
    return DASC_E_INVAL;
  if (io->k_tok < 0 || io->k_head < 0 || io->v_tok < 0 || io->v_head < 0 || io->pos_tok < 0 || io->pos_axis < 0)
    return DASC_E_INVAL;
  if (io->q && (io->q_tok < 0 || io->q_head < 0 ||
                !rows_apart(io->n_tokens, io->qo_tok, io->n_q_heads, io->qo_head, c.head_dim)))
    return DASC_E_INVAL;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (c.dtype == DASC_DTYPE_BF16) launch_type<bf16_t>(a, st);
  else launch_type<f16_t>(a, st);
  return launch_status();
}

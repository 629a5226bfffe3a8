// The norms before and after a block, with its gate and residual scale, in one pass over the row:
//
//     b  = act(gate) y rsqrt(mean(y^2) + eps) w_post
//     x' = x + scale channel_scale b
//     h  = x' rsqrt(mean(x'^2) + eps) w_pre
//
// A row stays in registers from its first load to its last store, on 16 or 64 lanes or a block of up to
// 16 waves, so every input is read once.  The sums are fp32.
//
// HBM bounds it: 8192 x 32 gated rows of 128 in bf16, 201 MB in 50 us (4.0 TB/s); 6001 rows of 2050, a gated
// bf16 block around an fp32 residual, 172 MB in 51 us (3.4 TB/s); a large copy runs at 4.9.  A block that
// takes several rows and keeps the weights in registers, which fewer waves then fit into: rows of 128 50 ->
// 47 us, but 2050 51 -> 64 and 5000 108 -> 121.

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "dasc/ops.h"
#include "launch_common.h"
#include "output_rows.h"
#include "row_io.h"

namespace dasc {
namespace {

constexpr int kMaxDim = 32768;

// Sum over the lanes of a row, 16 or 64 of them or (L = 0) a block's; every lane gets it.  The waves of
// a block meet in LDS.
template <int L>
__device__ inline float row_sum(float x, float* part) {
#pragma unroll
  for (int m = 1; m < (L == 16 ? 16 : 64); m *= 2) x += __shfl_xor(x, m);
  if constexpr (L == 0) {
    const int waves = blockDim.x / 64;
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = x;
    __syncthreads();
    x = 0;
    for (int i = 0; i < waves; ++i) x += part[i];
  }
  return x;
}

// 1 / (1 + e^-z) within 2 ulp: the exponent's rounding error, z large, goes back in as a factor.  (The
// library's exponential and division take some 30 instructions, which bound rows of 128: 57 us for
// 8192 x 32 of them with a gate.)
__device__ inline float sigmoid(float z) {
  const float t = -1.44269504f * z;
  float r = fmaf(-1.44269504f, z, -t);
  r = fmaf(-1.92596299e-8f, z, r);                    // log2 e is 1.44269504 + 1.92596299e-8
  r = fabsf(t) < 126.0f ? r : 0.0f;                  // (past it e is 0 or infinite)
  const float e = __builtin_amdgcn_exp2f(t);
  return __builtin_amdgcn_rcpf(fmaf(e, fmaf(0.693147182f, r, 1.0f), 1.0f));
}

// A row on 16 or 64 lanes, or (L = 0) on a block; a lane makes A accesses of VEC elements to each tensor.
// Everything a row needs is asked for before its first sum.  Rows (i, j) of [outer, inner]; `inner` is
// divided by as 32-bit numbers.  What lies past the row's end is zero throughout.
template <typename T, typename X, int L, int A, int VEC>
__global__ __launch_bounds__(L ? 256 : 1024) void block_norm_kernel(dasc_norm_io a, uint32_t row0, uint32_t rows) {
  __shared__ float part[2][16];
  const int lanes = L ? L : blockDim.x;
  const int lane = L ? threadIdx.x % lanes : threadIdx.x;
  const uint32_t row = row0 + (L ? blockIdx.x * (256 / lanes) + threadIdx.x / lanes : blockIdx.x);
  if (row >= rows) return;                            // whole rows: no barrier is left waiting
  const int64_t i = a.inner == 1 ? row : row / uint32_t(a.inner), j = a.inner == 1 ? 0 : row % uint32_t(a.inner);
  const int n = a.dim;
  const bool wide = a.w_dtype == DASC_DTYPE_F32;
  const float inv = 1.0f / float(n);

  const auto at = [&](int v) { return (v * lanes + lane) * VEC; };   // the column of access v
  const auto times = [&](const void* w, int v, float (&t)[VEC]) {    // t *= w
    float f[VEC];
    if (wide) load_vec<VEC>(static_cast<const float*>(w), at(v), n, f);
    else load_vec<VEC>(static_cast<const T*>(w), at(v), n, f);
#pragma unroll
    for (int e = 0; e < VEC; ++e) t[e] *= f[e];
  };

  float x[A][VEC], gate[A][VEC], res[A][VEC];
  const T* y = static_cast<const T*>(a.y) + i * a.y_out + j * a.y_in;
#pragma unroll
  for (int v = 0; v < A; ++v) load_vec<VEC>(y, at(v), n, x[v]);
  if (a.gate) {
    const T* g = static_cast<const T*>(a.gate) + i * a.gate_out + j * a.gate_in;
#pragma unroll
    for (int v = 0; v < A; ++v) load_vec<VEC>(g, at(v), n, gate[v]);
  }
  if (a.x) {
    const X* r = static_cast<const X*>(a.x) + i * a.x_row_out + j * a.x_row_in;
#pragma unroll
    for (int v = 0; v < A; ++v) load_vec<VEC>(r, at(v), n, res[v]);
  }
  float s = a.scale;
  if (a.w_post) {
    float ss = 0;
#pragma unroll
    for (int v = 0; v < A; ++v)
#pragma unroll
      for (int e = 0; e < VEC; ++e) ss = fmaf(x[v][e], x[v][e], ss);
    s *= rsqrtf(row_sum<L>(ss, part[0]) * inv + a.eps);
  }
  float ss = 0;
#pragma unroll
  for (int v = 0; v < A; ++v) {
    if (at(v) >= n) continue;
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[v][e] *= s;
    if (a.w_post) times(a.w_post, v, x[v]);
    if (a.gate) {
      if (a.act == DASC_ACT_SILU) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[v][e] *= gate[v][e] * sigmoid(gate[v][e]);
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[v][e] *= sigmoid(gate[v][e]);
      }
    }
    if (a.channel_scale) times(a.channel_scale, v, x[v]);
    if (a.x) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[v][e] += res[v][e];
    }
    if (a.x_out) store_vec<VEC>(static_cast<X*>(a.x_out) + i * a.xo_out + j * a.xo_in, at(v), n, x[v]);
#pragma unroll
    for (int e = 0; e < VEC; ++e) ss = fmaf(x[v][e], x[v][e], ss);
  }
  if (!a.h_out) return;
  const float r = rsqrtf(row_sum<L>(ss, part[1]) * inv + a.eps);
#pragma unroll
  for (int v = 0; v < A; ++v) {
    if (at(v) >= n) continue;
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[v][e] *= r;
    times(a.w_pre, v, x[v]);
    store_vec<VEC>(static_cast<T*>(a.h_out) + i * a.h_row_out + j * a.h_row_in, at(v), n, x[v]);
  }
}

constexpr int64_t kBlocksPerLaunch = int64_t(1) << 21;   // a grid counts threads in 32 bits

template <typename T, typename X, int L, int A, int VEC>
void launch(const dasc_norm_io& a, int threads, hipStream_t st) {
  constexpr int kRows = L ? 256 / L : 1;
  const int64_t rows = a.outer * a.inner;
  for (int64_t r0 = 0; r0 < rows; r0 += kBlocksPerLaunch * kRows) {
    const int64_t left = rows - r0;
    const int64_t n = left < kBlocksPerLaunch * kRows ? left : kBlocksPerLaunch * kRows;
    block_norm_kernel<T, X, L, A, VEC><<<uint32_t((n + kRows - 1) / kRows), threads, 0, st>>>(
        a, uint32_t(r0), uint32_t(r0 + n));
  }
}

// Whether every row of every tensor starts at a multiple of eight elements
bool by_eight(const dasc_norm_io& a, int e, int r, int w) {
  uint64_t bits = 0;
  const auto add = [&](const void* p, int size, int64_t so, int64_t si) {
    if (!p) return;
    bits |= reinterpret_cast<uintptr_t>(p) / size;
    if (a.outer > 1) bits |= uint64_t(so);
    if (a.inner > 1) bits |= uint64_t(si);
  };
  add(a.y, e, a.y_out, a.y_in);
  add(a.gate, e, a.gate_out, a.gate_in);
  add(a.x, r, a.x_row_out, a.x_row_in);
  add(a.x_out, r, a.xo_out, a.xo_in);
  add(a.h_out, e, a.h_row_out, a.h_row_in);
  add(a.w_post, w, 0, 0);
  add(a.w_pre, w, 0, 0);
  add(a.channel_scale, w, 0, 0);
  return bits % 8 == 0;
}

// The shape of a row, us for 6000 rows of a gated bf16 block and an fp32 residual:
// - accesses of eight elements where all rows are aligned to that (4096: 77, by four 83), of four where
//   not (1500: 36.5, by eight 45; 2052: 50.6 and 62; 1999: 52 and 62);
// - a wave for every 512, or begun 512.  Where a little is left over two, four or sixteen of them, a third
//   access instead of a wave that would have a SIMD to itself (or pass what a block may have): 1100 28.8 |
//   29.7, 2050 50.7 | 55.3, 2178 57.1 | 63.2, 8194 184 | 232.  Not elsewhere: 1540 43.5 | 39.3, 2562
//   75.4 | 67.6, 3330 91.6 | 79.7, 3970 114 | 95, 8002 228 | 187, and at eight or nine it is the same (4226 115 | 113);
// - rows of up to 128 on 16 lanes, eight elements each.
template <typename T, typename X>
void launch_dim(const dasc_norm_io& a, bool eight, hipStream_t st) {
  const int n = a.dim, whole = n / 512, over = n % 512;
  const auto threads = [n](int per) { return (n + 64 * per - 1) / (64 * per) * 64; };
  if (n <= 128) launch<T, X, 16, 1, 8>(a, 256, st);
  else if (n <= 512) launch<T, X, 64, 2, 4>(a, 256, st);
  else if (n <= 1024) launch<T, X, 64, 4, 4>(a, 256, st);
  else if (eight && n <= 8192) launch<T, X, 0, 1, 8>(a, threads(8), st);
  else if (over > 0 && over <= 64 * whole && (whole == 2 || whole == 4 || whole == 16))
    launch<T, X, 0, 3, 4>(a, 64 * whole, st);
  else if (n <= 8192) launch<T, X, 0, 2, 4>(a, threads(8), st);
  else if (n <= 16384) launch<T, X, 0, 4, 4>(a, threads(16), st);
  else launch<T, X, 0, 8, 4>(a, threads(32), st);
}

template <typename T>
void launch_res(const dasc_norm_io& a, bool eight, hipStream_t st) {
  if (a.res_dtype == a.dtype) launch_dim<T, T>(a, eight, st);
  else launch_dim<T, float>(a, eight, st);
}

bool aligned_to(const void* p, int n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
int size_of(int dtype) { return dtype == DASC_DTYPE_F32 ? 4 : 2; }
bool known(int dtype) { return dtype == DASC_DTYPE_BF16 || dtype == DASC_DTYPE_F16 || dtype == DASC_DTYPE_F32; }

}  // namespace
}  // namespace dasc

extern "C" int dasc_block_norm(const dasc_norm_io* io, dasc_stream_t stream) {
  using namespace dasc;
  if (!io) return DASC_E_INVAL;
  const dasc_norm_io& a = *io;
  if (a.outer < 0 || a.inner < 1 || a.dim < 1 || a.outer > INT32_MAX || a.outer * a.inner > INT32_MAX)
    return DASC_E_SHAPE;
  if (!known(a.dtype) || (a.res_dtype != a.dtype && a.res_dtype != DASC_DTYPE_F32) ||
      (a.w_dtype != a.dtype && a.w_dtype != DASC_DTYPE_F32))
    return DASC_E_INVAL;
  if (a.act != DASC_ACT_NONE && a.act != DASC_ACT_SIGMOID && a.act != DASC_ACT_SILU) return DASC_E_INVAL;
  if (!std::isfinite(a.eps) || a.eps < 0 || !std::isfinite(a.scale)) return DASC_E_INVAL;
  if (a.dim > kMaxDim) return DASC_E_UNSUPPORTED;
  if (a.outer == 0) return DASC_OK;
  if (!a.y || (!a.x_out && !a.h_out) || (a.h_out && !a.w_pre)) return DASC_E_INVAL;
  if ((a.gate != nullptr) != (a.act != DASC_ACT_NONE)) return DASC_E_INVAL;
  const int e = size_of(a.dtype), r = size_of(a.res_dtype), w = size_of(a.w_dtype);
  if (!aligned_to(a.y, e) || !aligned_to(a.gate, e) || !aligned_to(a.h_out, e) || !aligned_to(a.x, r) ||
      !aligned_to(a.x_out, r) || !aligned_to(a.w_post, w) || !aligned_to(a.w_pre, w) ||
      !aligned_to(a.channel_scale, w))
    return DASC_E_INVAL;
  if (a.y_out < 0 || a.y_in < 0) return DASC_E_INVAL;
  if (a.gate && (a.gate_out < 0 || a.gate_in < 0)) return DASC_E_INVAL;
  if (a.x && (a.x_row_out < 0 || a.x_row_in < 0)) return DASC_E_INVAL;
  // rows of an output must not overlap
  const auto apart = [&](int64_t so, int64_t si) { return rows_apart(a.outer, so, a.inner, si, a.dim); };
  if (a.x_out && !apart(a.xo_out, a.xo_in)) return DASC_E_INVAL;
  if (a.h_out && !apart(a.h_row_out, a.h_row_in)) return DASC_E_INVAL;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const bool eight = by_eight(a, e, r, w);
  switch (a.dtype) {
    case DASC_DTYPE_BF16: launch_res<bf16_t>(a, eight, st); break;
    case DASC_DTYPE_F16: launch_res<f16_t>(a, eight, st); break;
    default: launch_dim<float, float>(a, eight, st); break;
  }
  return launch_status();
}

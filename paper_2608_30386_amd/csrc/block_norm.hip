// The norms before and after a block, with its gate and residual scale, in one pass over the row:
//
//     b  = act(gate) y rsqrt(mean(y^2) + eps) w_post
//     x' = x + scale channel_scale b
//     h  = x' rsqrt(mean(x'^2) + eps) w_pre
//
// A row stays in registers from its first load to its last store, on 16, 64, 256 or 1024 lanes
// with up to four vectors of eight elements each, so every input is read once.  The sums are
// fp32.

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "dasc/ops.h"
#include "launch_common.h"
#include "row_io.h"

namespace dasc {
namespace {

constexpr int kMaxDim = 32768;

// Sum over the L lanes of a row; every lane gets it.  Rows of more than a wave meet in LDS.
template <int L>
__device__ inline float row_sum(float x, float* part) {
#pragma unroll
  for (int m = 1; m < (L < 64 ? L : 64); m *= 2) x += __shfl_xor(x, m);
  if constexpr (L > 64) {
    const int wave = threadIdx.x / 64;
    if (threadIdx.x % 64 == 0) part[wave] = x;
    __syncthreads();
    x = 0;
#pragma unroll
    for (int i = 0; i < L / 64; ++i) x += part[i];
  }
  return x;
}

template <typename T>
__device__ inline void weights8(const void* w, bool wide, int c, int n, float (&x)[8]) {
  if (wide) load8(static_cast<const float*>(w), c, n, x);
  else load8(static_cast<const T*>(w), c, n, x);
}

template <typename T, typename X, int L, int NV>
__global__ __launch_bounds__(L < 256 ? 256 : L) void block_norm_kernel(dasc_norm_io a, int64_t row0, int64_t rows) {
  constexpr int kRows = L < 256 ? 256 / L : 1;        // rows of a block
  __shared__ float part[2][L > 64 ? L / 64 : 1];
  const int lane = threadIdx.x % L;
  const int64_t row = row0 + int64_t(blockIdx.x) * kRows + threadIdx.x / L;
  if (row >= rows) return;                            // whole rows: no barrier is left waiting
  const int64_t i = row / a.inner, j = row % a.inner;
  const int n = a.dim;
  const bool wide = a.w_dtype == DASC_DTYPE_F32;
  const float inv = 1.0f / float(n);

  float x[NV][8];
  const T* y = static_cast<const T*>(a.y) + i * a.y_out + j * a.y_in;
#pragma unroll
  for (int v = 0; v < NV; ++v) load8(y, (v * L + lane) * 8, n, x[v]);
  float s = a.scale;
  if (a.w_post) {
    float ss = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(x[v][e], x[v][e], ss);
    ss = row_sum<L>(ss, part[0]);
    s *= 1.0f / sqrtf(ss * inv + a.eps);
  }
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * L + lane) * 8;
    if (c >= n) continue;
    float t[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[v][e] *= s;
    if (a.w_post) {
      weights8<T>(a.w_post, wide, c, n, t);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[v][e] *= t[e];
    }
    if (a.gate) {
      load8(static_cast<const T*>(a.gate) + i * a.gate_out + j * a.gate_in, c, n, t);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float sig = 1.0f / (1.0f + expf(-t[e]));
        x[v][e] *= a.act == DASC_ACT_SILU ? t[e] * sig : sig;
      }
    }
    if (a.channel_scale) {
      weights8<T>(a.channel_scale, wide, c, n, t);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[v][e] *= t[e];
    }
    if (a.x) {
      load8(static_cast<const X*>(a.x) + i * a.x_row_out + j * a.x_row_in, c, n, t);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[v][e] += t[e];
    }
    if (a.x_out) store8(static_cast<X*>(a.x_out) + i * a.xo_out + j * a.xo_in, c, n, x[v]);
  }
  if (!a.h_out) return;
  float ss = 0;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    if ((v * L + lane) * 8 >= n) continue;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if ((v * L + lane) * 8 + e < n) ss = fmaf(x[v][e], x[v][e], ss);
  }
  ss = row_sum<L>(ss, part[1]);
  const float r = 1.0f / sqrtf(ss * inv + a.eps);
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * L + lane) * 8;
    if (c >= n) continue;
    float t[8];
    weights8<T>(a.w_pre, wide, c, n, t);
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] *= x[v][e] * r;
    store8(static_cast<T*>(a.h_out) + i * a.h_row_out + j * a.h_row_in, c, n, t);
  }
}

constexpr int64_t kBlocksPerLaunch = int64_t(1) << 21;   // a grid counts threads in 32 bits

template <typename T, typename X, int L, int NV>
void launch(const dasc_norm_io& a, hipStream_t st) {
  constexpr int kRows = L < 256 ? 256 / L : 1;
  const int64_t rows = a.outer * a.inner;
  for (int64_t r0 = 0; r0 < rows; r0 += kBlocksPerLaunch * kRows) {
    const int64_t left = rows - r0;
    const int64_t n = left < kBlocksPerLaunch * kRows ? left : kBlocksPerLaunch * kRows;
    block_norm_kernel<T, X, L, NV><<<uint32_t((n + kRows - 1) / kRows), L < 256 ? 256 : L, 0, st>>>(a, r0, r0 + n);
  }
}

template <typename T, typename X>
void launch_dim(const dasc_norm_io& a, hipStream_t st) {
  const int n = a.dim;
  if (n <= 128) launch<T, X, 16, 1>(a, st);
  else if (n <= 512) launch<T, X, 64, 1>(a, st);
  else if (n <= 1024) launch<T, X, 64, 2>(a, st);
  else if (n <= 2048) launch<T, X, 256, 1>(a, st);
  else if (n <= 4096) launch<T, X, 256, 2>(a, st);
  else if (n <= 8192) launch<T, X, 256, 4>(a, st);
  else if (n <= 16384) launch<T, X, 1024, 2>(a, st);
  else launch<T, X, 1024, 4>(a, st);
}

template <typename T>
void launch_res(const dasc_norm_io& a, hipStream_t st) {
  if (a.res_dtype == a.dtype) launch_dim<T, T>(a, st);
  else launch_dim<T, float>(a, st);
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
  const auto apart = [&](int64_t so, int64_t si) {
    if (so < 0 || si < 0) return false;
    if (a.outer == 1) return a.inner == 1 || si >= a.dim;
    if (a.inner == 1) return so >= a.dim;
    const int64_t lo = so < si ? so : si, hi = so < si ? si : so;
    const int64_t n = so < si ? a.outer : a.inner;      // rows that lie `lo` apart
    return lo >= a.dim && hi / n >= lo;                 // hi >= n lo, without the product
  };
  if (a.x_out && !apart(a.xo_out, a.xo_in)) return DASC_E_INVAL;
  if (a.h_out && !apart(a.h_row_out, a.h_row_in)) return DASC_E_INVAL;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  switch (a.dtype) {
    case DASC_DTYPE_BF16: launch_res<bf16_t>(a, st); break;
    case DASC_DTYPE_F16: launch_res<f16_t>(a, st); break;
    default: launch_dim<float, float>(a, st); break;
  }
  return launch_status();
}

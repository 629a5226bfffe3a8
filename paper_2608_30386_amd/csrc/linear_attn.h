// What the two forms of linear attention share: the call's arguments as the kernels take
// them, and each form's launcher.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "dasc/ops.h"

namespace dasc {

struct LinearArgs {
  dasc_linear_io io;
  float* states;                       // layer 0 of slot 0
  int64_t slot_stride, layer_off;      // floats from slot to slot; this layer's first float
  int64_t n_pool;
  const int32_t *src, *dst, *cu, *lens;
  int64_t n_tokens;
  int32_t n_req, H, rep, dv;           // rep: value heads per key head
  float scale;
};

struct Span { int64_t begin; int32_t len; };

// Rows of request i: cu clamped to [0, n_tokens], lens to the request.
__device__ inline Span request_span(const LinearArgs& a, int i) {
  const int64_t n = a.n_tokens;
  int64_t b = a.cu[i], e = a.cu[i + 1];
  b = b < 0 ? 0 : b > n ? n : b;
  e = e < b ? b : e > n ? n : e;
  int64_t len = e - b;
  if (a.lens) {
    const int64_t l = a.lens[i];
    len = l < 0 ? 0 : l < len ? l : len;
  }
  return {b, int32_t(len)};
}

// The head's state in the slot that `slots` names for request i, or nullptr.
__device__ inline float* slot_state(const LinearArgs& a, const int32_t* slots, int i, int h, int dk) {
  if (!slots) return nullptr;
  const int64_t s = slots[i];
  if (s < 0 || s >= a.n_pool) return nullptr;
  return a.states + s * a.slot_stride + a.layer_off + int64_t(h) * dk * a.dv;
}

__device__ inline float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// What the host knows of a call, for the choice of its form and the size of its workspace
struct ChunkPlan {
  int32_t dk, dv, H, n_req, max_len;
  int64_t n_tokens;
  bool delta;
};

bool linear_chunk_supported(const ChunkPlan& c);
int64_t linear_chunk_workspace(ChunkPlan c);
void launch_linear_chunks(const ChunkPlan& c, const LinearArgs& a, void* ws, hipStream_t st);
void launch_linear_steps(const LinearArgs& a, int dk, hipStream_t st);

}  // namespace dasc

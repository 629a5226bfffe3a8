// Linear attention with a decay for each head: the entry point and the token-by-token form.
//
//     S~ = e^{g} S;   u = v (plain) or beta (v - S~^T k) (delta);   S' = S~ + k u^T;   o = scale S'^T q
//
// The columns of a head's state evolve on their own, so a wave takes all dk rows of 32 columns
// and needs nothing from another wave: lane (rg, cg) holds rows rg dk/8 .. of the four columns
// 4 cg.. .  The two sums over the rows that a token needs, S~^T k and S~^T q, are formed before
// the update and summed over the row groups together; o = S~^T q + (q . k) u.  Everything is
// fp32.
//
// A call reads and writes each state once, whatever its tokens, and that bounds it: 128 requests x 32 heads
// of 128 x 128, a token each, take 101 us, 5.3 TB/s (a large copy runs at 4.9).  Each token more costs 4 us
// of 64 requests and 1 us of one, the chain of its two sums.

#include "linear_attn.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "launch_common.h"
#include "linear_steps.h"
#include "output_rows.h"

namespace dasc {
namespace {

constexpr int kCols = 32;             // columns of a wave

template <int DK, bool DELTA, bool OUT>
__global__ __launch_bounds__(256) void linear_steps_kernel(LinearArgs a, int64_t wave0, int64_t waves,
                                                           int col_blocks) {
  const int64_t w = wave0 + int64_t(blockIdx.x) * 4 + threadIdx.x / 64;
  if (w >= waves) return;
  const int64_t rh = w / col_blocks;
  walk_tokens<DK, kCols, DELTA, OUT>(a, int(rh / a.H), int(rh % a.H), int(w % col_blocks) * kCols, threadIdx.x % 64);
}

// waves of one launch: a grid counts threads in 32 bits
constexpr int64_t kWavesPerLaunch = int64_t(1) << 24;

template <int DK>
void launch_steps(const LinearArgs& a, hipStream_t st) {
  const int cb = (a.dv + kCols - 1) / kCols;
  const int64_t waves = int64_t(a.n_req) * a.H * cb;
  for (int64_t w0 = 0; w0 < waves; w0 += kWavesPerLaunch) {
    const int64_t n = waves - w0 < kWavesPerLaunch ? waves - w0 : kWavesPerLaunch;
    const dim3 grid(uint32_t((n + 3) / 4));
    const bool delta = a.io.beta, out = a.io.o;
    auto* f = delta ? (out ? linear_steps_kernel<DK, true, true> : linear_steps_kernel<DK, true, false>)
                    : (out ? linear_steps_kernel<DK, false, true> : linear_steps_kernel<DK, false, false>);
    f<<<grid, 256, 0, st>>>(a, w0, w0 + n, cb);
  }
}

// Calls whose longest request has more tokens than this take the chunked form.  A token costs the other form
// the chain of its sums where there are few heads, and a pass over the state's registers where there are
// many; a chunk of the delta rule costs two launches more than one of the plain rule.  Token by token | in
// chunks, us, 32 heads, with an output:
//     tokens                                4          8          12         16         20         24
//     dk = dv = 128
//     1 request, delta rule              9 |  15   13 |  15   18 |  15   22 |  15   27 |  15   31 |  15
//     8 requests                        13 |  25   17 |  25   22 |  25   26 |  25   31 |  25   36 |  26
//     64 requests                       57 | 117   72 | 120   91 | 122  110 | 123  128 | 130  148 | 132
//     1 request, plain rule              8 |   7   12 |   7   15 |   7   19 |   7   22 |   7   26 |   7
//     8 requests                        12 |  13   15 |  13   19 |  13   23 |  13   27 |  13   31 |  13
//     64 requests                       55 |  82   66 |  84   81 |  85   96 |  86  109 |  87  123 |  89
//     dk = dv = 64
//     1 request, delta rule              8 |  14   11 |  14   15 |  14   18 |  14   22 |  14   25 |  14
//     64 requests                       18 |  53   24 |  53   31 |  54   36 |  54   43 |  58   50 |  58
//     1 request, plain rule              7 |   6    9 |   6   12 |   6   15 |   6   17 |   6   20 |   6
//     64 requests                       16 |  25   21 |  25   25 |  25   29 |  26   34 |  26   38 |  26
// (states only: the same places but for one request, delta rule: 14.)
int step_tokens(const ChunkPlan& c) {
  const bool few = int64_t(c.n_req) * c.H <= 256;
  if (!c.delta) return few ? 4 : 11;
  return few ? 11 : c.dk == 64 ? 26 : 19;
}
constexpr int kLeastSteps[2] = {4, 11};       // of any call: plain, delta

bool takes_chunks(const ChunkPlan& c) { return c.max_len > step_tokens(c) && linear_chunk_supported(c); }

bool bad_stride(int64_t s, int64_t multiple) { return s < 0 || s % multiple != 0; }

}  // namespace

void launch_linear_steps(const LinearArgs& a, int dk, hipStream_t st) {
  switch (dk) {
    case 16: launch_steps<16>(a, st); break;
    case 32: launch_steps<32>(a, st); break;
    case 64: launch_steps<64>(a, st); break;
    default: launch_steps<128>(a, st); break;
  }
}

}  // namespace dasc

extern "C" int dasc_linear_attn_workspace_bytes(const dasc_shape* shape, int32_t n_req,
                                                int64_t n_tokens, int32_t max_len, int32_t delta,
                                                size_t* bytes) {
  if (!shape || !bytes || n_req < 1 || n_tokens < 0 || max_len < 0) return DASC_E_INVAL;
  if (!dasc::valid_shape(shape)) return DASC_E_SHAPE;
  const dasc::ChunkPlan c{shape->dk, shape->dv, shape->n_heads, n_req, max_len, n_tokens, delta != 0};
  *bytes = max_len > dasc::kLeastSteps[delta != 0] ? size_t(dasc::linear_chunk_workspace(c)) : 0;
  return DASC_OK;
}

extern "C" int dasc_linear_attn(const dasc_shape* shape, int32_t layer, float* states,
                                int64_t n_pool, const int32_t* src_slot, const int32_t* dst_slot,
                                const dasc_linear_io* io, const int32_t* cu_seqlens,
                                const int32_t* lens, int32_t n_req, int64_t n_tokens,
                                int32_t max_len, float scale, void* workspace,
                                size_t workspace_bytes, dasc_stream_t stream) {
  if (!shape || !io) return DASC_E_INVAL;
  if (!dasc::valid_shape(shape) || shape->dv % 4 != 0) return DASC_E_SHAPE;
  if (layer < 0 || layer >= shape->n_layers || n_req < 1 || n_tokens < 0 || n_tokens > INT32_MAX ||
      max_len < 0 || n_pool < 1 || !std::isfinite(scale))
    return DASC_E_INVAL;
  if (!states || !cu_seqlens) return DASC_E_INVAL;
  if (n_tokens > 0 && (!io->k || !io->v || !io->g)) return DASC_E_INVAL;
  if (n_tokens > 0 && !io->o && !dst_slot) return DASC_E_INVAL;
  if (io->o && !io->q) return DASC_E_INVAL;
  using dasc::aligned16;
  if (!aligned16(states) || (io->o && !aligned16(io->q)) || !aligned16(io->k) || !aligned16(io->v) ||
      !aligned16(io->o) || (reinterpret_cast<uintptr_t>(io->g) & 3) ||
      (reinterpret_cast<uintptr_t>(io->beta) & 3))
    return DASC_E_INVAL;
  using dasc::bad_stride;
  if (bad_stride(io->k_tok, 8) || bad_stride(io->k_head, 8) || bad_stride(io->v_tok, 4) ||
      bad_stride(io->v_head, 4) || bad_stride(io->g_tok, 1) || bad_stride(io->g_head, 1))
    return DASC_E_INVAL;
  if (io->o && (bad_stride(io->q_tok, 8) || bad_stride(io->q_head, 8) || bad_stride(io->o_tok, 4) ||
                bad_stride(io->o_head, 4)))
    return DASC_E_INVAL;
  if (io->beta && (bad_stride(io->beta_tok, 1) || bad_stride(io->beta_head, 1))) return DASC_E_INVAL;
  const int dk = shape->dk, dv = shape->dv;
  if (shape->arch != DASC_ARCH_GDN || dv > 256 || (dk != 16 && dk != 32 && dk != 64 && dk != 128))
    return DASC_E_UNSUPPORTED;
  size_t need = 0;
  const int rc = dasc_linear_attn_workspace_bytes(shape, n_req, n_tokens, max_len, io->beta != nullptr, &need);
  if (rc != DASC_OK) return rc;
  if (workspace_bytes < need || (need > 0 && !workspace)) return DASC_E_WORKSPACE;
  if (need > 0 && !aligned16(workspace)) return DASC_E_INVAL;
  // rows of the output must not overlap
  if (io->o && !dasc::rows_apart(n_tokens, io->o_tok, shape->n_heads, io->o_head, dv)) return DASC_E_INVAL;
  if (n_tokens == 0 && !dst_slot) return DASC_OK;     // no output and no state to write

  dasc::LinearArgs a;
  a.io = *io;
  a.states = states;
  a.slot_stride = dasc::rows_per_state(shape) * dv;
  a.layer_off = int64_t(layer) * shape->n_heads * dk * dv;
  a.n_pool = n_pool;
  a.src = src_slot;
  a.dst = dst_slot;
  a.cu = cu_seqlens;
  a.lens = lens;
  a.n_tokens = n_tokens;
  a.n_req = n_req;
  a.H = shape->n_heads;
  a.rep = shape->n_heads / shape->n_qk_heads;
  a.dv = dv;
  a.scale = scale;
  (void)hipGetLastError();
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  // The chunked form loads 16 bytes of a row at a time and counts the bytes of 64 rows in 31 bits, and
  // its rows have to lie apart: what is past the last of them reads as zero there.  It multiplies factors
  // of up to 2^16 by the scale before anything else.
  const auto apart = [](int64_t tok, int width) { return tok >= width && tok < (int64_t(1) << 24); };
  const bool wide = std::fabs(scale) < 0x1p100f && io->v_tok % 8 == 0 && io->v_head % 8 == 0 &&
                    apart(io->k_tok, dk) && apart(io->v_tok, dv) &&
                    (!io->o || (apart(io->q_tok, dk) && apart(io->o_tok, dv)));
  const dasc::ChunkPlan plan{dk, dv, shape->n_heads, n_req, max_len, n_tokens, io->beta != nullptr};
  if (wide && dasc::takes_chunks(plan)) dasc::launch_linear_chunks(plan, a, workspace, st);
  else dasc::launch_linear_steps(a, dk, st);
  return dasc::launch_status();
}

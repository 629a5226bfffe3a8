// Linear attention with a decay for each head, token by token, over some columns of one request's head.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "linear_attn.h"
#include "wy_ops.h"

namespace dasc {

// R consecutive bf16 (R = 2, 4, 8 or 16), two to a word
template <int R>
__device__ inline void load_bf16(const uint16_t* p, uint32_t (&w)[R / 2]) {
  if constexpr (R == 2) {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else if constexpr (R == 4) {
    *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(p);
  } else {
#pragma unroll
    for (int i = 0; i < R / 8; ++i)
      reinterpret_cast<uint4*>(w)[i] = reinterpret_cast<const uint4*>(p)[i];
  }
}
template <int N>
__device__ inline void widen(const uint32_t (&w)[N], float (&x)[2 * N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    x[2 * i] = bf16_lo(w[i]);
    x[2 * i + 1] = bf16_hi(w[i]);
  }
}

__device__ inline uint32_t pack_bf16(float x0, float x1) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(dasc_wy::f32x2{x0, x1}, dasc_wy::bf16x2));
}

// sum over the row groups, lanes CG apart; every lane gets it
template <int CG>
__device__ inline float rows_sum(float x) {
#pragma unroll
  for (int m = CG; m < 64; m *= 2) x += __shfl_xor(x, m);
  return x;
}

// S e^g.  A decay near one is applied as S + S (e^g - 1): rounded to fp32 itself it would be off
// by up to 2^-25, the same way for the whole state, token after token.  A growth that fp32 may not hold goes
// in three steps, each of a whole number but the last: zero stays zero whatever it is, and a small state
// comes out right (beyond e^264 nothing else does).
template <int R>
__device__ inline void decay(dasc_wy::f32x4 (&S)[R], float g) {
  if (g > 64.0f) {
    const float top = fminf(g, 264.0f), third = rintf(top * (1.0f / 3.0f)), e = expf(third);
    const float rest = expf(top - 2.0f * third);
#pragma unroll
    for (int r = 0; r < R; ++r) S[r] = S[r] * e * e * rest;
  } else if (g > -0.5f) {
    const float m = expm1f(g);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int e = 0; e < 4; ++e) S[r][e] = fmaf(S[r][e], m, S[r][e]);
  } else {
    const float m = expf(g);
#pragma unroll
    for (int r = 0; r < R; ++r) S[r] *= m;
  }
}

// A wave walks the tokens of request i over columns col0 .. col0 + COLS - 1 of head h, from the source
// slot to the destination: lane (rg, cg) holds rows rg R .. of the columns col0 + 4 cg .. .  Columns from dv
// on are left out.
template <int DK, int COLS, bool DELTA, bool OUT>
__device__ __forceinline__ void walk_tokens(const LinearArgs& a, int i, int h, int col0, int lane) {
  using dasc_wy::f32x4;
  constexpr int CG = COLS / 4;          // column groups: lanes side by side on one row
  constexpr int R = DK * CG / 64;       // rows of a lane
  const int cg = lane % CG, rg = lane / CG;
  const int col = col0 + 4 * cg;
  const bool in = col < a.dv;
  const int hk = h / a.rep;

  const Span sp = request_span(a, i);
  const float* from = slot_state(a, a.src, i, h, DK);
  float* to = slot_state(a, a.dst, i, h, DK);
  const int64_t at = int64_t(rg) * R * a.dv + col;

  f32x4 S[R];
#pragma unroll
  for (int r = 0; r < R; ++r)
    S[r] = from && in ? *reinterpret_cast<const f32x4*>(from + at + int64_t(r) * a.dv) : f32x4{0, 0, 0, 0};

  struct Token {
    uint32_t k[R / 2], q[R / 2];
    uint2 v;
    float g, beta;
  };
  const auto load = [&](int t) {
    const int64_t row = sp.begin + t;
    Token x;
    x.g = a.io.g[row * a.io.g_tok + h * a.io.g_head];
    if (DELTA) x.beta = a.io.beta[row * a.io.beta_tok + h * a.io.beta_head];
    load_bf16<R>(a.io.k + row * a.io.k_tok + hk * a.io.k_head + rg * R, x.k);
    if (OUT) load_bf16<R>(a.io.q + row * a.io.q_tok + hk * a.io.q_head + rg * R, x.q);
    x.v = in ? *reinterpret_cast<const uint2*>(a.io.v + row * a.io.v_tok + h * a.io.v_head + col) : uint2{0, 0};
    return x;
  };
  Token next = {};
  if (sp.len > 0) next = load(0);
  for (int t = 0; t < sp.len; ++t) {        // a token is asked for while the one before it is worked on
    const Token x = next;
    if (t + 1 < sp.len) next = load(t + 1);
    const int64_t row = sp.begin + t;
    decay(S, x.g);
    float k[R], q[R];
    widen(x.k, k);
    if (OUT) widen(x.q, q);
    const f32x4 v = {bf16_lo(x.v.x), bf16_hi(x.v.x), bf16_lo(x.v.y), bf16_hi(x.v.y)};
    f32x4 sk = {0, 0, 0, 0}, sq = {0, 0, 0, 0};
    float qk = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (DELTA) sk += S[r] * k[r];
      if (OUT) {
        sq += S[r] * q[r];
        qk = fmaf(q[r], k[r], qk);
      }
    }
    f32x4 u = v;
    if (DELTA) {
#pragma unroll
      for (int e = 0; e < 4; ++e) u[e] = x.beta * (v[e] - rows_sum<CG>(sk[e]));
    }
#pragma unroll
    for (int r = 0; r < R; ++r) S[r] += u * k[r];
    if (OUT) {
      const float d = rows_sum<CG>(qk);
      f32x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = a.scale * (rows_sum<CG>(sq[e]) + d * u[e]);
      if (in && rg == 0)
        *reinterpret_cast<uint2*>(a.io.o + row * a.io.o_tok + h * a.io.o_head + col) =
            uint2{pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
    }
  }
  if (to && in && !(from == to && sp.len == 0)) {
#pragma unroll
    for (int r = 0; r < R; ++r) *reinterpret_cast<f32x4*>(to + at + int64_t(r) * a.dv) = S[r];
  }
}

}  // namespace dasc

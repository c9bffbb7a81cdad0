// ssm.h -- shared parts of the selective scan's kernels.
//
// The scan.  Per channel d and state n, with the step size dt_t (per channel) and B_t, C_t
// (per group of channels),
//   h_t = a_t h_{t-1} + dt_t x_t B_t,  a_t = e^(dt_t A),   y_t = sum_n C_t h_t.
// A lane holds one channel and all its states in registers, so that the sum over states
// needs no other lane and B and C, which a wave's 64 channels share, come through scalar
// registers.  Tokens are cut into chunks, one to a wave:
//   1. every chunk but the last goes from a zero state to what it leaves (and the sum of its
//      step sizes, which gives its decay e^(A sum dt) without a product per token);
//   2. what enters each chunk is folded from that, per channel and state;
//   3. every chunk goes over its tokens again from what enters it.
// The backward pass does the same with the states' gradients from the last chunk to the
// first.  A sequence that starts in a chunk (backward: ends) makes what leaves it
// independent of what enters, whatever that is.
#pragma once

#include "mixer_dev.h"

namespace hagdn {

typedef float f32x16 __attribute__((ext_vector_type(16)));
#ifdef __HIP_DEVICE_COMPILE__
#define HAGDN_CONSTANT __attribute__((address_space(4)))
#else
#define HAGDN_CONSTANT
#endif

// A wave's 64 channels: a column of a group of channels.
struct Column {
  uint32_t group, c;
  bool mine;  // lanes past the last channel follow it and store nothing
  __device__ Column(uint32_t col, const SsmArgs &a) : Column(col / columns(a), col % columns(a), a) {}
  __device__ Column(uint32_t g, uint32_t col, const SsmArgs &a) : group(g) {
    const uint32_t width = (uint32_t)a.D / a.G, at = col * 64 + lane_id();
    mine = at < width;
    c = g * width + min(at, width - 1);
  }
  __device__ static uint32_t columns(const SsmArgs &a) { return ((uint32_t)a.D / a.G + 63) / 64; }
};

// Rows of B and C of a token and group, in scalar registers: 16 states from 16 k on.
template <int NP> __device__ __forceinline__ const HAGDN_CONSTANT f32x16 *bc_row(const SsmArgs &a, uint32_t t, uint32_t group) {
  return (const HAGDN_CONSTANT f32x16 *)(a.bc + ((size_t)t * a.G + group) * (2 * NP));
}

// log2(e) A of a channel; states past S never decay and are never fed.
template <int NP> __device__ __forceinline__ void load_rates(const SsmArgs &a, uint32_t c, float (&r)[NP]) {
#pragma unroll
  for (int n = 0; n < NP; ++n) r[n] = n < a.S ? a.A[(size_t)c * a.S + n] * kLog2e : 0.f;
}
// Rows [NP][D] of states, at a channel.
template <int NP> __device__ __forceinline__ void load_states(const float *rows, const SsmArgs &a, uint32_t c, float (&h)[NP]) {
#pragma unroll
  for (int n = 0; n < NP; ++n) h[n] = n < a.S ? rows[(size_t)n * a.D + c] : 0.f;
}
template <int NP> __device__ __forceinline__ void store_states(float *rows, const SsmArgs &a, const Column &col, const float (&h)[NP]) {
  if (!col.mine) return;
#pragma unroll
  for (int n = 0; n < NP; ++n)
    if (n < a.S) rows[(size_t)n * a.D + col.c] = h[n];
}
// A sequence's state [D][S] in its caller's order; null: zero.
template <int NP> __device__ __forceinline__ void load_sequence(const float *s, int seq, const SsmArgs &a, uint32_t c, float (&h)[NP]) {
  const float *row = s + ((size_t)seq * a.D + c) * a.S;
#pragma unroll
  for (int n = 0; n < NP; ++n) h[n] = s && n < a.S ? row[n] : 0.f;
}
template <int NP>
__device__ __forceinline__ void store_sequence(float *s, int seq, const SsmArgs &a, const Column &col, const float (&h)[NP]) {
  if (!s || !col.mine) return;
  float *row = s + ((size_t)seq * a.D + col.c) * a.S;
#pragma unroll
  for (int n = 0; n < NP; ++n)
    if (n < a.S) row[n] = h[n];
}
// States of the sequences without tokens pass through.
__device__ __forceinline__ void pass_states(const SsmArgs &a, bool ok, const float *in, float *out, const Column &col) {
  if (!out) return;
  for_empty(a.cu, a.N, a.T, ok, [&](int seq) {
    const size_t at = ((size_t)seq * a.D + col.c) * a.S;
    for (int n = 0; n < a.S && col.mine; ++n) out[at + n] = in ? in[at + n] : 0.f;
  });
}

// The instance of a launcher for a call's types and padded states:
// f(T(), S(), integral_constant<NP>).
template <typename F> hipError_t ssm_dispatch(int states, bool bf16, bool dt_bf16, F f) {
  const auto sized = [&](auto t, auto s) {
    switch (ssm_padded(states)) {
      case 16: return f(t, s, std::integral_constant<int, 16>());
      case 32: return f(t, s, std::integral_constant<int, 32>());
      default: return f(t, s, std::integral_constant<int, 64>());
    }
  };
  if (!bf16) return sized(float(), float());
  return dt_bf16 ? sized(bf16_t(), bf16_t()) : sized(bf16_t(), float());
}

}  // namespace hagdn

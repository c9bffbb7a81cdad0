// ssm.h -- shared parts of the selective scan's kernels.
//
// The scan.  Per channel d and state n, with the step size dt_t (per channel) and B_t, C_t
// (per group of channels),
//   h_t = a_t h_{t-1} + dt_t x_t B_t,  a_t = e^(dt_t A),   y_t = sum_n C_t h_t.
// A lane holds one channel and all its states in registers, so that the sum over states
// needs no other lane; B and C, which all channels of a group share, come through LDS, where
// every lane reads the same word.  (Through scalar registers each wave waits for its own rows:
// 368 us for the outputs of 32768 x 2048 x 16, 324 through LDS, at the time.)  Tokens are cut
// into chunks, one to a wave:
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

// A wave's 64 channels: a column of a group of channels.
struct Column {
  uint32_t group, c;
  bool mine;  // lanes past the last channel follow it and store nothing
  bool idle;  // all of them: the wave only helps with what its workgroup shares
  __device__ Column(uint32_t g, uint32_t col, const SsmArgs &a) : group(g) {
    const uint32_t width = (uint32_t)a.D / a.G, at = col * 64 + lane_id();
    mine = at < width;
    idle = col * 64 >= width;
    c = g * width + min(at, width - 1);
  }
};

// B (WHAT 1), C (2) or both (3) of TOKENS tokens of one group as fp32 rows in LDS, padded
// with zeros, for the columns that a workgroup goes over together.  The next tokens' are on
// their way in registers meanwhile.
template <typename T, int NP, int WHAT, int TOKENS, int THREADS> struct Maps {
  static constexpr int kRow = WHAT == 3 ? 2 * NP : NP, kAll = TOKENS * kRow, kEach = (kAll + THREADS - 1) / THREADS;
  T v[kEach];
  __device__ void fetch(const SsmArgs &a, uint32_t group, int t, int end) {
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int at = e * THREADS + threadIdx.x, token = t + at / kRow, col = at % kRow, n = col % NP;
      v[e] = T(0);
      if (at < kAll && token < end && n < a.S) {
        const bool isC = WHAT == 2 || col >= NP;
        v[e] = (static_cast<const T *>(isC ? a.C : a.B) + (size_t)token * (isC ? a.Cs : a.Bs))[group * a.S + n];
      }
    }
  }
  __device__ void put(float *rows) const {
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int at = e * THREADS + threadIdx.x;
      if (at < kAll) rows[at] = Elt<T>::to_f32(v[e]);
    }
  }
};

// The compiler cannot trace a value back over this place: work on one token is not to be
// taken out of the loop over a run's sequences, where the work of all tokens at once does not
// fit the registers.
#ifdef __HIP_DEVICE_COMPILE__
#define HAGDN_OPAQUE_VECTOR(v) asm volatile("" : "+v"(v))
#define HAGDN_OPAQUE_SCALAR(v) asm volatile("" : "+s"(v))
#else
#define HAGDN_OPAQUE_VECTOR(v)
#define HAGDN_OPAQUE_SCALAR(v)
#endif

// Rows of floats in LDS at a lane's byte offset, which is opaque (above) in its own register,
// so that the rows' distances become the accesses' constants.
struct LdsRows {
  const HAGDN_LDS char *base;
  uint32_t at;
  __device__ LdsRows(const float *p, uint32_t first) : base((const HAGDN_LDS char *)p), at(first * 4) { HAGDN_OPAQUE_VECTOR(at); }
  __device__ void hold() { HAGDN_OPAQUE_VECTOR(at); }
  __device__ f32x4 four(int i) const { return *(const HAGDN_LDS f32x4 *)(base + at + i * 4); }
};

// The number of states, for conditions that are not to be kept in registers from one use to
// the next.
__device__ __forceinline__ int states(const SsmArgs &a) {
  int n = a.S;
  HAGDN_OPAQUE_SCALAR(n);
  return n;
}

// The first `count` of NP floats of a lane's row, the others zero.
template <int NP> __device__ __forceinline__ void load_row(const float *row, int count, float *v) {
  if (count >= NP) {
#pragma unroll
    for (int n = 0; n < NP; n += 4) {
      const auto p = load_pack<float, 4>(row, n);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[n + k] = p.v[k];
    }
    return;
  }
#pragma unroll
  for (int n = 0; n < NP; ++n) v[n] = n < count ? row[n] : 0.f;
}

// log2(e) A of a channel, from the first-th state on; states past S never decay and are never fed.
template <int NP> __device__ __forceinline__ void load_rates(const SsmArgs &a, uint32_t c, float (&r)[NP], int first = 0) {
  load_row<NP>(a.A + (size_t)c * a.S + first, states(a) - first, r);
#pragma unroll
  for (int n = 0; n < NP; ++n) r[n] *= kLog2e;
}
// Rows of states [padded][D], at a channel, from the first-th on.
template <int NP>
__device__ __forceinline__ void load_states(const float *rows, const SsmArgs &a, uint32_t c, float (&h)[NP], int first = 0) {
  const int count = states(a) - first;
  rows += (size_t)first * a.D;
#pragma unroll
  for (int n = 0; n < NP; ++n) h[n] = n < count ? rows[(size_t)n * a.D + c] : 0.f;
}
template <int NP>
__device__ __forceinline__ void store_states(float *rows, const SsmArgs &a, const Column &col, const float (&h)[NP], int first = 0) {
  const int count = states(a) - first;
  if (!col.mine) return;
  rows += (size_t)first * a.D;
#pragma unroll
  for (int n = 0; n < NP; ++n)
    if (n < count) rows[(size_t)n * a.D + col.c] = h[n];
}
// Some of a sequence's states, from the first-th on, in its caller's order [D][S]; null: zero.
template <int NP>
__device__ __forceinline__ void load_sequence(const float *s, int seq, const SsmArgs &a, uint32_t c, float *h, int first = 0) {
  load_row<NP>(s + ((size_t)seq * a.D + c) * a.S + first, s ? states(a) - first : 0, h);
  // Waited for here, where a sequence begins: else every token's first use of a state would
  // wait for all loads and stores under way (they may be these).
  __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
}
template <int NP>
__device__ __forceinline__ void store_sequence(float *s, int seq, const SsmArgs &a, const Column &col, const float *h, int first = 0) {
  const int count = s ? states(a) - first : 0;
  if (count <= 0 || !col.mine) return;
  float *row = s + ((size_t)seq * a.D + col.c) * a.S + first;
  if (count >= NP) {
#pragma unroll
    for (int n = 0; n < NP; n += 4) store_pack<float, 4>(row, n, Pack<float, 4>{{h[n], h[n + 1], h[n + 2], h[n + 3]}});
    return;
  }
#pragma unroll
  for (int n = 0; n < NP; ++n)
    if (n < count) row[n] = h[n];
}
// States of the sequences without tokens pass through.
__device__ __forceinline__ void pass_states(const SsmArgs &a, bool ok, const float *in, float *out, const Column &col) {
  if (!out) return;
  for_empty(a.cu, a.N, a.T, ok, [&](int seq) {
    const size_t at = ((size_t)seq * a.D + col.c) * a.S;
    for (int n = 0; n < a.S && col.mine; ++n) out[at + n] = in ? in[at + n] : 0.f;
  });
}

// Element c of N rows of a token matrix from t on, the last one before `end` in place of rows
// from there on.
template <typename T, int N>
__device__ __forceinline__ void load_tokens(const void *rows, long stride, int t, int end, uint32_t c, T (&v)[N]) {
  Rows<const T> row(static_cast<const T *>(rows) + (size_t)t * stride, stride, c);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = *row.here();
    if (t + i + 1 < end) row.advance();
  }
}
// The first `count` of N values to rows from t on.
template <typename T, int N>
__device__ __forceinline__ void store_tokens(void *rows, const SsmArgs &a, const Column &col, int t, int count, const float (&v)[N]) {
  if (!col.mine) return;
  Rows<T> out(static_cast<T *>(rows) + (size_t)t * a.D, a.D, col.c);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (i < count) *out.here() = Elt<T>::from_f32(v[i]);
    out.advance();
  }
}
// Step sizes, in 32 bits, from what is given, which raw ones follow with their bias.
template <typename S, int N>
__device__ __forceinline__ void step_sizes(const SsmArgs &a, const S (&given)[N], float bias, float (&v)[N], float (&step)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) step[i] = v[i] = Elt<S>::to_f32(given[i]) + bias;
  if (!a.raw) return;
#pragma unroll
  for (int i = 0; i < N; ++i) step[i] = softplus(v[i]);
}

// The instance of a launcher for a call's types, padded states and waves of a workgroup:
// f(T(), S(), integral_constant<NP>, integral_constant<W>).
template <typename F> hipError_t ssm_dispatch(const SsmArgs &a, bool bf16, bool dt_bf16, F f) {
  const auto sized = [&](auto t, auto s) {
    const auto wide = [&](auto np) {
      if (ssm_waves(a.D, a.G) == 1) return f(t, s, np, std::integral_constant<int, 1>());
      return f(t, s, np, std::integral_constant<int, 4>());
    };
    switch (ssm_padded(a.S)) {
      case 16: return wide(std::integral_constant<int, 16>());
      case 32: return wide(std::integral_constant<int, 32>());
      default: return wide(std::integral_constant<int, 64>());
    }
  };
  if (!bf16) return sized(float(), float());
  return dt_bf16 ? sized(bf16_t(), bf16_t()) : sized(bf16_t(), float());
}

}  // namespace hagdn

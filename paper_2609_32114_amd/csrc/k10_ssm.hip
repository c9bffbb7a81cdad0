// k10_ssm.hip -- the selective state space scan, forward (ssm.h has the scheme), and its
// step for single tokens.
#include "ssm.h"

namespace hagdn {

// B and C as rows of fp32, padded with zeros; the first workgroup checks the offsets.
template <typename T> __global__ __launch_bounds__(256) void ssm_setup_kernel(SsmArgs a, int padded) {
  const size_t total = (size_t)a.T * a.G * 2 * padded;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (size_t)gridDim.x * 256) {
    const size_t row = i / (2 * padded), t = row / a.G;  // padded: a power of two
    const int e = (int)(i & (2 * padded - 1)), n = e & (padded - 1), g = (int)(row - t * a.G);
    const T *src = e < padded ? static_cast<const T *>(a.B) + t * a.Bs : static_cast<const T *>(a.C) + t * a.Cs;
    a.bc[i] = n < a.S ? Elt<T>::to_f32(src[g * a.S + n]) : 0.f;
  }
  if (blockIdx.x != 0) return;
  const bool ok = offsets_ok(a.cu, a.N, a.T);
  if (threadIdx.x == 0) *a.status = ok ? 0 : kDevBadSeqlens;
}
hipError_t launch_ssm_setup(const SsmArgs &a, bool bf16, hipStream_t s) {
  const int padded = ssm_padded(a.S);
  const size_t total = (size_t)a.T * a.G * 2 * padded, blocks = (total + 1023) / 1024;
  const dim3 grid((unsigned)(blocks < 1 ? 1 : blocks < 8192 ? blocks : 8192));
  if (bf16) hipLaunchKernelGGL((ssm_setup_kernel<bf16_t>), grid, dim3(256), 0, s, a, padded);
  else hipLaunchKernelGGL((ssm_setup_kernel<float>), grid, dim3(256), 0, s, a, padded);
  return hipGetLastError();
}

constexpr int kSsmRows = 8;  // tokens whose rows are on their way at once; divides every chunk and group

// A chunk's tokens: what it leaves of a zero state (OUT false), or its outputs.
template <typename T, typename S, int NP, bool OUT>
__global__ __launch_bounds__(256) void ssm_scan_kernel(SsmArgs a, uint32_t cols, uint32_t items) {
  const uint32_t item = uniform(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (item >= items) return;
  const int chunk = (int)(item / cols);
  const Column col(item % cols, a);
  const uint32_t c = col.c;
  const bool ok = uniform(*a.status) == 0;
  if (OUT && chunk == 0) pass_states(a, ok, a.s0, a.s_final, col);
  const int t0 = chunk * a.chunk, t1 = (int)min((long)t0 + a.chunk, (long)a.T);
  if (!ok || t0 >= t1) return;

  float A[NP], h[NP];
  load_rates(a, c, A);
  if (OUT && chunk > 0) load_states(a.maps + (size_t)chunk * NP * a.D, a, c, h);
  else for (int n = 0; n < NP; ++n) h[n] = 0.f;
  const float bias = a.raw && a.bias ? a.bias[c] : 0.f, skip = OUT && a.skip ? a.skip[c] : 0.f;
  Cursor q(a.cu, a.N, a.T, t0);
  int first = q.start == t0 ? t0 : q.end;  // the next token that starts a sequence
  bool reset = false;
  float sum = 0.f;
  for (int base = t0; base < t1; base += kSsmRows) {
    T x[kSsmRows], z[kSsmRows];
    S dt[kSsmRows];
#pragma unroll
    for (int i = 0; i < kSsmRows; ++i) {
      const size_t t = min(base + i, t1 - 1);
      x[i] = static_cast<const T *>(a.x)[t * a.xs + c];
      dt[i] = static_cast<const S *>(a.dt)[t * a.dts + c];
      if (OUT) z[i] = a.z ? static_cast<const T *>(a.z)[t * a.zs + c] : T(0);
    }
    if (OUT && a.ckpt && base % (512 / NP) == 0) store_states(a.ckpt + (size_t)(base / (512 / NP)) * NP * a.D, a, col, h);
#pragma unroll
    for (int i = 0; i < kSsmRows; ++i) {
      const int t = base + i;
      if (t >= t1) break;
      if (t == first) {
        if (t == q.end) q.next();
        load_sequence(a.s0, q.seq, a, c, h);
        first = q.end;
        reset = true;
      }
      const float u = Elt<T>::to_f32(x[i]);
      float step = Elt<S>::to_f32(dt[i]);
      if (a.raw) step = softplus(step + bias);
      const float in = step * u;
      if (!OUT) sum += step;
      const HAGDN_CONSTANT f32x16 *row = bc_row<NP>(a, t, col.group);
      float y = skip * u;
#pragma unroll
      for (int k = 0; k < NP / 16; ++k) {
        const f32x16 B = row[k], C = OUT ? row[NP / 16 + k] : f32x16(0.f);
#pragma unroll
        for (int n = 0; n < 16; ++n) {
          float &s = h[16 * k + n];
          s = __builtin_fmaf(__builtin_amdgcn_exp2f(step * A[16 * k + n]), s, in * B[n]);
          if (OUT) y = __builtin_fmaf(C[n], s, y);
        }
      }
      if (OUT) {
        if (a.z) y *= silu(Elt<T>::to_f32(z[i]));
        if (col.mine) static_cast<T *>(a.y)[(size_t)t * a.D + c] = Elt<T>::from_f32(y);
        if (t + 1 == q.end) store_sequence(a.s_final, q.seq, a, col, h);
      }
    }
  }
  if (OUT) return;
  store_states(a.maps + (size_t)chunk * NP * a.D, a, col, h);
  if (col.mine) a.sums[(size_t)chunk * a.D + c] = sum;
  if (item % cols == 0 && lane_id() == 0) a.resets[chunk] = reset;
}

// What enters each chunk, in place of what it leaves of nothing.  A workgroup has one state
// of 64 channels; its 16 waves take the chunks in 16 runs, fold their own, meet in LDS and
// go over their run again.  The last chunk in the scan's order passes nothing on.
template <bool BACKWARD> __global__ __launch_bounds__(1024) void ssm_carry_kernel(SsmArgs a, int padded) {
  __shared__ float sState[16][64], sSum[16][64];
  __shared__ int sReset[16];
  if (*a.status != 0) return;
  const int wave = uniform(threadIdx.x >> 6), lane = lane_id();
  const uint32_t at = blockIdx.x * 64 + lane, c = min(at, (uint32_t)a.D - 1);
  const int n = blockIdx.y;
  const float rate = a.A[(size_t)c * a.S + n] * kLog2e;
  const int share = (a.chunks + 15) / 16, lo = wave * share, hi = min(lo + share, a.chunks);
  const auto row = [&](int i) { return BACKWARD ? a.chunks - 1 - i : i; };
  float state = 0.f, sum = 0.f;
  int reset = 0;
#pragma unroll 4
  for (int i = lo; i < min(hi, a.chunks - 1); ++i) {
    const int k = row(i);
    const float left = a.maps[((size_t)k * padded + n) * a.D + c], part = a.sums[(size_t)k * a.D + c];
    const int r = uniform(a.resets[k]);
    state = r ? left : __builtin_fmaf(__builtin_amdgcn_exp2f(rate * part), state, left);
    sum += part;
    reset |= r;
  }
  sState[wave][lane] = state;
  sSum[wave][lane] = sum;
  if (lane == 0) sReset[wave] = reset;
  __syncthreads();
  float s = 0.f;
  for (int w = 0; w < wave; ++w)
    s = sReset[w] ? sState[w][lane] : __builtin_fmaf(__builtin_amdgcn_exp2f(rate * sSum[w][lane]), s, sState[w][lane]);
#pragma unroll 4
  for (int i = lo; i < hi; ++i) {
    const int k = row(i);
    float *p = a.maps + ((size_t)k * padded + n) * a.D + c;
    float next = 0.f;
    if (i + 1 < a.chunks) {
      const float left = *p, part = a.sums[(size_t)k * a.D + c];
      next = uniform(a.resets[k]) ? left : __builtin_fmaf(__builtin_amdgcn_exp2f(rate * part), s, left);
    }
    if (at < (uint32_t)a.D) *p = s;
    s = next;
  }
}
hipError_t launch_ssm_carry(const SsmArgs &a, bool backward, hipStream_t s) {
  const dim3 grid(((unsigned)a.D + 63) / 64, (unsigned)a.S);
  const int padded = ssm_padded(a.S);
  if (backward) hipLaunchKernelGGL((ssm_carry_kernel<true>), grid, dim3(1024), 0, s, a, padded);
  else hipLaunchKernelGGL((ssm_carry_kernel<false>), grid, dim3(1024), 0, s, a, padded);
  return hipGetLastError();
}

hipError_t launch_ssm_forward(const SsmArgs &a, bool bf16, bool dt_bf16, hipStream_t s) {
  hipError_t e = launch_ssm_setup(a, bf16, s);
  if (e != hipSuccess) return e;
  return ssm_dispatch(a.S, bf16, dt_bf16, [&](auto t, auto st, auto np) {
    using T = decltype(t);
    using S = decltype(st);
    constexpr int NP = decltype(np)::value;
    const uint32_t cols = (uint32_t)ssm_columns(a.D, a.G) * a.G;
    const long all = (long)a.chunks * cols;
    if (all > 0x3fffffffl) return hipErrorInvalidValue;
    if (a.chunks > 1) {
      const uint32_t items = (uint32_t)(all - cols);
      hipLaunchKernelGGL((ssm_scan_kernel<T, S, NP, false>), dim3((items + 3) / 4), dim3(256), 0, s, a, cols, items);
      hipError_t e = hipGetLastError();
      if (e == hipSuccess) e = launch_ssm_carry(a, false, s);
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((ssm_scan_kernel<T, S, NP, true>), dim3(((uint32_t)all + 3) / 4), dim3(256), 0, s, a, cols, (uint32_t)all);
    return hipGetLastError();
  });
}

// ------------------------------------------------------------- single tokens
// P states of a channel to a lane, S / P lanes (a power of two up to 16) to a channel; P = 0: a
// lane goes over all of a channel's states.
template <typename T, typename S, int P>
__global__ __launch_bounds__(256) void ssm_step_kernel(SsmStepArgs a, uint32_t lanes, uint64_t items) {
  for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < items; i += (uint64_t)gridDim.x * 256) {
    const uint32_t part = (uint32_t)i & (lanes - 1);
    const uint64_t row = i / lanes;
    const uint32_t n = (uint32_t)(row / (uint32_t)a.D), c = (uint32_t)(row - (uint64_t)n * a.D);
    const int slot = a.slots ? a.slots[n] : (int)n;
    const bool live = slot >= 0 && slot < a.num_slots;
    float y = 0.f, x = 0.f;
    if (live) {
      x = Elt<T>::to_f32(static_cast<const T *>(a.x)[(size_t)n * a.xs + c]);
      float step = Elt<S>::to_f32(static_cast<const S *>(a.dt)[(size_t)n * a.dts + c]);
      if (a.raw) step = softplus(step + (a.bias ? a.bias[c] : 0.f));
      const float in = step * x;
      const uint32_t g = c / ((uint32_t)a.D / a.G);
      const T *B = static_cast<const T *>(a.B) + (size_t)n * a.Bs + g * a.S, *C = static_cast<const T *>(a.C) + (size_t)n * a.Cs + g * a.S;
      float *state = a.state + ((size_t)slot * a.D + c) * a.S;
      const float *A = a.A + (size_t)c * a.S;
      if constexpr (P > 0) {
        const uint32_t at = part * P;
        auto s = load_pack<float, P>(state, at);
        const auto r = load_pack<float, P>(A, at);
        const auto b = load_pack<T, P>(B, at), w = load_pack<T, P>(C, at);
#pragma unroll
        for (int k = 0; k < P; ++k) {
          s.v[k] = __builtin_fmaf(__builtin_amdgcn_exp2f(step * (r.v[k] * kLog2e)), s.v[k], in * Elt<T>::to_f32(b.v[k]));
          y = __builtin_fmaf(Elt<T>::to_f32(w.v[k]), s.v[k], y);
        }
        store_pack<float, P>(state, at, s);
      } else {
        for (int k = 0; k < a.S; ++k) {
          const float s = __builtin_fmaf(__builtin_amdgcn_exp2f(step * (A[k] * kLog2e)), state[k], in * Elt<T>::to_f32(B[k]));
          y = __builtin_fmaf(Elt<T>::to_f32(C[k]), s, y);
          state[k] = s;
        }
      }
    }
    for (uint32_t d = 1; d < lanes; d *= 2) y += __shfl_xor(y, (int)d);
    if (part == 0) {
      if (live) {
        if (a.skip) y = __builtin_fmaf(a.skip[c], x, y);
        if (a.z) y *= silu(Elt<T>::to_f32(static_cast<const T *>(a.z)[(size_t)n * a.zs + c]));
      }
      static_cast<T *>(a.y)[(size_t)n * a.D + c] = Elt<T>::from_f32(y);
    }
  }
}

template <typename T, typename S> hipError_t ssm_step(const SsmStepArgs &a, hipStream_t s) {
  const bool four = a.S % 4 == 0 && (a.S & (a.S - 1)) == 0;
  const uint32_t lanes = four ? (uint32_t)a.S / 4 : 1;
  const uint64_t items = (uint64_t)a.N * a.D * lanes, blocks = (items + 255) / 256;
  const dim3 grid((unsigned)(blocks < 1u << 20 ? blocks : 1u << 20));
  if (four) hipLaunchKernelGGL((ssm_step_kernel<T, S, 4>), grid, dim3(256), 0, s, a, lanes, items);
  else hipLaunchKernelGGL((ssm_step_kernel<T, S, 0>), grid, dim3(256), 0, s, a, lanes, items);
  return hipGetLastError();
}
hipError_t launch_ssm_step(const SsmStepArgs &a, bool bf16, bool dt_bf16, hipStream_t s) {
  if (!bf16) return ssm_step<float, float>(a, s);
  return dt_bf16 ? ssm_step<bf16_t, bf16_t>(a, s) : ssm_step<bf16_t, float>(a, s);
}

}  // namespace hagdn

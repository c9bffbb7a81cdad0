// k10_ssm.hip -- the selective state space scan, forward (ssm.h has the scheme), and its
// step for single tokens.
//
// Bound by its arithmetic: per token, channel and state a product, an exponential (8 cycles
// of a wave, the others 4) and three or, for outputs, four more operations, and both passes over
// the chunks take them.  32768 tokens x 2048 channels x 16 states, x, z, y and dt in bf16: what
// chunks leave 204 to 224 us, what enters them 10, outputs 266 to 289 (the clock falls under
// this load from 2.4 to 2.2 GHz), where 539 MB would take 104 us of HBM.  The vector units are
// busy 90 % of the time; 18 of 82 instructions a token and lane are the step size's softplus
// and conversions, in outputs 29 of 109.  On the way (both passes): B and C through scalar loads
// and each sequence's end inside an unrolled loop 697 us; B and C through LDS, ends apart 573;
// the next rows on their way, no copies around the states 535; the hardware's logarithm 520.
#include "ssm.h"

namespace hagdn {

constexpr int kSsmRows = 8;  // tokens whose rows are on their way at once; divides every chunk and group

// A chunk's tokens: what it leaves of a zero state (OUT false), or its outputs.  The W waves
// of a workgroup have columns of one group and the same chunk.
template <typename T, typename S, int NP, int W, bool OUT>
__global__ __launch_bounds__(W * 64, NP == 16 ? 4 : NP == 32 ? 2 : 1) void ssm_scan_kernel(SsmArgs a, uint32_t teams) {
  using Stage = Maps<T, NP, OUT ? 3 : 1, kSsmRows, W * 64>;
  __shared__ __align__(16) float sMaps[2][Stage::kAll];
  __shared__ int32_t sCu[kCheckInPlace + 1];
  Offsets32 cu;
  const bool ok = stage_offsets(a.cu, a.N, a.T, a.status, sCu, cu);
  const uint32_t team = blockIdx.x % (teams * a.G), group = team / teams;
  const int chunk = (int)(blockIdx.x / (teams * a.G));
  const Column col(group, (team - group * teams) * W + uniform(threadIdx.x >> 6), a);
  const uint32_t c = col.c;
  if (OUT && chunk == 0) pass_states(a, ok, a.s0, a.s_final, col);
  int t0 = chunk * a.chunk;
  const int t1 = (int)min((long)t0 + a.chunk, (long)a.T);
  if (!ok || t0 >= t1) return;
  if (!OUT) {  // what a chunk leaves is its last sequence's
    const Cursor last(cu, t1 - 1);
    if (last.start > t0) t0 += (last.start - t0) / kSsmRows * kSsmRows;
  }

  // x, dt, B and C of the first tokens are on their way before anything waits; z, which only
  // the outputs need, is read in its turn
  T x[kSsmRows], z[kSsmRows];
  S dt[kSsmRows];
  Stage stage;
  load_tokens(a.dt, a.dts, t0, t1, c, dt);
  load_tokens(a.x, a.xs, t0, t1, c, x);
  stage.fetch(a, group, t0, t1);
  float A[NP], h[NP];
  load_rates(a, c, A);
  if (OUT && chunk > 0) load_states(a.maps + (size_t)chunk * NP * a.D, a, c, h);
  else for (int n = 0; n < NP; ++n) h[n] = 0.f;
  const float bias = a.raw && a.bias ? a.bias[c] : 0.f, skip = OUT && a.skip ? a.skip[c] : 0.f;
  Cursor q(cu, t0);
  int first = q.start == t0 ? t0 : q.end;  // the next token that starts a sequence
  bool reset = false;
  float sum = 0.f;
  int turn = 0;
  for (int base = t0; base < t1; base += kSsmRows, turn ^= 1) {
    const int count = min(kSsmRows, t1 - base);
    stage.put(sMaps[turn]);
    __syncthreads();
    if (col.idle) {
      if (base + kSsmRows < t1) stage.fetch(a, group, base + kSsmRows, t1);
      continue;
    }
    float u[kSsmRows], given[kSsmRows], step[kSsmRows], y[kSsmRows];
    step_sizes(a, dt, bias, given, step);
#pragma unroll
    for (int i = 0; i < kSsmRows; ++i) u[i] = Elt<T>::to_f32(x[i]);
    if (OUT && a.z) load_tokens(a.z, a.zs, base, t1, c, z);
    if (base + kSsmRows < t1) {
      load_tokens(a.dt, a.dts, base + kSsmRows, t1, c, dt);
      load_tokens(a.x, a.xs, base + kSsmRows, t1, c, x);
      stage.fetch(a, group, base + kSsmRows, t1);
    }
    if (OUT && a.ckpt && base % kSsmGroup == 0) store_states(a.ckpt + (size_t)(base / kSsmGroup) * NP * a.D, a, col, h);
    LdsRows rows(sMaps[0], turn * Stage::kAll);
    for (int lo = 0; lo < count;) {  // from one sequence's first token to the next one's
      if (base + lo == first) {
        if (first == q.end) q.next();
        load_sequence<NP>(a.s0, q.seq, a, c, h);
        first = q.end;
        reset = true;
      }
      const int hi = min(count, first - base);
#pragma unroll
      for (int i = 0; i < kSsmRows; ++i)
        if (i >= lo && i < hi) {
          rows.hold();
          HAGDN_OPAQUE_VECTOR(step[i]);
          const float in = step[i] * u[i];
          if (!OUT) sum += step[i];
          y[i] = skip * u[i];
#pragma unroll
          for (int n = 0; n < NP; n += 4) {
            const f32x4 B = rows.four(i * Stage::kRow + n), C = OUT ? rows.four(i * Stage::kRow + NP + n) : f32x4{};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              float &s = h[n + k];
              // (in place: a product and a fused sum into the state's own register)
              s *= __builtin_amdgcn_exp2f(step[i] * A[n + k]);
              s = __builtin_fmaf(in, B[k], s);
              if (OUT) y[i] = __builtin_fmaf(C[k], s, y[i]);
            }
          }
        }
      if (OUT && base + hi == q.end) store_sequence<NP>(a.s_final, q.seq, a, col, h);
      lo = hi;
    }
    if (OUT) {
      if (a.z) {
#pragma unroll
        for (int i = 0; i < kSsmRows; ++i) y[i] *= silu(Elt<T>::to_f32(z[i]));
      }
      store_tokens<T>(a.y, a, col, base, count, y);
    }
  }
  if (OUT) return;
  store_states(a.maps + (size_t)chunk * NP * a.D, a, col, h);
  if (col.mine) a.sums[(size_t)chunk * a.D + c] = sum;
  if (team == 0 && threadIdx.x == 0) a.resets[chunk] = reset;
}

// What enters each chunk, in place of what it leaves of nothing.  A workgroup has one state
// of 64 channels; its 16 waves take the chunks in 16 runs, fold their own, meet in LDS and
// go over their run again.  The last chunk in the scan's order passes nothing on.  Runs of up to
// kHeld chunks stay in registers for that.
constexpr int kHeld = 8;
struct Passed {  // by a chunk
  float left, sum;
  bool reset;
};
template <bool BACKWARD, bool HELD> __global__ __launch_bounds__(1024) void ssm_carry_kernel(SsmArgs a, int padded) {
  __shared__ float sState[16][64], sSum[16][64];
  __shared__ int sReset[16];
  if (*a.status != 0) return;
  const int wave = uniform(threadIdx.x >> 6), lane = lane_id();
  const uint32_t at = blockIdx.x * 64 + lane, c = min(at, (uint32_t)a.D - 1);
  const int n = blockIdx.y;
  const float rate = a.A[(size_t)c * a.S + n] * kLog2e;
  const int share = (a.chunks + 15) / 16, lo = wave * share, hi = min(lo + share, a.chunks);
  const auto place = [&](int i) {
    return a.maps + ((size_t)(BACKWARD ? a.chunks - 1 - i : i) * padded + n) * a.D + c;
  };
  const auto passed = [&](int i) {  // the last one's own is not there
    const int k = BACKWARD ? a.chunks - 1 - i : i;
    return i < min(hi, a.chunks - 1) ? Passed{*place(i), a.sums[(size_t)k * a.D + c], uniform(a.resets[k]) != 0} : Passed{0.f, 0.f, false};
  };
  // The factor is applied as two of half its exponent, and not to a state of zero: over a run of
  // chunks a positive rate may pass fp32's range where the state itself, small or not fed yet, does not.
  const auto fold = [&](const Passed &p, float s) {
    const float half = __builtin_amdgcn_exp2f(0.5f * rate * p.sum);
    return p.reset || s == 0.f ? p.left : __builtin_fmaf(half, half * s, p.left);
  };
  Passed held[kHeld];
  float state = 0.f, sum = 0.f;
  int reset = 0;
  const auto gather = [&](const Passed &p) {
    state = fold(p, state);
    sum += p.sum;
    reset |= p.reset;
  };
  if (HELD) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i) held[i] = passed(lo + i);
#pragma unroll
    for (int i = 0; i < kHeld; ++i) gather(held[i]);
  } else {
#pragma unroll 4
    for (int i = lo; i < hi; ++i) gather(passed(i));
  }
  sState[wave][lane] = state;
  sSum[wave][lane] = sum;
  if (lane == 0) sReset[wave] = reset;
  __syncthreads();
  float s = 0.f;
  for (int w = 0; w < wave; ++w) s = fold(Passed{sState[w][lane], sSum[w][lane], sReset[w] != 0}, s);
  const auto give = [&](int i, const Passed &p) {
    if (i < hi && at < (uint32_t)a.D) *place(i) = s;
    s = fold(p, s);
  };
  if (HELD) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i) give(lo + i, held[i]);
  } else {
#pragma unroll 4
    for (int i = lo; i < hi; ++i) give(i, passed(i));
  }
}
hipError_t launch_ssm_carry(const SsmArgs &a, bool backward, hipStream_t s) {
  const dim3 grid(((unsigned)a.D + 63) / 64, (unsigned)a.S);
  const int padded = ssm_padded(a.S);
  const bool held = a.chunks <= 16 * kHeld;
  if (backward && held) hipLaunchKernelGGL((ssm_carry_kernel<true, true>), grid, dim3(1024), 0, s, a, padded);
  else if (backward) hipLaunchKernelGGL((ssm_carry_kernel<true, false>), grid, dim3(1024), 0, s, a, padded);
  else if (held) hipLaunchKernelGGL((ssm_carry_kernel<false, true>), grid, dim3(1024), 0, s, a, padded);
  else hipLaunchKernelGGL((ssm_carry_kernel<false, false>), grid, dim3(1024), 0, s, a, padded);
  return hipGetLastError();
}

hipError_t launch_ssm_forward(const SsmArgs &a, bool bf16, bool dt_bf16, hipStream_t s) {
  return ssm_dispatch(a, bf16, dt_bf16, [&](auto t, auto st, auto np, auto w) {
    using T = decltype(t);
    using S = decltype(st);
    constexpr int NP = decltype(np)::value, W = decltype(w)::value;
    const uint32_t teams = (uint32_t)ssm_teams(a.D, a.G);
    const long each = (long)teams * a.G, all = a.chunks * each;
    if (all > 0x7fffffffl) return hipErrorInvalidValue;
    hipError_t e = a.N > kCheckInPlace ? launch_check_offsets(a.cu, a.N, a.T, a.status, s) : hipSuccess;
    if (e != hipSuccess) return e;
    if (a.chunks > 1) {
      hipLaunchKernelGGL((ssm_scan_kernel<T, S, NP, W, false>), dim3((unsigned)(all - each)), dim3(W * 64), 0, s, a, teams);
      e = hipGetLastError();
      if (e == hipSuccess) e = launch_ssm_carry(a, false, s);
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((ssm_scan_kernel<T, S, NP, W, true>), dim3((unsigned)all), dim3(W * 64), 0, s, a, teams);
    return hipGetLastError();
  });
}

// ------------------------------------------------------------- single tokens
// Four states of a channel to a lane, the power of two of lanes (up to 16) that covers S to a
// channel, so that a wave's loads lie side by side. QUADS, where 4 divides S: a lane's four are
// neighbours, in one load. Otherwise they stand a channel's lanes apart (168 x 1280 channels x 61
// states 37 us, 2.9 TB/s of states; with a channel's states in one lane, apart in memory, 197).
// 256 x 4096 x 16 in bf16: 31 us, 4.3 TB/s of states.
template <typename T, typename S, bool QUADS>
__global__ __launch_bounds__(256) void ssm_step_kernel(SsmStepArgs a, uint32_t lanes, uint32_t items) {
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < items; i += gridDim.x * 256) {  // N x D x S < 2^31
    const uint32_t part = i & (lanes - 1), row = i / lanes, n = row / (uint32_t)a.D, c = row - n * (uint32_t)a.D;
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
      if (QUADS) {
        const uint32_t at = part * 4;
        if (at < (uint32_t)a.S) {
          auto s = load_pack<float, 4>(state, at);
          const auto r = load_pack<float, 4>(A, at);
          const auto b = load_pack<T, 4>(B, at), w = load_pack<T, 4>(C, at);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            s.v[k] = __builtin_fmaf(__builtin_amdgcn_exp2f(step * (r.v[k] * kLog2e)), s.v[k], in * Elt<T>::to_f32(b.v[k]));
            y = __builtin_fmaf(Elt<T>::to_f32(w.v[k]), s.v[k], y);
          }
          store_pack<float, 4>(state, at, s);
        }
      } else {
        float s[4], r[4], b[4], w[4];
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) {
          const uint32_t at = part + k * lanes;
          const bool in_range = at < (uint32_t)a.S;
          s[k] = in_range ? state[at] : 0.f;
          r[k] = in_range ? A[at] : 0.f;
          b[k] = in_range ? Elt<T>::to_f32(B[at]) : 0.f;
          w[k] = in_range ? Elt<T>::to_f32(C[at]) : 0.f;
        }
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) {
          const uint32_t at = part + k * lanes;
          if (at >= (uint32_t)a.S) break;
          s[k] = __builtin_fmaf(__builtin_amdgcn_exp2f(step * (r[k] * kLog2e)), s[k], in * b[k]);
          y = __builtin_fmaf(w[k], s[k], y);
          state[at] = s[k];
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
  uint32_t lanes = 1;
  while (lanes * 4 < (uint32_t)a.S) lanes *= 2;
  const uint32_t items = (uint32_t)a.N * a.D * lanes, blocks = (items + 255) / 256;
  const dim3 grid(blocks < 1u << 20 ? blocks : 1u << 20);
  if (a.S % 4 == 0) hipLaunchKernelGGL((ssm_step_kernel<T, S, true>), grid, dim3(256), 0, s, a, lanes, items);
  else hipLaunchKernelGGL((ssm_step_kernel<T, S, false>), grid, dim3(256), 0, s, a, lanes, items);
  return hipGetLastError();
}
hipError_t launch_ssm_step(const SsmStepArgs &a, bool bf16, bool dt_bf16, hipStream_t s) {
  if (!bf16) return ssm_step<float, float>(a, s);
  return dt_bf16 ? ssm_step<bf16_t, bf16_t>(a, s) : ssm_step<bf16_t, float>(a, s);
}

}  // namespace hagdn

// k11_ssm_backward.hip -- the selective scan's backward pass (ssm.h has the scheme).  With
// dy the gradient of the ungated output and e the gradient that reaches a state from later
// tokens,
//   dh_t = e_t + C_t dy_t,  e_{t-1} = a_t dh_t,
//   dC_t = sum_d dy_t h_t,  dB_t = sum_d dh_t dt_t x_t,  w_t = sum_n dh_t B_t,
//   dx_t = dt_t w_t + skip dy_t,  d(dt_t) = x_t w_t + sum_n A dh_t a_t h_{t-1},
//   dA = sum_t dt_t dh_t a_t h_{t-1}.
#include "ssm.h"

namespace hagdn {

constexpr int kBackRows = 8;

// What a chunk passes back of a zero gradient.
template <typename T, typename S, int NP>
__global__ __launch_bounds__(256) void ssm_back_local_kernel(SsmArgs a, uint32_t cols, uint32_t items) {
  const uint32_t item = uniform(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (item >= items) return;
  const int chunk = 1 + (int)(item / cols);  // the first chunk passes nothing on
  const Column col(item % cols, a);
  const uint32_t c = col.c;
  if (uniform(*a.status) != 0) return;
  const int t0 = chunk * a.chunk, t1 = (int)min((long)t0 + a.chunk, (long)a.T);
  float A[NP], e[NP];
  load_rates(a, c, A);
#pragma unroll
  for (int n = 0; n < NP; ++n) e[n] = 0.f;
  const float bias = a.raw && a.bias ? a.bias[c] : 0.f;
  Cursor q(a.cu, a.N, a.T, t1 - 1);
  bool reset = false;
  float sum = 0.f;
  for (int top = t1; top > t0; top -= kBackRows) {
    T dy[kBackRows], z[kBackRows];
    S dt[kBackRows];
#pragma unroll
    for (int i = 0; i < kBackRows; ++i) {
      const size_t t = max(top - 1 - i, t0);
      dy[i] = static_cast<const T *>(a.dy)[t * a.dys + c];
      dt[i] = static_cast<const S *>(a.dt)[t * a.dts + c];
      z[i] = a.z ? static_cast<const T *>(a.z)[t * a.zs + c] : T(0);
    }
#pragma unroll
    for (int i = 0; i < kBackRows; ++i) {
      const int t = top - 1 - i;
      if (t < t0) break;
      if (t + 1 == q.start) q.previous();
      if (t + 1 == q.end) {
        load_sequence(a.dfinal, q.seq, a, c, e);
        reset = true;
      }
      float d = Elt<T>::to_f32(dy[i]), step = Elt<S>::to_f32(dt[i]);
      if (a.raw) step = softplus(step + bias);
      if (a.z) d *= silu(Elt<T>::to_f32(z[i]));
      sum += step;
      const HAGDN_CONSTANT f32x16 *row = bc_row<NP>(a, t, col.group);
#pragma unroll
      for (int k = 0; k < NP / 16; ++k) {
        const f32x16 C = row[NP / 16 + k];
#pragma unroll
        for (int n = 0; n < 16; ++n) {
          float &v = e[16 * k + n];
          v = __builtin_amdgcn_exp2f(step * A[16 * k + n]) * __builtin_fmaf(C[n], d, v);
        }
      }
    }
  }
  store_states(a.maps + (size_t)chunk * NP * a.D, a, col, e);
  if (col.mine) a.sums[(size_t)chunk * a.D + c] = sum;
  if (item % cols == 0 && lane_id() == 0) a.resets[chunk] = reset;
}

// Sums of 16 values over the wave's 64 lanes: value n to the lanes 4 n .. 4 n + 3.  Each
// exchange halves the values that a lane still holds: 35 instructions instead of the 96 of
// 16 separate sums.
template <int CTRL> __device__ __forceinline__ float dpp(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float sum_lanes(const float (&in)[16]) {
  float v[8], w[4];
#pragma unroll
  for (int i = 0; i < 8; ++i) {  // halves of 32 lanes
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(in[i]), __float_as_uint(in[i + 8]), false, false);
    v[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {  // rows of 16
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[i]), __float_as_uint(v[i + 4]), false, false);
    w[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  const bool high8 = lane_id() & 8, high4 = lane_id() & 4;
#pragma unroll
  for (int i = 0; i < 2; ++i) w[i] = (high8 ? w[i + 2] : w[i]) + dpp<0x128>(high8 ? w[i] : w[i + 2]);  // lane + 8 of 16
  float s = (high4 ? w[1] : w[0]) + dpp<0x141>(high4 ? w[0] : w[1]);                                   // lane 7 - i of 8
  s += dpp<0xb1>(s);                                                                                   // lane ^ 1
  return s + dpp<0x4e>(s);                                                                             // lane ^ 2
}

// The forms for NP padded states: SUB tokens whose states are held in registers, four
// times as many to a saved state, WAVES columns to a workgroup.  The states at the four
// runs' starts lie in LDS.
template <int NP> struct BackForm {
  static constexpr int kSub = 128 / NP, kGroup = 512 / NP, kWaves = NP == 64 ? 2 : 4;  // ssm_waves()
  static constexpr size_t kStates = (size_t)kWaves * 4 * NP * 64, kSums = (size_t)kWaves * kGroup * 2 * NP;
  static constexpr size_t kLds = (kStates + kSums) * sizeof(float);
};

template <typename T, typename S, int NP>
__global__ __launch_bounds__(BackForm<NP>::kWaves * 64, NP == 16 ? 2 : 1) void ssm_backward_kernel(SsmArgs a, uint32_t quads) {
  using F = BackForm<NP>;
  extern __shared__ __align__(16) float lds[];
  const int wave = uniform(threadIdx.x >> 6), lane = lane_id();
  float *starts = lds + (size_t)wave * 4 * NP * 64 + lane;  // [4][NP][64]
  float *sums = lds + F::kStates;                            // [waves][group][2 NP]
  const uint32_t quad = blockIdx.x % (quads * a.G), group = quad / quads, in_group = quad % quads;
  const int chunk = (int)(blockIdx.x / (quads * a.G));
  const Column col(group, in_group * F::kWaves + wave, a);
  const uint32_t c = col.c;
  const bool ok = uniform(*a.status) == 0;
  if (chunk == 0) pass_states(a, ok, a.dfinal, a.ds0, col);
  const int t0 = chunk * a.chunk, t1 = ok ? (int)min((long)t0 + a.chunk, (long)a.T) : t0;

  float A[NP], e[NP], dA[NP], dskip = 0.f, dbias = 0.f;
  load_rates(a, c, A);
#pragma unroll
  for (int n = 0; n < NP; ++n) e[n] = dA[n] = 0.f;
  if (ok && chunk + 1 < a.chunks) load_states(a.maps + (size_t)chunk * NP * a.D, a, c, e);
  const float bias = a.raw && a.bias ? a.bias[c] : 0.f, skip = a.skip ? a.skip[c] : 0.f;
  const auto step_at = [&](size_t t) { return Elt<S>::to_f32(static_cast<const S *>(a.dt)[t * a.dts + c]); };
  const auto x_at = [&](size_t t) { return Elt<T>::to_f32(static_cast<const T *>(a.x)[t * a.xs + c]); };

  for (int g0 = t0 + (t1 - 1 - t0) / F::kGroup * F::kGroup; t1 > t0 && g0 >= t0; g0 -= F::kGroup) {
    const int g1 = min(g0 + F::kGroup, t1);
    float h[NP];
    load_states(a.ckpt + (size_t)(g0 / F::kGroup) * NP * a.D, a, c, h);
    const int subs = (g1 - g0 + F::kSub - 1) / F::kSub;
    {  // the states at the runs' starts
      Cursor q(a.cu, a.N, a.T, g0);
      int first = q.start == g0 ? g0 : q.end;
      for (int sub = 0; sub < subs; ++sub) {
#pragma unroll
        for (int n = 0; n < NP; ++n) starts[(sub * NP + n) * 64] = h[n];
        if (sub + 1 == subs) break;
        const int s0 = g0 + sub * F::kSub;
        float x[F::kSub], dt[F::kSub];
#pragma unroll
        for (int i = 0; i < F::kSub; ++i) {
          x[i] = x_at(s0 + i);
          dt[i] = step_at(s0 + i);
        }
#pragma unroll
        for (int i = 0; i < F::kSub; ++i) {
          const int t = s0 + i;
          if (t == first) {
            if (t == q.end) q.next();
            load_sequence(a.s0, q.seq, a, c, h);
            first = q.end;
          }
          const float step = a.raw ? softplus(dt[i] + bias) : dt[i], in = step * x[i];
          const HAGDN_CONSTANT f32x16 *row = bc_row<NP>(a, t, group);
#pragma unroll
          for (int k = 0; k < NP / 16; ++k) {
            const f32x16 B = row[k];
#pragma unroll
            for (int n = 0; n < 16; ++n)
              h[16 * k + n] = __builtin_fmaf(__builtin_amdgcn_exp2f(step * A[16 * k + n]), h[16 * k + n], in * B[n]);
          }
        }
      }
    }
    for (int sub = subs - 1; sub >= 0; --sub) {
      const int s0 = g0 + sub * F::kSub, s1 = min(s0 + F::kSub, g1);
      float x[F::kSub], v[F::kSub], step[F::kSub], dy[F::kSub], z[F::kSub];  // v: the step as given, with its bias
#pragma unroll
      for (int i = 0; i < F::kSub; ++i) {
        const size_t t = min(s0 + i, s1 - 1);
        x[i] = x_at(t);
        v[i] = step_at(t) + bias;
        dy[i] = col.mine ? Elt<T>::to_f32(static_cast<const T *>(a.dy)[t * a.dys + c]) : 0.f;
        z[i] = a.z ? Elt<T>::to_f32(static_cast<const T *>(a.z)[t * a.zs + c]) : 0.f;
      }
#pragma unroll
      for (int n = 0; n < NP; ++n) h[n] = starts[(sub * NP + n) * 64];
      Cursor q(a.cu, a.N, a.T, s0);
      int first = q.start == s0 ? s0 : q.end;
      float kept[F::kSub][NP];  // a_t h_{t-1}
#pragma unroll
      for (int i = 0; i < F::kSub; ++i) {
        const int t = s0 + i;
        step[i] = a.raw ? softplus(v[i]) : v[i];
        if (t >= s1) break;
        if (t == first) {
          if (t == q.end) q.next();
          load_sequence(a.s0, q.seq, a, c, h);
          first = q.end;
        }
        const float in = step[i] * x[i];
        const HAGDN_CONSTANT f32x16 *row = bc_row<NP>(a, t, group);
#pragma unroll
        for (int k = 0; k < NP / 16; ++k) {
          const f32x16 B = row[k];
#pragma unroll
          for (int m = 0; m < 16; ++m) {
            const int n = 16 * k + m;
            kept[i][n] = __builtin_amdgcn_exp2f(step[i] * A[n]) * h[n];
            h[n] = __builtin_fmaf(in, B[m], kept[i][n]);
          }
        }
      }
#pragma unroll
      for (int i = F::kSub - 1; i >= 0; --i) {
        const int t = s0 + i;
        if (t >= s1) continue;
        if (t + 1 == q.start) q.previous();
        if (t + 1 == q.end) load_sequence(a.dfinal, q.seq, a, c, e);
        const float in = step[i] * x[i];
        Logistic gate = {1.f, 0.f};
        float d = dy[i];
        if (a.z) {
          gate = logistic(z[i]);
          d *= z[i] * gate.s;
        }
        float y = skip * x[i], w = 0.f, ds = 0.f;
        const HAGDN_CONSTANT f32x16 *row = bc_row<NP>(a, t, group);
#pragma unroll
        for (int k = 0; k < NP / 16; ++k) {
          const f32x16 B = row[k], C = row[NP / 16 + k];
          float vB[16], vC[16];
#pragma unroll
          for (int m = 0; m < 16; ++m) {
            const int n = 16 * k + m;
            const float hn = __builtin_fmaf(in, B[m], kept[i][n]), dh = __builtin_fmaf(C[m], d, e[n]);
            y = __builtin_fmaf(C[m], hn, y);
            w = __builtin_fmaf(B[m], dh, w);
            vC[m] = d * hn;
            vB[m] = dh * in;
            const float p = dh * kept[i][n];
            ds = __builtin_fmaf(A[n], p, ds);
            dA[n] = __builtin_fmaf(step[i], p, dA[n]);
            e[n] = __builtin_amdgcn_exp2f(step[i] * A[n]) * dh;
          }
          if (!col.mine) {
#pragma unroll
            for (int m = 0; m < 16; ++m) vB[m] = 0.f;
          }
          const float rB = sum_lanes(vB), rC = sum_lanes(vC);
          if ((lane & 2) == 0)
            sums[((size_t)wave * F::kGroup + (t - g0)) * (2 * NP) + (lane & 1) * NP + 16 * k + (lane >> 2)] = lane & 1 ? rC : rB;
        }
        if (t == q.start) store_sequence(a.ds0, q.seq, a, col, e);
        const float du = step[i] * w + skip * d;
        float dv = x[i] * w + ds * (1.f / kLog2e);
        if (a.raw) dv *= logistic(v[i]).s;
        dskip = __builtin_fmaf(d, x[i], dskip);
        dbias += dv;
        if (col.mine) {
          const size_t at = (size_t)t * a.D + c;
          static_cast<T *>(a.dx)[at] = Elt<T>::from_f32(du);
          static_cast<S *>(a.ddt)[at] = Elt<S>::from_f32(dv);
          if (a.z) static_cast<T *>(a.dz)[at] = Elt<T>::from_f32(dy[i] * y * (gate.s * __builtin_fmaf(z[i], gate.rest, 1.f)));
        }
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < (g1 - g0) * 2 * NP; i += F::kWaves * 64) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < F::kWaves; ++w) s += sums[(size_t)w * F::kGroup * 2 * NP + i];
      const size_t t = g0 + i / (2 * NP);
      a.dbc[(((size_t)in_group * a.T + t) * a.G + group) * (2 * NP) + i % (2 * NP)] = s;
    }
    __syncthreads();
  }
  if (!col.mine) return;
  float *out = a.dweights + (size_t)chunk * (NP + 2) * a.D + c;
#pragma unroll
  for (int n = 0; n < NP; ++n)
    if (n < a.S) out[(size_t)n * a.D] = dA[n];
  out[(size_t)NP * a.D] = dskip;
  out[(size_t)(NP + 1) * a.D] = dbias;
}

// dB and dC from the column groups' sums, in their order.
template <typename T> __global__ __launch_bounds__(256) void ssm_sum_bc_kernel(SsmArgs a, int padded, uint32_t quads) {
  if (*a.status != 0) return;
  const size_t rows = (size_t)a.T * a.G, total = rows * 2 * padded;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (size_t)gridDim.x * 256) {
    const size_t row = i / (2 * padded);
    const int e = (int)(i & (2 * padded - 1)), n = e & (padded - 1);
    if (n >= a.S) continue;
    float s = 0.f;
    for (uint32_t q = 0; q < quads; ++q) s += a.dbc[q * total + i];
    static_cast<T *>(e < padded ? a.dB : a.dC)[row * a.S + n] = Elt<T>::from_f32(s);
  }
}

// dA, dskip and dbias from the chunks' sums: 16 waves take a share of the chunks each.
__global__ __launch_bounds__(1024) void ssm_sum_weights_kernel(SsmArgs a, int padded) {
  __shared__ float part[16][64];
  const int j = blockIdx.y < (unsigned)a.S ? blockIdx.y : padded + (blockIdx.y - a.S), wave = threadIdx.x >> 6;
  const uint32_t c = blockIdx.x * 64 + lane_id();
  const int share = (a.chunks + 15) / 16, lo = wave * share, hi = min(lo + share, a.chunks);
  const float *p = a.dweights + (size_t)j * a.D + min(c, (uint32_t)a.D - 1);
  const size_t step = (size_t)(padded + 2) * a.D;
  float sum = 0.f;
#pragma unroll 8
  for (int i = lo; i < hi; ++i) sum += p[i * step];
  part[wave][lane_id()] = sum;
  __syncthreads();
  if (wave != 0 || c >= (uint32_t)a.D) return;
  sum = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) sum += part[i][lane_id()];
  if (j < a.S) a.dA[(size_t)c * a.S + j] = sum;
  else if (j == padded && a.dskip) a.dskip[c] = sum;
  else if (j == padded + 1 && a.dbias) a.dbias[c] = sum;
}

hipError_t launch_ssm_backward(const SsmArgs &a, bool bf16, bool dt_bf16, hipStream_t s) {
  hipError_t e = launch_ssm_setup(a, bf16, s);
  if (e != hipSuccess) return e;
  return ssm_dispatch(a.S, bf16, dt_bf16, [&](auto t, auto st, auto np) {
    using T = decltype(t);
    using S = decltype(st);
    constexpr int NP = decltype(np)::value;
    using F = BackForm<NP>;
    const uint32_t cols = (uint32_t)ssm_columns(a.D, a.G) * a.G;
    const uint32_t quads = (uint32_t)ssm_quads(a.D, a.G, a.S);
    const long all = (long)a.chunks * cols;
    if (all > 0x3fffffffl) return hipErrorInvalidValue;
    hipError_t e = hipSuccess;
    if (a.chunks > 1) {
      const uint32_t items = (uint32_t)(all - cols);
      hipLaunchKernelGGL((ssm_back_local_kernel<T, S, NP>), dim3((items + 3) / 4), dim3(256), 0, s, a, cols, items);
      e = hipGetLastError();
      if (e == hipSuccess) e = launch_ssm_carry(a, true, s);
      if (e != hipSuccess) return e;
    }
    const void *kernel = reinterpret_cast<const void *>(&ssm_backward_kernel<T, S, NP>);
    e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)F::kLds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((ssm_backward_kernel<T, S, NP>), dim3((unsigned)((long)a.chunks * quads * a.G)), dim3(F::kWaves * 64),
                       F::kLds, s, a, quads);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    const size_t blocks = ((size_t)a.T * a.G * 2 * NP + 255) / 256;
    hipLaunchKernelGGL((ssm_sum_bc_kernel<T>), dim3((unsigned)(blocks < 1 ? 1 : blocks < 16384 ? blocks : 16384)), dim3(256), 0, s,
                       a, NP, quads);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(ssm_sum_weights_kernel, dim3(((unsigned)a.D + 63) / 64, (unsigned)a.S + 2), dim3(1024), 0, s, a, NP);
    return hipGetLastError();
  });
}

}  // namespace hagdn

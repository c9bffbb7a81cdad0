// k11_ssm_backward.hip -- the selective scan's backward pass (ssm.h has the scheme).  With
// dy the gradient of the ungated output and e the gradient that reaches a state from later
// tokens,
//   dh_t = e_t + C_t dy_t,  e_{t-1} = a_t dh_t,
//   dC_t = sum_d dy_t h_t,  dB_t = sum_d dh_t dt_t x_t,  w_t = sum_n dh_t B_t,
//   dx_t = dt_t w_t + skip dy_t,  d(dt_t) = x_t w_t + sum_n A dh_t a_t h_{t-1},
//   dA = sum_t dt_t dh_t a_t h_{t-1}.
//
// Bound by its arithmetic, as the forward pass: some 28 instructions per token, channel and
// state in the main kernel, of which 4.4 are the sums of dB and dC over lanes and 8 form the
// states again.  17401 x 2048 x 16 in bf16, packed from eight sequences: what chunks pass back
// 144 us, what reaches them 8, the main kernel 645 to 666, sums 16.  The vector units are busy 3/4 of
// the time: two waves a SIMD, 232 registers each.  On the way: states formed again over 64
// tokens from scalar rows 1665 us; through LDS, 8 states at a time 1020; chunks that fill every
// CU alike 760; states saved every 16 tokens instead of 32 720 (every 8: 660, for twice the
// memory); sums written by all lanes that have them 690.  Three waves a SIMD with 4 states at a
// time spill (808); a branch-free copy for whole runs spills too (871); sums over lanes
// through LDS 680 to 720; decays kept instead of formed again 685.
#include "ssm.h"

namespace hagdn {

constexpr int kBackRows = 8;

// What a chunk passes back of a zero gradient.
template <typename T, typename S, int NP, int W>
__global__ __launch_bounds__(W * 64, NP == 16 ? 4 : NP == 32 ? 2 : 1) void ssm_back_local_kernel(SsmArgs a, uint32_t teams) {
  using Stage = Maps<T, NP, 2, kBackRows, W * 64>;
  __shared__ __align__(16) float sMaps[2][Stage::kAll];
  __shared__ int32_t sCu[kCheckInPlace + 1];
  Offsets32 cu;
  const bool ok = stage_offsets(a.cu, a.N, a.T, a.status, sCu, cu);
  const uint32_t team = blockIdx.x % (teams * a.G), group = team / teams;
  const int chunk = 1 + (int)(blockIdx.x / (teams * a.G));  // the first chunk passes nothing on
  const Column col(group, (team - group * teams) * W + uniform(threadIdx.x >> 6), a);
  const uint32_t c = col.c;
  if (!ok) return;
  const int t0 = chunk * a.chunk;
  int t1 = (int)min((long)t0 + a.chunk, (long)a.T);
  {  // what a chunk passes back is its first sequence's
    const Cursor first(cu, t0);
    if (first.end < t1) t1 = min(t1, t0 + (first.end - t0 + kBackRows - 1) / kBackRows * kBackRows);
  }
  float A[NP], e[NP];
  load_rates(a, c, A);
#pragma unroll
  for (int n = 0; n < NP; ++n) e[n] = 0.f;
  const float bias = a.raw && a.bias ? a.bias[c] : 0.f;
  Cursor q(cu, t1 - 1);
  bool reset = false;
  float sum = 0.f;
  int base = t0 + (t1 - 1 - t0) / kBackRows * kBackRows, turn = 0;
  Stage stage;
  stage.fetch(a, group, base, t1);
  for (; base >= t0; base -= kBackRows, turn ^= 1) {
    const int count = min(kBackRows, t1 - base);
    LdsRows rows(sMaps[0], turn * Stage::kAll);
    T dy[kBackRows], z[kBackRows];
    S dt[kBackRows];
    load_tokens(a.dy, a.dys, base, t1, c, dy);
    load_tokens(a.dt, a.dts, base, t1, c, dt);
    if (a.z) load_tokens(a.z, a.zs, base, t1, c, z);
    stage.put(sMaps[turn]);
    __syncthreads();
    if (base > t0) stage.fetch(a, group, base - kBackRows, t1);
    if (col.idle) continue;
    float given[kBackRows], step[kBackRows], d[kBackRows];
    step_sizes(a, dt, bias, given, step);
#pragma unroll
    for (int i = 0; i < kBackRows; ++i) d[i] = Elt<T>::to_f32(dy[i]);
    if (a.z) {
#pragma unroll
      for (int i = 0; i < kBackRows; ++i) d[i] *= silu(Elt<T>::to_f32(z[i]));
    }
    for (int hi = count; hi > 0;) {  // from one sequence's last token back to its first
      if (base + hi == q.start) q.previous();
      if (base + hi == q.end) {
        load_sequence<NP>(a.dfinal, q.seq, a, c, e);
        reset = true;
      }
      const int lo = max(0, q.start - base);
#pragma unroll
      for (int i = kBackRows - 1; i >= 0; --i)
        if (i >= lo && i < hi) {
          rows.hold();
          HAGDN_OPAQUE_VECTOR(step[i]);
          sum += step[i];
#pragma unroll
          for (int n = 0; n < NP; n += 4) {
            const f32x4 C = rows.four(i * Stage::kRow + n);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              float &v = e[n + k];
              v = __builtin_amdgcn_exp2f(step[i] * A[n + k]) * __builtin_fmaf(C[k], d[i], v);
            }
          }
        }
      hi = lo;
    }
  }
  store_states(a.maps + (size_t)chunk * NP * a.D, a, col, e);
  if (col.mine) a.sums[(size_t)chunk * a.D + c] = sum;
  if (team == 0 && threadIdx.x == 0) a.resets[chunk] = reset;
}

// Sums of 16 values over the wave's 64 lanes: value n to lanes 4 n to 4 n + 3.  Each exchange
// halves the values that a lane still holds: 35 instructions instead of the 96 of separate sums.
template <int CTRL> __device__ __forceinline__ float dpp(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float sum_lanes(float (&v)[16]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {  // halves of 32 lanes
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[i]), __float_as_uint(v[i + 8]), false, false);
    v[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {  // rows of 16
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[i]), __float_as_uint(v[i + 4]), false, false);
    v[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  const bool high8 = lane_id() & 8, high4 = lane_id() & 4;
#pragma unroll
  for (int i = 0; i < 2; ++i) v[i] = (high8 ? v[i + 2] : v[i]) + dpp<0x128>(high8 ? v[i] : v[i + 2]);  // lane + 8 of 16
  float s = (high4 ? v[1] : v[0]) + dpp<0x141>(high4 ? v[0] : v[1]);                                   // lane 7 - i of 8
  s += dpp<0xb1>(s);        // lane ^ 1
  return s + dpp<0x4e>(s);  // lane ^ 2
}

// The LDS of NP padded states and W waves: the states at the starts of a group's runs of 8
// tokens, the group's B and C, and a run's sums of dB and dC for each wave.
//
// Up to 32 states are gone over together, in code of up to 65 KB.  With 64 it would be 86 KB, more
// than the instruction cache holds, and every run would fetch it anew (17401 x 2048 x 64: 6960 us):
// there a loop takes blocks of 16, whose rates, gradients and sums are loaded and stored for each
// run (3440 us).  The gradients that go on to earlier tokens lie in the place of the first run's
// states, which the saved ones are; the sums of dA in their workspace.  With 32 states blocks of
// 16 are slower (1470 us against 1330).
template <int NP, int W> struct BackForm {
  static constexpr int kRuns = kSsmGroup / kBackRows;
  static constexpr int kBlock = NP < 64 ? NP : 16;
  static constexpr bool kWhole = kBlock == NP;
  static constexpr size_t kStates = (size_t)W * kRuns * NP * 64, kSums = (size_t)W * kBackRows * 2 * NP;
  static constexpr size_t kMaps = (size_t)kSsmGroup * 2 * NP;
  static constexpr size_t kLds = (kStates + kSums + kMaps) * sizeof(float);
};
constexpr int kSlice = 8;  // states whose run of 8 tokens is held in registers at once

// A group of 16 tokens at a time, the last first: its states at every eighth token are formed
// from the saved ones; then a run of 8 tokens at a time, the last first, and of 8 states of
// it, goes forward again, its a_t h_{t-1} kept in registers, and back.
template <typename T, typename S, int NP, int W>
__global__ __launch_bounds__(W * 64, NP <= 32 ? 2 : 1) void ssm_backward_kernel(SsmArgs a, uint32_t teams) {
  using F = BackForm<NP, W>;
  using Stage = Maps<T, NP, 3, kSsmGroup, W * 64>;
  extern __shared__ __align__(16) float lds[];
  const int wave = uniform(threadIdx.x >> 6), lane = lane_id();
  float *starts = lds + (size_t)wave * F::kRuns * NP * 64 + lane;  // [runs][NP][64]
  float *sums = lds + F::kStates;                                   // [waves][8][2 NP]
  float *maps = sums + F::kSums;                                    // [group][2 NP]
  constexpr int kEach = 64 / (2 * kSlice);                          // lanes that get one of sum_lanes' sums
  float *my_sums = sums + wave * kBackRows * 2 * NP + lane / kEach % kSlice + (lane >= 32 ? NP : 0);
  __shared__ int32_t sCu[kCheckInPlace + 1];
  Offsets32 cu;
  const bool ok = stage_offsets(a.cu, a.N, a.T, a.status, sCu, cu);
  const uint32_t team = blockIdx.x % (teams * a.G), group = team / teams, in_group = team - group * teams;
  const int chunk = (int)(blockIdx.x / (teams * a.G));
  const Column col(group, in_group * W + wave, a);
  const uint32_t c = col.c;
  if (chunk == 0) pass_states(a, ok, a.dfinal, a.ds0, col);
  const int t0 = chunk * a.chunk, t1 = ok ? (int)min((long)t0 + a.chunk, (long)a.T) : t0;

  constexpr int NB = F::kBlock;
  const int blocks_end = F::kWhole ? NP : states(a);
  float A[NB], e[NB], dA[NB], dskip = 0.f, dbias = 0.f;
  float *passed = starts;
  const auto weights = [&] { return a.dweights + (size_t)chunk * (NP + 2) * a.D; };
  bool fresh = true;  // no run has been gone over
  if (F::kWhole) load_rates(a, c, A);
#pragma unroll
  for (int n = 0; n < NB; ++n) e[n] = dA[n] = 0.f;
  const bool later = ok && chunk + 1 < a.chunks;
  if (F::kWhole && later) load_states(a.maps + (size_t)chunk * NP * a.D, a, c, e);
  for (int b = 0; b < blocks_end && !F::kWhole; b += NB) {
    if (later) load_states(a.maps + (size_t)chunk * NP * a.D, a, c, e, b);
#pragma unroll
    for (int n = 0; n < NB; ++n) passed[(b + n) * 64] = e[n];
  }
  const float bias = a.raw && a.bias ? a.bias[c] : 0.f, skip = a.skip ? a.skip[c] : 0.f;

  // waves of the workgroup that have channels
  const int working = min(W, (int)(((uint32_t)a.D / a.G + 63) / 64 - in_group * W));
  Stage stage;
  for (int g0 = t0 + (t1 - 1 - t0) / kSsmGroup * kSsmGroup; t1 > t0 && g0 >= t0; g0 -= kSsmGroup) {
    const int g1 = min(g0 + kSsmGroup, t1), runs = (g1 - g0 + kBackRows - 1) / kBackRows;
    stage.fetch(a, group, g0, g1);
    const auto saved = [&] { return a.ckpt + (size_t)(g0 / kSsmGroup) * NP * a.D; };
    {
      float h[NB];
      load_states(saved(), a, c, h);
      static_assert(F::kRuns == 2, "the second run's start is formed, the first one's saved");
      stage.put(maps);  // the last group's have been read: its runs end at a barrier
      __syncthreads();
      T x[kBackRows];
      S dt[kBackRows];
      float given[kBackRows], step[kBackRows];
      for (int b = 0; b < blocks_end; b += NB) {
        if (!F::kWhole) load_rates(a, c, A, b);
        if (b) load_states(saved(), a, c, h, b);
        Cursor q(cu, g0);
        int first = q.start == g0 ? g0 : q.end;
        for (int run = 0; run < runs && !col.idle; ++run) {
#pragma unroll
          for (int n = 0; n < NB; ++n)
            if (F::kWhole || run) starts[(run * NP + b + n) * 64] = h[n];
          if (run + 1 == runs) break;
          const int base = g0 + run * kBackRows;
          if (F::kWhole || !b) {  // the first run, for all blocks
            load_tokens(a.x, a.xs, base, t1, c, x);
            load_tokens(a.dt, a.dts, base, t1, c, dt);
            step_sizes(a, dt, bias, given, step);
          }
          LdsRows rows(maps, run * kBackRows * 2 * NP + b);
          for (int lo = 0; lo < kBackRows;) {
            if (base + lo == first) {
              if (first == q.end) q.next();
              load_sequence<NB>(a.s0, q.seq, a, c, h, b);
              first = q.end;
            }
            const int hi = min(kBackRows, first - base);
#pragma unroll
            for (int i = 0; i < kBackRows; ++i)
              if (i >= lo && i < hi) {
                rows.hold();
                HAGDN_OPAQUE_VECTOR(step[i]);
                const float in = step[i] * Elt<T>::to_f32(x[i]);
#pragma unroll
                for (int n = 0; n < NB; n += 4) {
                  const f32x4 B = rows.four(i * 2 * NP + n);
#pragma unroll
                  for (int k = 0; k < 4; ++k)
                    h[n + k] = __builtin_fmaf(in, B[k], __builtin_amdgcn_exp2f(step[i] * A[n + k]) * h[n + k]);
                }
              }
            lo = hi;
          }
        }
      }
    }
    for (int run = runs - 1; run >= 0; --run) {
      const int base = g0 + run * kBackRows, count = min(kBackRows, g1 - base);
      if (!col.idle) {
        LdsRows rows(maps, run * kBackRows * 2 * NP);
        float x[kBackRows], given[kBackRows], step[kBackRows], d[kBackRows], dgate[kBackRows];
        {
          T xs[kBackRows], dys[kBackRows], zs[kBackRows];
          S dts[kBackRows];
          load_tokens(a.x, a.xs, base, g1, c, xs);
          load_tokens(a.dt, a.dts, base, g1, c, dts);
          load_tokens(a.dy, a.dys, base, g1, c, dys);
          if (a.z) load_tokens(a.z, a.zs, base, g1, c, zs);
          step_sizes(a, dts, bias, given, step);
#pragma unroll
          for (int i = 0; i < kBackRows; ++i) {
            x[i] = Elt<T>::to_f32(xs[i]);
            d[i] = col.mine ? Elt<T>::to_f32(dys[i]) : 0.f;
          }
          if (a.z) {  // the gradient of the ungated output, and of z but for that output
#pragma unroll
            for (int i = 0; i < kBackRows; ++i) {
              const float z = Elt<T>::to_f32(zs[i]);
              const float s = logistic(z);
              dgate[i] = d[i] * silu_slope(z, s);
              d[i] *= z * s;
            }
          }
        }
        float y[kBackRows], w[kBackRows], ds[kBackRows];
#pragma unroll
        for (int i = 0; i < kBackRows; ++i) {
          y[i] = skip * x[i];
          w[i] = ds[i] = 0.f;
        }
        const Cursor at(cu, base);
        for (int b = 0; b < blocks_end; b += NB) {
          if (!F::kWhole) rows = LdsRows(maps, run * kBackRows * 2 * NP + b);
          float first_run[NB];
          if (!F::kWhole) {
            load_rates(a, c, A, b);
            if (!run) load_states(saved(), a, c, first_run, b);
            if (!fresh) load_states(weights(), a, c, dA, b);
#pragma unroll
            for (int n = 0; n < NB; ++n) {
              e[n] = passed[(b + n) * 64];
              if (fresh) dA[n] = 0.f;
            }
          }
#pragma unroll
          for (int n0 = 0; n0 < NB; n0 += kSlice) {
            float kept[kBackRows][kSlice], h[kSlice];  // kept: a_t h_{t-1}
#pragma unroll
            for (int k = 0; k < kSlice; ++k) h[k] = F::kWhole || run ? starts[(run * NP + b + n0 + k) * 64] : first_run[n0 + k];
            Cursor q = at;
            int first = q.start == base ? base : q.end;
            for (int lo = 0; lo < count;) {
              if (base + lo == first) {
                if (first == q.end) q.next();
                load_sequence<kSlice>(a.s0, q.seq, a, c, h, b + n0);
                first = q.end;
              }
              const int hi = min(count, first - base);
#pragma unroll
              for (int i = 0; i < kBackRows; ++i)
                if (i >= lo && i < hi) {
                  rows.hold();
                  HAGDN_OPAQUE_VECTOR(step[i]);
                  const float in = step[i] * x[i];
#pragma unroll
                  for (int n = 0; n < kSlice; n += 4) {
                    const f32x4 B = rows.four(i * 2 * NP + n0 + n);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                      kept[i][n + k] = __builtin_amdgcn_exp2f(step[i] * A[n0 + n + k]) * h[n + k];
                      h[n + k] = __builtin_fmaf(in, B[k], kept[i][n + k]);
                    }
                  }
                }
              lo = hi;
            }
            const auto back = [&](int i) {
              rows.hold();
              HAGDN_OPAQUE_VECTOR(step[i]);
              const float in = step[i] * x[i], fed = col.mine ? in : 0.f;
              float terms[2 * kSlice];  // of dB and dC
#pragma unroll
              for (int m = 0; m < kSlice; m += 4) {
                const f32x4 B = rows.four(i * 2 * NP + n0 + m), C = rows.four(i * 2 * NP + NP + n0 + m);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  const int k = m + j, n = n0 + k;
                  const float hn = __builtin_fmaf(in, B[j], kept[i][k]), dh = __builtin_fmaf(C[j], d[i], e[n]);
                  y[i] = __builtin_fmaf(C[j], hn, y[i]);
                  w[i] = __builtin_fmaf(B[j], dh, w[i]);
                  terms[k] = dh * fed;
                  terms[kSlice + k] = d[i] * hn;
                  const float p = dh * kept[i][k];
                  ds[i] = __builtin_fmaf(A[n], p, ds[i]);
                  dA[n] = __builtin_fmaf(step[i], p, dA[n]);
                  e[n] = __builtin_amdgcn_exp2f(step[i] * A[n]) * dh;
                }
              }
              my_sums[i * 2 * NP + b + n0] = sum_lanes(terms);  // (by all lanes that have the same one)
            };
            for (int hi = count; hi > 0;) {
              if (base + hi == q.start) q.previous();
              if (base + hi == q.end) load_sequence<kSlice>(a.dfinal, q.seq, a, c, e + n0, b + n0);
              const int lo = max(0, q.start - base);
#pragma unroll
              for (int i = kBackRows - 1; i >= 0; --i)
                if (i >= lo && i < hi) back(i);
              if (base + lo == q.start) store_sequence<kSlice>(a.ds0, q.seq, a, col, e + n0, b + n0);
              hi = lo;
            }
          }
          if (!F::kWhole) {
            store_states(weights(), a, col, dA, b);
#pragma unroll
            for (int n = 0; n < NB; ++n) passed[(b + n) * 64] = e[n];
          }
        }
        fresh = false;
        float dx[kBackRows], dv[kBackRows];
#pragma unroll
        for (int i = 0; i < kBackRows; ++i) {
          dx[i] = __builtin_fmaf(skip, d[i], step[i] * w[i]);
          dv[i] = __builtin_fmaf(ds[i], 1.f / kLog2e, x[i] * w[i]);
          dgate[i] *= y[i];
        }
        if (a.raw) {
#pragma unroll
          for (int i = 0; i < kBackRows; ++i) dv[i] *= logistic(given[i]);
        }
#pragma unroll
        for (int i = 0; i < kBackRows; ++i)
          if (i < count) {
            dskip = __builtin_fmaf(d[i], x[i], dskip);
            dbias += dv[i];
          }
        store_tokens<T>(a.dx, a, col, base, count, dx);
        store_tokens<S>(a.ddt, a, col, base, count, dv);
        if (a.z) store_tokens<T>(a.dz, a, col, base, count, dgate);
      }
      __syncthreads();
      for (int i = threadIdx.x; i < count * 2 * NP; i += W * 64) {
        float s = 0.f;
        for (int v = 0; v < working; ++v) s += sums[v * kBackRows * 2 * NP + i];
        const size_t t = base + i / (2 * NP);
        a.dbc[(((size_t)in_group * a.T + t) * a.G + group) * (2 * NP) + i % (2 * NP)] = s;
      }
      __syncthreads();
    }
  }
  if (!col.mine) return;
  for (int b = 0; b < blocks_end && (F::kWhole || fresh); b += NB) store_states(weights(), a, col, dA, b);
  weights()[(size_t)NP * a.D + c] = dskip;
  weights()[(size_t)(NP + 1) * a.D + c] = dbias;
}

// dB and dC from the teams' sums, in their order.
template <typename T> __global__ __launch_bounds__(256) void ssm_sum_bc_kernel(SsmArgs a, int padded, uint32_t teams) {
  if (*a.status != 0) return;
  const size_t rows = (size_t)a.T * a.G, total = rows * 2 * padded;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (size_t)gridDim.x * 256) {
    const size_t row = i / (2 * padded);
    const int e = (int)(i & (2 * padded - 1)), n = e & (padded - 1);
    if (n >= a.S) continue;
    float s = 0.f;
    for (uint32_t q = 0; q < teams; ++q) s += a.dbc[q * total + i];
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
  return ssm_dispatch(a, bf16, dt_bf16, [&](auto t, auto st, auto np, auto w) {
    using T = decltype(t);
    using S = decltype(st);
    constexpr int NP = decltype(np)::value, W = decltype(w)::value;
    using F = BackForm<NP, W>;
    const uint32_t teams = (uint32_t)ssm_teams(a.D, a.G);
    const long each = (long)teams * a.G, all = a.chunks * each;
    if (all > 0x7fffffffl) return hipErrorInvalidValue;
    hipError_t e = a.N > kCheckInPlace ? launch_check_offsets(a.cu, a.N, a.T, a.status, s) : hipSuccess;
    if (e != hipSuccess) return e;
    if (a.chunks > 1) {
      hipLaunchKernelGGL((ssm_back_local_kernel<T, S, NP, W>), dim3((unsigned)(all - each)), dim3(W * 64), 0, s, a, teams);
      e = hipGetLastError();
      if (e == hipSuccess) e = launch_ssm_carry(a, true, s);
      if (e != hipSuccess) return e;
    }
    if (F::kLds > 48 * 1024) {
      const void *kernel = reinterpret_cast<const void *>(&ssm_backward_kernel<T, S, NP, W>);
      e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)F::kLds);
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((ssm_backward_kernel<T, S, NP, W>), dim3((unsigned)all), dim3(W * 64), F::kLds, s, a, teams);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    const size_t blocks = ((size_t)a.T * a.G * 2 * NP + 255) / 256;
    hipLaunchKernelGGL((ssm_sum_bc_kernel<T>), dim3((unsigned)(blocks < 1 ? 1 : blocks < 16384 ? blocks : 16384)), dim3(256), 0, s,
                       a, NP, teams);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(ssm_sum_weights_kernel, dim3(((unsigned)a.D + 63) / 64, (unsigned)a.S + 2), dim3(1024), 0, s, a, NP);
    return hipGetLastError();
  });
}

}  // namespace hagdn

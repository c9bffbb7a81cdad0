// k9_conv.hip -- the short causal convolution over packed sequences, per channel
//   p_t = b + sum_j w_j x_{t-W+1+j},  y_t = p_t or p_t / (1 + e^-p_t),
// with a window of the W - 1 inputs before each sequence, its backward pass and its step
// for single tokens.
//
// A lane has four neighbouring channels (8 bytes of bf16) and goes over a run of tokens with
// the last W inputs in registers, so that every input is read once but for the W - 1 before
// each run.  Bound by HBM: 34800 x 2048 in bf16, four taps, packed from eight sequences,
// forward 60 us (285 MB, 4.8 TB/s; a copy of 1 GiB 5.2), backward 101 (428 MB, 4.2 TB/s, and
// some 28 operations an element, half its time) with 5 us of sums.  Runs of up to 64 tokens
// forward; backward as many as give every SIMD four waves, since each leaves partial sums of
// the weights' gradients.  Narrow calls, below 256 channels, have a channel a lane.
#include "mixer_dev.h"

namespace hagdn {

__global__ __launch_bounds__(256) void check_kernel(const int32_t *cu, int N, int T, int *status) {
  int bad = 0;
  for (int i = threadIdx.x; i < N; i += 256) bad |= cu[i] > cu[i + 1];
  if (threadIdx.x == 0) bad |= cu[0] != 0 || cu[N] != T;
  bad = __syncthreads_or(bad);
  if (threadIdx.x == 0) *status = bad ? kDevBadSeqlens : 0;
}
hipError_t launch_check_offsets(const int32_t *cu, int N, int T, int *status, hipStream_t s) {
  hipLaunchKernelGGL(check_kernel, dim3(1), dim3(256), 0, s, cu, N, T, status);
  return hipGetLastError();
}

// The channels of a lane: V from c on.  Lanes past the last channel, and the last one where
// D is no multiple of V, step back to the row's end; those past it store nothing.
template <int V> struct Channels {
  uint32_t c;
  bool mine;
  __device__ Channels(uint32_t col, int D) {
    const uint32_t at = (col * 64 + lane_id()) * V;
    mine = at < (uint32_t)D;
    c = min(at, (uint32_t)(D - V));
  }
};

template <typename T, int W, int V> struct Taps {
  float w[W][V], b[V];
  __device__ Taps(const float *pw, const float *pb, uint32_t c) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
#pragma unroll
      for (int j = 0; j < W; ++j) w[j][v] = pw[(size_t)(c + v) * W + j];
      b[v] = pb ? pb[c + v] : 0.f;
    }
  }
};

// The W - 1 inputs before token t of a sequence that starts at `start`: its window's rows,
// then its own.
template <typename T, int W, int V>
__device__ __forceinline__ void load_history(const ConvArgs &a, int seq, int start, int t, uint32_t c, float (&h)[W][V]) {
#pragma unroll
  for (int j = 0; j < W - 1; ++j) {
    const int p = t - (W - 1) + j;
    if (p >= start) {
      const auto r = load_pack<T, V>(a.x, (size_t)p * a.xs + c);
#pragma unroll
      for (int v = 0; v < V; ++v) h[j + 1][v] = Elt<T>::to_f32(r.v[v]);
    } else if (a.w0) {
      const auto r = load_pack<T, V>(a.w0, ((size_t)seq * (W - 1) + (W - 1 + p - start)) * a.D + c);
#pragma unroll
      for (int v = 0; v < V; ++v) h[j + 1][v] = Elt<T>::to_f32(r.v[v]);
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) h[j + 1][v] = 0.f;
    }
  }
}

// A row joins the W newest inputs, h[W - 1] the newest.
template <typename T, int W, int V> __device__ __forceinline__ void push(float (&h)[W][V], const Pack<T, V> &row) {
#pragma unroll
  for (int v = 0; v < V; ++v) {
#pragma unroll
    for (int j = 0; j + 1 < W; ++j) h[j][v] = h[j + 1][v];
    h[W - 1][v] = Elt<T>::to_f32(row.v[v]);
  }
}

// Windows of the sequences without tokens pass through.
template <typename T, int W, int V>
__device__ __forceinline__ void pass_windows(const ConvArgs &a, bool ok, const void *in, void *out, const Channels<V> &ch) {
  if (!out) return;
  for_empty(a.cu, a.N, a.T, ok, [&](int n) {
    if (!ch.mine) return;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      const size_t at = ((size_t)n * (W - 1) + j) * a.D + ch.c;
      Pack<T, V> r = {};
      if (in) r = load_pack<T, V>(in, at);
      store_pack<T, V>(out, at, r);
    }
  });
}

constexpr int kConvRows = 8;      // rows on their way at once
constexpr int kConvBackRows = 4;  // and the next four

template <typename T, int W, int V>
__global__ __launch_bounds__(256) void conv_forward_kernel(ConvArgs a, uint32_t cols, uint32_t items) {
  __shared__ int32_t sCu[kCheckInPlace + 1];
  Offsets32 cu;
  const bool ok = stage_offsets(a.cu, a.N, a.T, a.status, sCu, cu);
  const uint32_t item = uniform(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (item >= items) return;
  const uint32_t run = item / cols;
  const Channels<V> ch(item - run * cols, a.D);
  if (run == 0) pass_windows<T, W, V>(a, ok, a.w0, a.w_final, ch);
  const int t0 = (int)min((long)run * a.run, (long)a.T), t1 = (int)min((long)t0 + a.run, (long)a.T);
  if (!ok || t0 >= t1) return;
  const Taps<T, W, V> k(a.w, a.b, ch.c);
  Cursor q(cu, t0);
  float h[W][V];
  load_history<T, W, V>(a, q.seq, q.start, t0, ch.c, h);
  for (int base = t0; base < t1; base += kConvRows) {
    Pack<T, V> rows[kConvRows];
#pragma unroll
    for (int i = 0; i < kConvRows; ++i) rows[i] = load_pack<T, V>(a.x, (size_t)min(base + i, t1 - 1) * a.xs + ch.c);
#pragma unroll
    for (int i = 0; i < kConvRows; ++i) {
      const int t = base + i;
      if (t >= t1) break;
      if (t == q.end) {
        q.next();
        load_history<T, W, V>(a, q.seq, q.start, t, ch.c, h);
      }
      push<T, W, V>(h, rows[i]);
      Pack<T, V> y;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float p = k.b[v];
#pragma unroll
        for (int j = 0; j < W; ++j) p = __builtin_fmaf(k.w[j][v], h[j][v], p);
        y.v[v] = Elt<T>::from_f32(a.silu ? silu(p) : p);
      }
      if (ch.mine) store_pack<T, V>(a.y, (size_t)t * a.D + ch.c, y);
      if (t + 1 == q.end && a.w_final && ch.mine) {
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
          Pack<T, V> r;
#pragma unroll
          for (int v = 0; v < V; ++v) r.v[v] = Elt<T>::from_f32(h[j + 1][v]);
          store_pack<T, V>(a.w_final, ((size_t)q.seq * (W - 1) + j) * a.D + ch.c, r);
        }
      }
    }
  }
}

// Backward.  A wave goes over its run and the W - 1 tokens after it, whose dp reaches back
// into the run.  The next four rows of x and dy are on their way while it works on four: 101 us
// for the case above, 107 with eight rows and none ahead, 109 to 124 with eight and eight ahead.  acc[j] gathers the gradient of the input at t - W + 1 + j, tap j of token
// t; the oldest is whole after token t.  An input before the sequence's start is a row of
// its window, written by the wave of the sequence's first token.
template <typename T, int W, int V>
__global__ __launch_bounds__(256) void conv_backward_kernel(ConvArgs a, uint32_t cols, uint32_t items) {
  __shared__ int32_t sCu[kCheckInPlace + 1];
  Offsets32 cu;
  const bool ok = stage_offsets(a.cu, a.N, a.T, a.status, sCu, cu);
  const uint32_t item = uniform(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (item >= items) return;
  const uint32_t run = item / cols;
  const Channels<V> ch(item - run * cols, a.D);
  if (run == 0) pass_windows<T, W, V>(a, ok, a.dfinal, a.dw0, ch);
  const int t0 = (int)min((long)run * a.run, (long)a.T), t1 = (int)min((long)t0 + a.run, (long)a.T);
  float dw[W][V] = {}, db[V] = {};
  if (ok && t0 < t1) {
    const int stop = (int)min((long)t1 + W - 1, (long)a.T);
    const Taps<T, W, V> k(a.w, a.b, ch.c);
    Cursor q(cu, t0);
    float h[W][V], acc[W][V] = {};
    load_history<T, W, V>(a, q.seq, q.start, t0, ch.c, h);
    const auto emit = [&](int pos, const float (&g)[V]) {
      Pack<T, V> r;
#pragma unroll
      for (int v = 0; v < V; ++v) r.v[v] = Elt<T>::from_f32(g[v]);
      if (!ch.mine) return;
      if (pos >= q.start) {
        if (pos >= t0 && pos < t1) store_pack<T, V>(a.dx, (size_t)pos * a.D + ch.c, r);
      } else if (a.dw0 && q.start >= t0 && q.start < t1) {
        store_pack<T, V>(a.dw0, ((size_t)q.seq * (W - 1) + (W - 1 + pos - q.start)) * a.D + ch.c, r);
      }
    };
    Pack<T, V> rows[kConvBackRows], grads[kConvBackRows], next_rows[kConvBackRows], next_grads[kConvBackRows];
    const auto fetch = [&](int base) {
#pragma unroll
      for (int i = 0; i < kConvBackRows; ++i) {
        const size_t t = min(base + i, stop - 1);
        next_rows[i] = load_pack<T, V>(a.x, t * a.xs + ch.c);
        next_grads[i] = load_pack<T, V>(a.dy, t * a.dys + ch.c);
      }
    };
    fetch(t0);
    for (int base = t0; base < stop; base += kConvBackRows) {
#pragma unroll
      for (int i = 0; i < kConvBackRows; ++i) {
        rows[i] = next_rows[i];
        grads[i] = next_grads[i];
      }
      fetch(base + kConvBackRows);
#pragma unroll
      for (int i = 0; i < kConvBackRows; ++i) {
        const int t = base + i;
        if (t >= stop || (t >= t1 && t == q.end)) {  // a sequence that starts after the run is none of its
          base = stop;
          break;
        }
        if (t == q.end) {
          q.next();
          load_history<T, W, V>(a, q.seq, q.start, t, ch.c, h);
#pragma unroll
          for (int j = 0; j < W; ++j)
#pragma unroll
            for (int v = 0; v < V; ++v) acc[j][v] = 0.f;
        }
        push<T, W, V>(h, rows[i]);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          float d = Elt<T>::to_f32(grads[i].v[v]);
          if (a.silu) {
            float p = k.b[v];
#pragma unroll
            for (int j = 0; j < W; ++j) p = __builtin_fmaf(k.w[j][v], h[j][v], p);
            d *= silu_slope(p, logistic(p));
          }
#pragma unroll
          for (int j = 0; j < W; ++j) acc[j][v] = __builtin_fmaf(k.w[j][v], d, j + 1 < W ? acc[j + 1][v] : 0.f);
          if (t < t1) {
#pragma unroll
            for (int j = 0; j < W; ++j) dw[j][v] = __builtin_fmaf(d, h[j][v], dw[j][v]);
            db[v] += d;
          }
        }
        emit(t - W + 1, acc[0]);
        if (t + 1 == q.end) {
#pragma unroll
          for (int j = 1; j < W; ++j) {
            if (a.dfinal) {
              const auto g = load_pack<T, V>(a.dfinal, ((size_t)q.seq * (W - 1) + j - 1) * a.D + ch.c);
#pragma unroll
              for (int v = 0; v < V; ++v) acc[j][v] += Elt<T>::to_f32(g.v[v]);
            }
            emit(t - W + 1 + j, acc[j]);
          }
        }
      }
    }
  }
  if (!ch.mine) return;
  float *out = a.partial + (size_t)run * (W + 1) * a.D + ch.c;
#pragma unroll
  for (int j = 0; j <= W; ++j) {
    Pack<float, V> r;
#pragma unroll
    for (int v = 0; v < V; ++v) r.v[v] = j < W ? dw[j < W ? j : 0][v] : db[v];
    store_pack<float, V>(out, (size_t)j * a.D, r);
  }
}

// The runs' sums, in their order: 16 waves take a share of the runs each.
__global__ __launch_bounds__(1024) void conv_sum_kernel(ConvArgs a) {
  __shared__ float part[16][64];
  const int j = blockIdx.y, wave = threadIdx.x >> 6;
  const uint32_t c = blockIdx.x * 64 + lane_id();
  const int share = (a.parts + 15) / 16, lo = wave * share, hi = min(lo + share, a.parts);
  const float *p = a.partial + (size_t)j * a.D + min(c, (uint32_t)a.D - 1);
  const size_t step = (size_t)(a.W + 1) * a.D;
  float sum = 0.f;
#pragma unroll 8
  for (int i = lo; i < hi; ++i) sum += p[i * step];
  part[wave][lane_id()] = sum;
  __syncthreads();
  if (wave != 0 || c >= (uint32_t)a.D) return;
  sum = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) sum += part[i][lane_id()];
  if (j < a.W) a.dw[(size_t)c * a.W + j] = sum;
  else if (a.db) a.db[c] = sum;
}

// ------------------------------------------------------------- single tokens
// Four channels of one sequence a lane (one, where D is no multiple of four): 256 sequences x
// 4096 channels 6.3 us (16.6 MB), few sequences the launch.
template <typename T, int W, int V> __global__ __launch_bounds__(256) void conv_step_kernel(ConvStepArgs a, uint32_t cols, uint32_t items) {
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < items; i += gridDim.x * 256) {
    const uint32_t n = i / cols, c = (i - n * cols) * V;
    const int slot = a.slots ? a.slots[n] : (int)n;
    Pack<T, V> y = {};
    if (slot >= 0 && slot < a.num_slots) {
      const auto x = load_pack<T, V>(a.x, (size_t)n * a.xs + c);
      const size_t at = (size_t)slot * (W - 1) * a.D + c;
      Pack<T, V> h[W];
#pragma unroll
      for (int j = 0; j < W - 1; ++j) h[j] = load_pack<T, V>(a.state, at + (size_t)j * a.D);
      h[W - 1] = x;
      const Taps<T, W, V> k(a.w, a.b, c);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float p = k.b[v];
#pragma unroll
        for (int j = 0; j < W; ++j) p = __builtin_fmaf(k.w[j][v], Elt<T>::to_f32(h[j].v[v]), p);
        y.v[v] = Elt<T>::from_f32(a.silu ? silu(p) : p);
      }
#pragma unroll
      for (int j = 0; j < W - 1; ++j) store_pack<T, V>(a.state, at + (size_t)j * a.D, h[j + 1]);
    }
    store_pack<T, V>(a.y, (size_t)n * a.D + c, y);
  }
}

// ----------------------------------------------------------------- launchers
// Calls f with the instance's element type, taps and channels a lane.
template <typename T, int W, typename F> hipError_t conv_width(int D, F f) {
  if (D >= 256) return f(T(), std::integral_constant<int, W>(), std::integral_constant<int, 4>());
  return f(T(), std::integral_constant<int, W>(), std::integral_constant<int, 1>());
}
template <typename T, typename F> hipError_t conv_taps(int W, int D, F f) {
  switch (W) {
    case 2: return conv_width<T, 2>(D, f);
    case 3: return conv_width<T, 3>(D, f);
    case 4: return conv_width<T, 4>(D, f);
    case 5: return conv_width<T, 5>(D, f);
    case 6: return conv_width<T, 6>(D, f);
    case 7: return conv_width<T, 7>(D, f);
    default: return conv_width<T, 8>(D, f);
  }
}
template <typename F> hipError_t conv_dispatch(bool bf16, int W, int D, F f) {
  return bf16 ? conv_taps<bf16_t>(W, D, f) : conv_taps<float>(W, D, f);
}
inline uint32_t conv_columns(int D, int V) { return ((uint32_t)D + 64 * V - 1) / (64 * V); }

hipError_t launch_conv_forward(const ConvArgs &args, bool bf16, hipStream_t s) {
  return conv_dispatch(bf16, args.W, args.D, [&](auto t, auto w, auto v) {
    using T = decltype(t);
    constexpr int W = decltype(w)::value, V = decltype(v)::value;
    ConvArgs a = args;
    const uint32_t cols = conv_columns(a.D, V);
    const long runs = a.T > 0 ? ((long)a.T - 1) / a.run + 1 : 1, items = runs * cols;
    if (items > 0x3fffffffl) return hipErrorInvalidValue;
    if (a.N > kCheckInPlace) {
      const hipError_t e = launch_check_offsets(a.cu, a.N, a.T, a.status, s);
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((conv_forward_kernel<T, W, V>), dim3((unsigned)((items + 3) / 4)), dim3(256), 0, s, a, cols, (uint32_t)items);
    return hipGetLastError();
  });
}

hipError_t launch_conv_backward(const ConvArgs &args, bool bf16, hipStream_t s) {
  return conv_dispatch(bf16, args.W, args.D, [&](auto t, auto w, auto v) {
    using T = decltype(t);
    constexpr int W = decltype(w)::value, V = decltype(v)::value;
    ConvArgs a = args;
    const uint32_t cols = conv_columns(a.D, V);
    const long items = (long)a.parts * cols;
    if (items > 0x3fffffffl) return hipErrorInvalidValue;
    if (a.N > kCheckInPlace) {
      const hipError_t e = launch_check_offsets(a.cu, a.N, a.T, a.status, s);
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((conv_backward_kernel<T, W, V>), dim3((unsigned)((items + 3) / 4)), dim3(256), 0, s, a, cols, (uint32_t)items);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(conv_sum_kernel, dim3(((unsigned)a.D + 63) / 64, (unsigned)W + 1), dim3(1024), 0, s, a);
    return hipGetLastError();
  });
}

hipError_t launch_conv_step(const ConvStepArgs &args, bool bf16, hipStream_t s) {
  // windows are updated in place, so that no two lanes may share a channel
  return conv_dispatch(bf16, args.W, args.D % 4 == 0 ? 256 : 1, [&](auto t, auto w, auto v) {
    using T = decltype(t);
    constexpr int W = decltype(w)::value, V = decltype(v)::value;
    const uint32_t cols = (uint32_t)args.D / V, items = cols * (uint32_t)args.N;
    const uint32_t blocks = (items + 255) / 256;
    hipLaunchKernelGGL((conv_step_kernel<T, W, V>), dim3(blocks < 1u << 20 ? blocks : 1u << 20), dim3(256), 0, s, args, cols, items);
    return hipGetLastError();
  });
}

}  // namespace hagdn

// k6_glr.hip -- the gated linear recurrence, forward: h_t = a_t h_{t-1} + w_t x_t per
// channel over packed sequences (a_t = e^g_t, w_t = 1 or 1 - a_t), and its step for
// single tokens.
//
// The forward pass is the scan of glr.h over tiles of 128 tokens x 64 V channels:
// eight waves of 16 tokens, a lane holding V channels of each.  It is bound by HBM:
// x and g are read once and h written once, for some 15 operations an element.
#include "glr.h"

namespace hagdn {

constexpr int kGlrWaves = 8;
constexpr int kGlrRun = kGlrTile / kGlrWaves;  // tokens of a wave
constexpr unsigned kGlrMaxGrid = 1 << 20;      // workgroups: a launch holds fewer than 2^32 threads

// Clears `words` words and the tile counter, checks the sequence offsets (workgroup 0)
// and writes the status.
__global__ __launch_bounds__(256) void glr_setup_kernel(GlrArgs a, size_t words) {
  typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));
  u64x2 *w = reinterpret_cast<u64x2 *>(a.words);
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < words / 2; i += (size_t)gridDim.x * 256) w[i] = u64x2{0, 0};
  if (blockIdx.x != 0) return;
  const bool ok = glr_seqlens_ok(a.cu, a.N, a.T);
  if (threadIdx.x == 0) {
    *a.counter = 0;
    *a.status = ok ? 0 : kDevBadSeqlens;
  }
}

// out[n] = in[n] (null: 0) for the sequences without tokens (all of them if !ok), for
// one workgroup's channels.
template <int V>
__device__ __forceinline__ void pass_empty(const int32_t *cu, int N, int T, bool ok, const float *in, float *out, int D, int c) {
  if (!out) return;
  const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6, lane = lane_id();
  for (long base = (long)wave * 64; base < N; base += waves * 64) {
    const long n = base + lane;
    const bool empty = n < N && (!ok || (cu ? cu[n] == cu[n + 1] : T == 0));
    for (uint64_t left = __ballot(empty); left; left &= left - 1) {
      const size_t at = (size_t)(base + __builtin_ctzll(left)) * D + c;
      if (c < D)
#pragma unroll
        for (int e = 0; e < V; ++e) out[at + e] = in ? in[at + e] : 0.f;
    }
  }
}

template <typename T, typename G, int V, bool RAW, bool CONVEX>
__global__ __launch_bounds__(kGlrWaves * 64, 4) void glr_forward_kernel(GlrArgs a, uint32_t tiles, uint32_t cols) {
  constexpr int L = kGlrRun, W = kGlrWaves;
  __shared__ float sA[W][V][64], sB[W][V][64], sIn[V][64];
  __shared__ int sIds[W][2 * L], sReset[W];
  __shared__ uint32_t sNext;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  bool ok = true;
  if (tiles > 1) {
    ok = *a.status == 0;
  } else {  // no setup kernel ran
    ok = glr_seqlens_ok(a.cu, a.N, a.T);
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = ok ? 0 : kDevBadSeqlens;
  }
  for (uint32_t turn = blockIdx.x;; turn += gridDim.x) {
    uint32_t item = turn;
    if (tiles > 1) {
      if (threadIdx.x == 0) sNext = atomicAdd(a.counter, 1u);
      __syncthreads();
      item = __builtin_amdgcn_readfirstlane(sNext);
    }
    if (item >= tiles * cols) return;
    const uint32_t tile = __builtin_amdgcn_readfirstlane(item / cols);
    const int c = (int)(item - tile * cols) * 64 * V + lane * V;
    const uint32_t cl = c < a.D ? c : 0;  // lanes past the last channel compute the first one's, and store nothing
    if (tile == 0) pass_empty<V>(a.cu, a.N, a.T, ok, a.s0, a.s_final, a.D, c);
    if (!ok || a.T == 0) {
      __syncthreads();  // sNext is written again in the next turn
      continue;
    }

    // the wave's tokens; rows past the end are loaded from the last one
    const long t0 = (long)tile * kGlrTile + wave * L;
    const int count = (int)min((long)L, max(0l, (long)a.T - t0));
    Elems<T, V> x[L];
    Elems<G, V> g[L];
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const long t = min(t0 + i, (long)a.T - 1);
      x[i] = load_elems<T, V>(static_cast<const T *>(a.x) + t * a.xs, cl);
      g[i] = load_elems<G, V>(static_cast<const G *>(a.g) + t * a.gs, cl);
    }
    const Marks<L> m = find_marks<L>(a.cu, a.N, a.T, t0, sIds[wave]);
    // The initial state of the last sequence that starts here, the only one that can
    // reach past the wave's tokens.  It is read before the tile's map is published, the
    // others' when their tokens' turn comes: where s_final is s0, a state is written by
    // this wave after that, or by one that waits for the map.
    const int start = m.first ? 31 - __builtin_clz(m.first) : -1;
    float s0[V] = {};
    if (m.first && a.s0) load_state<V>(a.s0 + (size_t)m.starts(start) * a.D, cl, s0);

    float k[L][V], b[L][V];  // h_t = k h_{t-1} + b
#pragma unroll
    for (int i = 0; i < L; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const Gate q = glr_gate<RAW>(Elt<G>::to_f32(g[i].v[e]));
        const float u = Elt<T>::to_f32(x[i].v[e]);
        k[i][e] = i < count ? q.a : 1.f;
        b[i][e] = i < count ? CONVEX ? q.forget * u : u : 0.f;
      }
    float A[V], B[V];
#pragma unroll
    for (int e = 0; e < V; ++e) A[e] = 1.f, B[e] = 0.f;
#pragma unroll
    for (int i = 0; i < L; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        A[e] *= k[i][e];
        B[e] = k[i][e] * (i == start ? s0[e] : B[e]) + b[i][e];
      }
#pragma unroll
    for (int e = 0; e < V; ++e) sA[wave][e][lane] = A[e], sB[wave][e][lane] = B[e];
    if (lane == 0) sReset[wave] = m.first != 0;
    __syncthreads();

    if (wave == 0) {
      bool reset = false;
#pragma unroll
      for (int e = 0; e < V; ++e) A[e] = 1.f, B[e] = 0.f;
#pragma unroll 1
      for (int w = 0; w < W; ++w) {
        const bool r = sReset[w];
        reset |= r;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          B[e] = r ? sB[w][e][lane] : sA[w][e][lane] * B[e] + sB[w][e][lane];
          A[e] *= sA[w][e][lane];
        }
      }
      const bool pass_on = tile + 1 < tiles && c < a.D;
      uint64_t *words = a.words + (size_t)tile * 2 * a.D;
      if (pass_on)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          if (!reset) publish(words, cl + e, A[e], kMap);
          publish(words + a.D, cl + e, B[e], reset ? kState : kMap);
        }
      float s[V];
#pragma unroll
      for (int e = 0; e < V; ++e) s[e] = 0.f;
      if (tile > 0 && !(m.first & 1)) look_back<V>(a.words, a.D, cl, (long)tile - 1, -1, tile, a.status, s);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        if (pass_on && !reset) publish(words + a.D, cl + e, A[e] * s[e] + B[e], kState);
        sIn[e][lane] = s[e];
      }
    }
    __syncthreads();

    float s[V];
#pragma unroll
    for (int e = 0; e < V; ++e) s[e] = sIn[e][lane];
#pragma unroll 1
    for (int w = 0; w < wave; ++w) {
      const bool r = sReset[w];
#pragma unroll
      for (int e = 0; e < V; ++e) s[e] = r ? sB[w][e][lane] : sA[w][e][lane] * s[e] + sB[w][e][lane];
    }
    const bool mine = c < a.D;
    if (a.ckpt && t0 % kGlrGroup == 0 && count > 0 && mine) store_elems<float, V>(a.ckpt + (size_t)(t0 / kGlrGroup) * a.D, cl, s);
    T *h = static_cast<T *>(a.h) + (size_t)t0 * a.D;
    // from one sequence's first token to the next one's; mostly a single turn
    for (int lo = 0; lo < count;) {
      if (m.first >> lo & 1) {
#pragma unroll
        for (int e = 0; e < V; ++e) s[e] = lo == start ? s0[e] : 0.f;
        if (lo != start && a.s0) load_state<V>(a.s0 + (size_t)m.starts(lo) * a.D, cl, s);
      }
      const uint32_t later = m.first & ~((2u << lo) - 1);
      const int hi = later ? __builtin_ctz(later) : count;
#pragma unroll
      for (int i = 0; i < L; ++i)
        if (i >= lo && i < hi) {
#pragma unroll
          for (int e = 0; e < V; ++e) s[e] = k[i][e] * s[e] + b[i][e];
          if (mine) store_elems<T, V>(h + (size_t)i * a.D, cl, s);
        }
      if ((m.last >> (hi - 1) & 1) && a.s_final && mine)
        store_elems<float, V>(a.s_final + (size_t)m.ends(hi - 1) * a.D, cl, s);
      lo = hi;
    }
    __syncthreads();  // LDS is used again in the next turn
  }
}

constexpr int kStepThreads = 64;

template <typename T, typename G, bool RAW, bool CONVEX>
__global__ __launch_bounds__(kStepThreads) void glr_step_kernel(GlrStepArgs a) {
  const int cols = (a.D + kStepThreads - 1) / kStepThreads;
  const int n = blockIdx.x / cols, c = blockIdx.x % cols * kStepThreads + threadIdx.x;
  if (c >= a.D) return;
  T *h = static_cast<T *>(a.h) + (size_t)n * a.D + c;
  const int slot = a.slots ? a.slots[n] : n;
  if (slot < 0 || slot >= a.num_slots) {  // padding entry
    *h = Elt<T>::from_f32(0.f);
    return;
  }
  float *s = a.state + (size_t)slot * a.D + c;
  const Gate k = glr_gate<RAW>(Elt<G>::to_f32(static_cast<const G *>(a.g)[(size_t)n * a.gs + c]));
  const float u = Elt<T>::to_f32(static_cast<const T *>(a.x)[(size_t)n * a.xs + c]);
  const float r = k.a * *s + (CONVEX ? k.forget * u : u);
  *s = r;
  *h = Elt<T>::from_f32(r);
}

hipError_t launch_glr_setup(const GlrArgs &a, size_t words, hipStream_t s) {
  const size_t blocks = (words / 2 + 256 * 4 - 1) / (256 * 4);
  hipLaunchKernelGGL(glr_setup_kernel, dim3((unsigned)(blocks < 1 ? 1 : blocks < 4096 ? blocks : 4096)), dim3(256), 0, s, a,
                     words);
  return hipGetLastError();
}

template <typename T, typename G, int V, bool RAW, bool CONVEX>
static hipError_t launch_forward(const GlrArgs &a, hipStream_t s) {
  const long tiles = a.T > 0 ? ((long)a.T + kGlrTile - 1) / kGlrTile : 1, cols = ((long)a.D + 64 * V - 1) / (64 * V);
  if (tiles * cols > 0xffff0000l) return hipErrorInvalidValue;  // the counter's range
  if (tiles > 1) {
    const hipError_t e = launch_glr_setup(a, (size_t)tiles * 2 * a.D, s);
    if (e != hipSuccess) return e;
  }
  const unsigned grid = (unsigned)(tiles * cols < kGlrMaxGrid ? tiles * cols : kGlrMaxGrid);
  hipLaunchKernelGGL((glr_forward_kernel<T, G, V, RAW, CONVEX>), dim3(grid), dim3(kGlrWaves * 64), 0, s, a,
                     (uint32_t)tiles, (uint32_t)cols);
  return hipGetLastError();
}

template <typename T, typename G> struct Forward {
  template <bool RAW, bool CONVEX> static hipError_t go(const GlrArgs &a, hipStream_t s) {
    return a.D % 2 == 0 ? launch_forward<T, G, 2, RAW, CONVEX>(a, s) : launch_forward<T, G, 1, RAW, CONVEX>(a, s);
  }
};
template <typename T, typename G> struct Step {
  template <bool RAW, bool CONVEX> static hipError_t go(const GlrStepArgs &a, hipStream_t s) {
    const dim3 grid((unsigned)((size_t)a.N * ((a.D + kStepThreads - 1) / kStepThreads)));
    hipLaunchKernelGGL((glr_step_kernel<T, G, RAW, CONVEX>), grid, dim3(kStepThreads), 0, s, a);
    return hipGetLastError();
  }
};

hipError_t launch_glr_forward(const GlrArgs &a, const GlrForm &f, hipStream_t s) { return glr_dispatch<Forward>(a, f, s); }
hipError_t launch_glr_step(const GlrStepArgs &a, const GlrForm &f, hipStream_t s) { return glr_dispatch<Step>(a, f, s); }

}  // namespace hagdn

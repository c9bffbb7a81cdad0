// k6_glr.hip -- the gated linear recurrence, forward: h_t = a_t h_{t-1} + w_t x_t per
// channel over packed sequences (a_t = e^g_t, w_t = 1 or 1 - a_t), and its step for
// single tokens.
//
// The forward pass is the scan of glr.h over tiles of 64 to 512 tokens x 64 channels (in
// long calls eight waves of 32 tokens, a lane to a channel, two workgroups a CU: what the
// registers hold).  It is bound by HBM: x and g are read once and h written once, for some
// 15 operations an element.  32768 tokens x 2048 channels, x in bf16 and g in fp32: 115 us,
// 4.7 TB/s of the 537 MB that must move (a copy of 1 GiB 4.9 to 5.3 TB/s), in convex form 121;
// the gate in bf16 103 to 105 us, 3.9 TB/s; 32768 x 2000, whose rows do not begin at memory
// lines, 163 us.  Of the forms of 32 tokens a wave, the raw convex ones and all bf16 ones but
// those convex alone spill 4 to 7 of their 128 registers.  What is left: a tile's loads, its
// wait for the state and its stores follow each other, and two workgroups overlap them in
// part (of 119 us, at the time, 115 without the wait and 100 without all but one in 32 of the
// stores).  Four or sixteen waves a workgroup took 135 and 126 us there.
#include "glr.h"

namespace hagdn {

// Empties `words` words and clears the columns' counters, checks the sequence offsets
// (workgroup 0) and writes the status.
__global__ __launch_bounds__(256) void glr_setup_kernel(GlrArgs a, size_t words, uint32_t cols) {
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < cols; i += gridDim.x * 256) a.counters[(size_t)i * kGlrCounterStride] = 0;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < words; i += (size_t)gridDim.x * 256) a.words[i] = ~0ull;
  if (blockIdx.x != 0) return;
  const bool ok = glr_seqlens_ok(a.cu, a.N, a.T);
  if (threadIdx.x == 0) {
    *a.status = ok ? 0 : kDevBadSeqlens;
  }
}

template <typename T, typename G, bool RAW, bool CONVEX, int L, int W>
__global__ __launch_bounds__(W * 64, 4) void glr_forward_kernel(GlrArgs a, uint32_t tiles, uint32_t cols) {
  __shared__ float sA[W][64], sB[W][64], sIn[64];
  __shared__ int sIds[W][2 * L], sReset[W];
  __shared__ int32_t sCu[kLdsOffsets + 1];
  __shared__ uint32_t sNext;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Offsets cu = stage_offsets(a.cu, a.N, sCu);
  bool ok = true;
  if (tiles > 1) {
    ok = *a.status == 0;
  } else {  // no setup kernel ran
    ok = glr_seqlens_ok(a.cu, a.N, a.T);
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = ok ? 0 : kDevBadSeqlens;
  }
  if (!ok || a.T == 0) {  // no tokens: the states pass through
    for (uint32_t col = blockIdx.x; col < cols; col += gridDim.x)
      pass_empty(a.cu, a.N, a.T, ok, a.s0, a.s_final, a.D, col * 64 + lane);
    return;
  }
  for (uint32_t turn = blockIdx.x; turn < tiles * cols; turn += gridDim.x) {
    const uint32_t col = __builtin_amdgcn_readfirstlane(turn % cols), at = col * 64 + lane;
    if (threadIdx.x == 0) sNext = tiles > 1 ? take_tile(a, col) : 0;
    __syncthreads();
    const uint32_t tile = __builtin_amdgcn_readfirstlane(sNext);
    const bool mine = at < (uint32_t)a.D;
    const uint32_t c = glr_channel(at, (uint32_t)a.D);  // lanes that are not `mine` store nothing
    if (tile == 0) pass_empty(a.cu, a.N, a.T, ok, a.s0, a.s_final, a.D, at);

    // the wave's tokens; rows past the end are loaded from the last one
    const long t0 = (long)tile * (W * L) + wave * L;
    const int count = (int)min((long)L, max(0l, (long)a.T - t0));
    T x[L];
    G g[L];
    const T *px = static_cast<const T *>(a.x) + min(t0, (long)a.T - 1) * a.xs;
    const G *pg = static_cast<const G *>(a.g) + min(t0, (long)a.T - 1) * a.gs;
#pragma unroll
    for (int i = 0; i < L; ++i) {
      x[i] = __builtin_nontemporal_load(in_row(px, c));
      g[i] = __builtin_nontemporal_load(in_row(pg, c));
      px += i + 1 < count ? a.xs : 0;
      pg += i + 1 < count ? a.gs : 0;
    }
    const Marks<L> m = find_marks<L>(cu, a.T, t0, sIds[wave]);
    // The initial state of the last sequence that starts here, the only one that can
    // reach past the wave's tokens.  It is read before the tile's map is published, the
    // others' when their tokens' turn comes: where s_final is s0, a state is written by
    // this wave after that, or by one that waits for the map.
    const int start = m.first ? 31 - __builtin_clz(m.first) : -1;
    float s0 = 0.f;
    if (m.first && a.s0) s0 = *in_row(a.s0 + (size_t)m.starts(start) * a.D, c);

    if (count < L) {  // the last tile: tokens past the end pass the state on
#pragma unroll
      for (int i = 0; i < L; ++i)
        if (i >= count) {
          x[i] = Elt<T>::from_f32(0.f);
          g[i] = Elt<G>::from_f32(RAW ? -__builtin_inff() : 0.f);
        }
    }
    float k[L], b[L], A = 1.f, B = 0.f;  // h_t = k h_{t-1} + b; over the wave's tokens A h + B
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const Gate q = glr_gate<RAW>(Elt<G>::to_f32(g[i]));
      const float u = Elt<T>::to_f32(x[i]);
      k[i] = q.a;
      b[i] = CONVEX ? q.forget * u : u;
    }
    if (m.first == 0) {
#pragma unroll
      for (int i = 0; i < L; ++i) {
        A *= k[i];
        B = k[i] * B + b[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < L; ++i) B = k[i] * (i == start ? s0 : B) + b[i];
    }
    sA[wave][lane] = A;
    sB[wave][lane] = B;
    if (lane == 0) sReset[wave] = m.first != 0;
    __syncthreads();

    if (wave == 0) {
      bool reset = false;
      A = 1.f;
      B = 0.f;
#pragma unroll 1
      for (int w = 0; w < W; ++w) {
        const bool r = sReset[w];
        reset |= r;
        B = r ? sB[w][lane] : sA[w][lane] * B + sB[w][lane];
        A *= sA[w][lane];
      }
      const bool pass_on = tile + 1 < tiles && mine;
      uint64_t *row = a.words + (size_t)tile * a.D;
      if (pass_on) {
        if (reset) publish(row, c, kState, B);
        else publish_map(row, c, A, B);
      }
      float s = 0.f;
      if (tile > 0 && !(m.first & 1)) s = look_back(a.words, a.D, c, (long)tile - 1, -1, tile, a.status);
      if (pass_on && !reset) publish(row, c, kState, __builtin_fmaf(A, s, B));
      sIn[lane] = s;
    }
    __syncthreads();

    float s = sIn[lane];
#pragma unroll 1
    for (int w = 0; w < wave; ++w) s = sReset[w] ? sB[w][lane] : sA[w][lane] * s + sB[w][lane];
    if (a.ckpt && t0 % kGlrGroup == 0 && count > 0 && mine) *in_row(a.ckpt + (size_t)(t0 / kGlrGroup) * a.D, c) = s;
    if ((m.first | m.last) == 0 && count == L) {
      Rows<T> rh(static_cast<T *>(a.h) + (size_t)t0 * a.D, a.D, c);
#pragma unroll
      for (int i = 0; i < L; ++i) {
        s = k[i] * s + b[i];
        if (mine) __builtin_nontemporal_store(Elt<T>::from_f32(s), rh.here());
        rh.advance();
      }
    } else {
      for (int lo = 0; lo < count;) {  // from one sequence's first token to the next one's
        if (m.first >> lo & 1) {
          s = lo == start ? s0 : 0.f;
          if (lo != start && a.s0) s = *in_row(a.s0 + (size_t)m.starts(lo) * a.D, c);
        }
        const uint32_t later = m.first & ~((2u << lo) - 1);
        const int hi = later ? __builtin_ctz(later) : count;
#pragma unroll
        for (int i = 0; i < L; ++i)
          if (i >= lo && i < hi) {
            s = k[i] * s + b[i];
            if (mine) *in_row(static_cast<T *>(a.h) + (size_t)(t0 + i) * a.D, c) = Elt<T>::from_f32(s);
          }
        if ((m.last >> (hi - 1) & 1) && a.s_final && mine) *in_row(a.s_final + (size_t)m.ends(hi - 1) * a.D, c) = s;
        lo = hi;
      }
    }
    __syncthreads();  // LDS is used again in the next turn
  }
}

// ------------------------------------------------------------- single tokens
// A thread holds four channels of one sequence (one, where D is no multiple of four): bound
// by the state's way there and back, 256 sequences x 4096 channels 4.5 us (14 MB), and for
// few sequences by the launch (one of 2048 channels 2.0 us).
constexpr int kStepThreads = 256;

template <typename T, int V> struct __attribute__((packed, aligned(sizeof(T)))) Elems {
  T v[V];
};

template <typename T, typename G, bool RAW, bool CONVEX, int V>
__global__ __launch_bounds__(kStepThreads) void glr_step_kernel(GlrStepArgs a, uint32_t cols, uint32_t items) {
  for (uint32_t i = blockIdx.x * kStepThreads + threadIdx.x; i < items; i += gridDim.x * kStepThreads) {
    const uint32_t n = i / cols, c = (i - n * cols) * V;
    Elems<T, V> *h = reinterpret_cast<Elems<T, V> *>(static_cast<T *>(a.h) + (size_t)n * a.D + c);
    const auto g = *reinterpret_cast<const Elems<G, V> *>(static_cast<const G *>(a.g) + (size_t)n * a.gs + c);
    const auto x = *reinterpret_cast<const Elems<T, V> *>(static_cast<const T *>(a.x) + (size_t)n * a.xs + c);
    const int slot = a.slots ? a.slots[n] : (int)n;
    Elems<T, V> out;
    if (slot < 0 || slot >= a.num_slots) {  // padding entry
#pragma unroll
      for (int e = 0; e < V; ++e) out.v[e] = Elt<T>::from_f32(0.f);
      *h = out;
      continue;
    }
    Elems<float, V> *row = reinterpret_cast<Elems<float, V> *>(a.state + (size_t)slot * a.D + c);
    Elems<float, V> s = *row;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const Gate k = glr_gate<RAW>(Elt<G>::to_f32(g.v[e]));
      const float u = Elt<T>::to_f32(x.v[e]);
      s.v[e] = k.a * s.v[e] + (CONVEX ? k.forget * u : u);
      out.v[e] = Elt<T>::from_f32(s.v[e]);
    }
    *row = s;
    *h = out;
  }
}

hipError_t launch_glr_setup(const GlrArgs &a, size_t words, uint32_t cols, hipStream_t s) {
  const size_t blocks = (words + 256 * 8 - 1) / (256 * 8);
  hipLaunchKernelGGL(glr_setup_kernel, dim3((unsigned)(blocks < 1 ? 1 : blocks < 4096 ? blocks : 4096)), dim3(256), 0, s, a,
                     words, cols);
  return hipGetLastError();
}

template <typename T, typename G> struct Forward {
  template <bool RAW, bool CONVEX, int L, int W> static hipError_t tiled(const GlrArgs &a, hipStream_t s) {
    constexpr int kTile = W * L;
    const long tiles = a.T > 0 ? ((long)a.T + kTile - 1) / kTile : 1, cols = ((long)a.D + 63) / 64;
    if (tiles * cols > 0xffff0000l) return hipErrorInvalidValue;  // the turns' range
    if (tiles > 1 && kTile < kGlrLeastTile) return hipErrorInvalidValue;  // the workspace's words
    if (tiles > 1) {
      const hipError_t e = launch_glr_setup(a, (size_t)tiles * a.D, (uint32_t)cols, s);
      if (e != hipSuccess) return e;
    }
    const long resident = 16 / W * glr_cus(a);  // 16 waves a CU
    const unsigned grid = (unsigned)(tiles * cols < resident ? tiles * cols : resident);
    hipLaunchKernelGGL((glr_forward_kernel<T, G, RAW, CONVEX, L, W>), dim3(grid), dim3(W * 64), 0, s, a, (uint32_t)tiles,
                       (uint32_t)cols);
    return hipGetLastError();
  }
  // Up to 256 tokens a call is one tile, which needs no setup kernel and a launch less (512
  // in one tile of 16 x 32 take longer than the setup: 400 x 2048 14.7 us and 11.2).
  // Beyond, few tiles keep the chain of states short, but there should be as many as CUs.
  // Tiles of 128 tokens instead of 256, us a call: 777 x 1280 11.2 and 14.6, 2048 x 2048
  // fp32 17.4 and 20.4, 8192 x 256 17.9 and 19.1; but 4096 x 2048 (512 tiles of 256) 25.9
  // and 23.2, 32768 x 2048 157 and 119.  Of 64 instead of 128: 777 x 1280 10.6 and 11.2,
  // 4096 x 256 16.8 and 15.0, 2048 x 2048 fp32 20.6 and 17.3.  Where a long call has few
  // channels its tiles all wait for each other.  In tiles of 128, 256 (the better of 8 waves
  // x 32 and 16 x 16) and 512:
  //    8192 x 256   18.7  17.8  20.6      20000 x 128  27.2  21.2  22.0
  //   10000 x 256   19.4  17.6  19.2      30000 x 128  36.3  25.7  23.6
  //   16384 x 256   25.9  22.0  23.2      50000 x 64   52.9  33.5  27.4
  template <bool RAW, bool CONVEX> static hipError_t go(const GlrArgs &a, hipStream_t s) {
    if (a.T <= 64) return tiled<RAW, CONVEX, 8, 8>(a, s);
    if (a.T <= 128) return tiled<RAW, CONVEX, 16, 8>(a, s);
    if (a.T <= 256) return tiled<RAW, CONVEX, 16, 16>(a, s);
    if (glr_tiles(a, 256) > glr_cus(a)) return tiled<RAW, CONVEX, 32, 8>(a, s);
    return a.T <= 8192 ? tiled<RAW, CONVEX, 16, 8>(a, s) : tiled<RAW, CONVEX, 32, 16>(a, s);
  }
};

template <typename T, typename G> struct Step {
  template <bool RAW, bool CONVEX, int V> static hipError_t wide(const GlrStepArgs &a, hipStream_t s) {
    const uint32_t cols = (uint32_t)a.D / V, items = cols * (uint32_t)a.N;  // N x D < 2^31
    const uint32_t blocks = (items + kStepThreads - 1) / kStepThreads;
    hipLaunchKernelGGL((glr_step_kernel<T, G, RAW, CONVEX, V>), dim3(blocks < 1u << 20 ? blocks : 1u << 20),
                       dim3(kStepThreads), 0, s, a, cols, items);
    return hipGetLastError();
  }
  template <bool RAW, bool CONVEX> static hipError_t go(const GlrStepArgs &a, hipStream_t s) {
    return a.D % 4 == 0 ? wide<RAW, CONVEX, 4>(a, s) : wide<RAW, CONVEX, 1>(a, s);
  }
};

hipError_t launch_glr_forward(const GlrArgs &a, const GlrForm &f, hipStream_t s) { return glr_dispatch<Forward>(a, f, s); }
hipError_t launch_glr_step(const GlrStepArgs &a, const GlrForm &f, hipStream_t s) { return glr_dispatch<Step>(a, f, s); }

}  // namespace hagdn

// k7_glr_backward.hip -- the gated linear recurrence's backward pass.  With d_t the
// gradient of h_t and e_t = a_t d_t,
//   d_t = dh_t + e_{t+1},  dx_t = w_t d_t,  d(log a_t) = e_t (h_{t-1} - [convex] x_t).
//
// The scan of glr.h runs over e from the last tile to the first, eight waves of 16
// tokens to a tile of 64 channels.  The states h_{t-1} are not read: each tile forms them
// again in fp32 from the saved state before its first token, in the same registers and
// with one more map a wave in LDS, which costs three operations an element and saves
// reading h, and its rounding.  Bound by HBM: x, g and dh are read once, dx and dg written
// once.  32768 tokens x 2048 channels, bf16 with an fp32 gate: 190 us, 4.9 TB/s of the
// 940 MB that must move, in convex form 202; the gate in bf16 163 us and, raw and convex,
// 181 (4.1 and 3.7 TB/s: the same two workgroups a CU hold fewer bytes in flight).  The raw
// and the convex forms spill 7 to 11 of their 128 registers.
#include "glr.h"

namespace hagdn {

template <typename T, typename G, bool RAW, bool CONVEX, int L, int W>
__global__ __launch_bounds__(W * 64, 4) void glr_backward_kernel(GlrArgs a, uint32_t tiles, uint32_t cols) {
  static_assert(W * L % kGlrGroup == 0, "a tile starts at a saved state");
  __shared__ float sA[W][64], sF[W][64], sR[W][64], sIn[64];
  __shared__ int sIds[W][2 * L], sFirst[W], sLast[W], sEnded;
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
      pass_empty(a.cu, a.N, a.T, ok, a.dfinal, a.ds0, a.D, col * 64 + lane);
    return;
  }
  for (uint32_t turn = blockIdx.x; turn < tiles * cols; turn += gridDim.x) {
    const uint32_t col = __builtin_amdgcn_readfirstlane(turn % cols), at = col * 64 + lane;
    if (threadIdx.x == 0) sNext = tiles > 1 ? take_tile(a, col) : 0;
    __syncthreads();
    const uint32_t tile = tiles - 1 - __builtin_amdgcn_readfirstlane(sNext);
    const bool mine = at < (uint32_t)a.D;
    const uint32_t c = glr_channel(at, (uint32_t)a.D);  // lanes that are not `mine` store nothing
    if (tile == 0) pass_empty(a.cu, a.N, a.T, ok, a.dfinal, a.ds0, a.D, at);

    // the wave's tokens; rows past the end are loaded from the last one
    const long t0 = (long)tile * (W * L) + wave * L;
    const int count = (int)min((long)L, max(0l, (long)a.T - t0));
    T x[L], y[L];  // y: dh
    G g[L];
    const long row = min(t0, (long)a.T - 1);
    Rows<const T> rx(static_cast<const T *>(a.x) + row * a.xs, a.xs, c);
    Rows<const G> rg(static_cast<const G *>(a.g) + row * a.gs, a.gs, c);
    Rows<const T> ry(static_cast<const T *>(a.dh) + row * a.dhs, a.dhs, c);
    if (count == L) {
#pragma unroll
      for (int i = 0; i < L; ++i) {
        x[i] = __builtin_nontemporal_load(rx.here());
        g[i] = __builtin_nontemporal_load(rg.here());
        y[i] = __builtin_nontemporal_load(ry.here());
        rx.advance();
        rg.advance();
        ry.advance();
      }
    } else {
#pragma unroll
      for (int i = 0; i < L; ++i) {
        x[i] = *rx.here();
        g[i] = *rg.here();
        y[i] = *ry.here();
        if (i + 1 < count) rx.advance(), rg.advance(), ry.advance();
      }
    }
    float s = *in_row(a.ckpt + (size_t)tile * (W * L / kGlrGroup) * a.D, c);
    const Marks<L> m = find_marks<L>(cu, a.T, t0, sIds[wave]);
    // The last sequence that starts here is the only one to reach past the wave's tokens,
    // the first that ends here the only one to come from before them; its dfinal is read
    // before the tile's map is published, the others' when their tokens' turn comes:
    // where ds0 is dfinal, a gradient is written by this wave after that, or by one that
    // waits for the map.
    const int start = m.first ? 31 - __builtin_clz(m.first) : -1, end = m.last ? __builtin_ctz(m.last) : -1;
    float s0 = 0.f, df = 0.f;
    if (m.first && a.s0) s0 = *in_row(a.s0 + (size_t)m.starts(start) * a.D, c);
    if (m.last && a.dfinal) df = *in_row(a.dfinal + (size_t)m.ends(end) * a.D, c);

    if (count < L) {  // the last tile: tokens past the end pass everything on
#pragma unroll
      for (int i = 0; i < L; ++i)
        if (i >= count) {
          x[i] = y[i] = Elt<T>::from_f32(0.f);
          g[i] = Elt<G>::from_f32(RAW ? -__builtin_inff() : 0.f);
        }
    }
    float k[L], f[L], u[L], d[L];  // decay, its complement, x, dh
    float A = 1.f, F = 0.f, R = 0.f;  // the tokens' maps: of the state A h + F, of e going back A e + R
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const Gate q = glr_gate<RAW>(Elt<G>::to_f32(g[i]));
      k[i] = q.a;
      f[i] = q.forget;
      u[i] = Elt<T>::to_f32(x[i]);
      d[i] = Elt<T>::to_f32(y[i]);
    }
    auto step = [&](int i, float h) { return k[i] * h + (CONVEX ? f[i] * u[i] : u[i]); };
    if (m.first == 0) {
#pragma unroll
      for (int i = 0; i < L; ++i) A *= k[i], F = step(i, F);
    } else {
#pragma unroll
      for (int i = 0; i < L; ++i) A *= k[i], F = step(i, i == start ? s0 : F);
    }
    if (m.last == 0) {
#pragma unroll
      for (int i = L - 1; i >= 0; --i) R = k[i] * (d[i] + R);
    } else {
#pragma unroll
      for (int i = L - 1; i >= 0; --i) R = k[i] * (d[i] + (i == end ? df : R));
    }
    sA[wave][lane] = A;
    sF[wave][lane] = F;
    sR[wave][lane] = R;
    if (lane == 0) {
      sFirst[wave] = m.first != 0;
      sLast[wave] = m.last != 0;
      if (wave == W - 1) sEnded = m.last >> (L - 1) & 1;
    }
    __syncthreads();

    if (wave == 0) {
      bool reset = false;
      A = 1.f;
      R = 0.f;
#pragma unroll 1
      for (int w = W - 1; w >= 0; --w) {
        const bool r = sLast[w];
        reset |= r;
        R = r ? sR[w][lane] : sA[w][lane] * R + sR[w][lane];
        A *= sA[w][lane];
      }
      const bool pass_on = tile > 0 && mine;
      uint64_t *words = a.words + (size_t)tile * a.D;
      if (pass_on) {
        if (reset) publish(words, c, kState, R);
        else publish_map(words, c, A, R);
      }
      float e = 0.f;
      if (tile + 1 < tiles && !sEnded) e = look_back(a.words, a.D, c, (long)tile + 1, 1, (long)tiles - 1 - tile, a.status);
      if (pass_on && !reset) publish(words, c, kState, __builtin_fmaf(A, e, R));
      sIn[lane] = e;
    }
    __syncthreads();

    float e = sIn[lane];
#pragma unroll 1
    for (int w = W - 1; w > wave; --w) e = sLast[w] ? sR[w][lane] : sA[w][lane] * e + sR[w][lane];
#pragma unroll 1
    for (int w = 0; w < wave; ++w) s = sFirst[w] ? sF[w][lane] : sA[w][lane] * s + sF[w][lane];

    auto state = [&](int i) {  // u: the state before the token, less x where convex
      const float h = step(i, s);
      u[i] = CONVEX ? s - u[i] : s;
      s = h;
    };
    auto grads = [&](int i, T &dx, G &dg) {
      const float di = d[i] + e;
      e = k[i] * di;
      dx = Elt<T>::from_f32(CONVEX ? f[i] * di : di);
      dg = Elt<G>::from_f32(RAW ? -f[i] * (e * u[i]) : e * u[i]);
    };
    if ((m.first | m.last) == 0 && count == L) {
#pragma unroll
      for (int i = 0; i < L; ++i) state(i);
      Rows<T> rdx(static_cast<T *>(a.dx) + (size_t)(t0 + L - 1) * a.D, -(long)a.D, c);
      Rows<G> rdg(static_cast<G *>(a.dg) + (size_t)(t0 + L - 1) * a.D, -(long)a.D, c);
#pragma unroll
      for (int i = L - 1; i >= 0; --i) {
        T dx;
        G dg;
        grads(i, dx, dg);
        if (mine) {
          __builtin_nontemporal_store(dx, rdx.here());
          __builtin_nontemporal_store(dg, rdg.here());
        }
        rdx.advance();
        rdg.advance();
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
          if (i >= lo && i < hi) state(i);
        lo = hi;
      }
      for (int hi = count; hi > 0;) {  // from one sequence's last token back to the one before
        if (m.last >> (hi - 1) & 1) {
          e = hi - 1 == end ? df : 0.f;
          if (hi - 1 != end && a.dfinal) e = *in_row(a.dfinal + (size_t)m.ends(hi - 1) * a.D, c);
        }
        const uint32_t sooner = m.last & ((1u << (hi - 1)) - 1);
        const int lo = sooner ? 32 - __builtin_clz(sooner) : 0;
#pragma unroll
        for (int i = L - 1; i >= 0; --i)
          if (i >= lo && i < hi) {
            T dx;
            G dg;
            grads(i, dx, dg);
            if (mine) {
              *in_row(static_cast<T *>(a.dx) + (size_t)(t0 + i) * a.D, c) = dx;
              *in_row(static_cast<G *>(a.dg) + (size_t)(t0 + i) * a.D, c) = dg;
            }
          }
        if ((m.first >> lo & 1) && a.ds0 && mine) *in_row(a.ds0 + (size_t)m.starts(lo) * a.D, c) = e;
        hi = lo;
      }
    }
    __syncthreads();  // LDS is used again in the next turn
  }
}

template <typename T, typename G> struct Backward {
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
    hipLaunchKernelGGL((glr_backward_kernel<T, G, RAW, CONVEX, L, W>), dim3(grid), dim3(W * 64), 0, s, a, (uint32_t)tiles,
                       (uint32_t)cols);
    return hipGetLastError();
  }
  // Tiles of 128 tokens; of 256 where that makes one tile of a call, and where a long call
  // has so few channels that its tiles all wait for each other (forward: k6_glr.hip).  Tiles
  // of 128 and 256, us a call: 4096 x 256 15.9 and 17.1, 6000 x 128 17.4 and 17.5, 8192 x 256
  // 20.3 and 19.4, 10000 x 256 22.2 and 20.2, 20000 x 128 30.6 and 24.5, 50000 x 64 57.9 and 37.7.
  template <bool RAW, bool CONVEX> static hipError_t go(const GlrArgs &a, hipStream_t s) {
    const bool narrow = a.T > 8192 && glr_tiles(a, 128) <= 2 * glr_cus(a);
    return (a.T > 128 && a.T <= 256) || narrow ? tiled<RAW, CONVEX, 16, 16>(a, s) : tiled<RAW, CONVEX, 16, 8>(a, s);
  }
};

hipError_t launch_glr_backward(const GlrArgs &a, const GlrForm &f, hipStream_t s) { return glr_dispatch<Backward>(a, f, s); }

}  // namespace hagdn

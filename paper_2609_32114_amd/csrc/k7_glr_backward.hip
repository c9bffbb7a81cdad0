// k7_glr_backward.hip -- the gated linear recurrence's backward pass.
#include "glr.h"

namespace hagdn {

constexpr int kGlrThreads = 64;

template <typename T, typename G, bool RAW, bool CONVEX>
__global__ __launch_bounds__(kGlrThreads) void glr_backward_kernel(GlrArgs a) {
  __shared__ float before[kGlrGroup][kGlrThreads];  // the states before a group's tokens
  const int cols = (a.D + kGlrThreads - 1) / kGlrThreads;
  const int n = blockIdx.x / cols, c = blockIdx.x % cols * kGlrThreads + threadIdx.x;
  const bool ok = glr_seqlens_ok(a.cu, a.N, a.T);
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = ok ? 0 : kDevBadSeqlens;
  if (c >= a.D) return;
  const int t0 = !ok ? 0 : a.cu ? a.cu[n] : 0, t1 = !ok ? 0 : a.cu ? a.cu[n + 1] : a.T;
  const T *x = static_cast<const T *>(a.x) + c, *dh = static_cast<const T *>(a.dh) + c;
  const G *g = static_cast<const G *>(a.g) + c;
  T *dx = static_cast<T *>(a.dx) + c;
  G *dg = static_cast<G *>(a.dg) + c;
  float e = a.dfinal ? a.dfinal[(size_t)n * a.D + c] : 0.f;
  for (int hi = t1; hi > t0;) {
    const int grp = (hi - 1) / kGlrGroup, lo = max(t0, grp * kGlrGroup);
    float s = lo > t0 ? a.ckpt[(size_t)grp * a.D + c] : a.s0 ? a.s0[(size_t)n * a.D + c] : 0.f;
    for (int t = lo; t < hi; ++t) {
      before[t - lo][threadIdx.x] = s;
      const Gate k = glr_gate<RAW>(Elt<G>::to_f32(g[(size_t)t * a.gs]));
      const float u = Elt<T>::to_f32(x[(size_t)t * a.xs]);
      s = k.a * s + (CONVEX ? k.forget * u : u);
    }
    for (int t = hi - 1; t >= lo; --t) {
      const Gate k = glr_gate<RAW>(Elt<G>::to_f32(g[(size_t)t * a.gs]));
      const float d = Elt<T>::to_f32(dh[(size_t)t * a.dhs]) + e;
      e = k.a * d;
      float u = before[t - lo][threadIdx.x];
      if (CONVEX) u -= Elt<T>::to_f32(x[(size_t)t * a.xs]);
      dx[(size_t)t * a.D] = Elt<T>::from_f32(CONVEX ? k.forget * d : d);
      dg[(size_t)t * a.D] = Elt<G>::from_f32(RAW ? -k.forget * (e * u) : e * u);
    }
    hi = lo;
  }
  if (a.ds0) a.ds0[(size_t)n * a.D + c] = e;
}

template <typename T, typename G> struct Backward {
  template <bool RAW, bool CONVEX> static hipError_t go(const GlrArgs &a, hipStream_t s) {
    const dim3 grid((unsigned)((size_t)a.N * ((a.D + kGlrThreads - 1) / kGlrThreads)));
    hipLaunchKernelGGL((glr_backward_kernel<T, G, RAW, CONVEX>), grid, dim3(kGlrThreads), 0, s, a);
    return hipGetLastError();
  }
};

hipError_t launch_glr_backward(const GlrArgs &a, const GlrForm &f, hipStream_t s) { return glr_dispatch<Backward>(a, f, s); }

}  // namespace hagdn

// k6_glr.hip -- the gated linear recurrence: h_t = a_t h_{t-1} + w_t x_t per
// channel, with a_t = e^g_t and w_t = 1 or 1 - a_t, over packed sequences; its
// backward pass; and one step for single tokens.
//
// One thread walks one channel of one sequence.
#include "device.h"
#include "glr.h"
#include "layer.h"
#include "prefill.h"

namespace hagdn {

constexpr int kGlrThreads = 64;

// Whether cu[0 .. N] are the offsets of N sequences over T tokens; every thread of
// the workgroup takes part and gets the answer.
__device__ __forceinline__ bool glr_seqlens_ok(const int32_t *cu, int N, int T) {
  if (!cu) return true;
  int bad = 0;
  for (int i = threadIdx.x; i < N; i += blockDim.x) bad |= cu[i] > cu[i + 1];
  if (threadIdx.x == 0) bad |= cu[0] != 0 || cu[N] != T;
  return !__syncthreads_or(bad);
}

template <typename T, typename G, bool RAW, bool CONVEX>
__global__ __launch_bounds__(kGlrThreads) void glr_forward_kernel(GlrArgs a) {
  const int cols = (a.D + kGlrThreads - 1) / kGlrThreads;
  const int n = blockIdx.x / cols, c = blockIdx.x % cols * kGlrThreads + threadIdx.x;
  const bool ok = glr_seqlens_ok(a.cu, a.N, a.T);
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = ok ? 0 : kDevBadSeqlens;
  if (c >= a.D) return;
  const int t0 = !ok ? 0 : a.cu ? a.cu[n] : 0, t1 = !ok ? 0 : a.cu ? a.cu[n + 1] : a.T;
  const T *x = static_cast<const T *>(a.x) + c;
  const G *g = static_cast<const G *>(a.g) + c;
  T *h = static_cast<T *>(a.h) + c;
  float s = a.s0 ? a.s0[(size_t)n * a.D + c] : 0.f;
  for (int t = t0; t < t1; ++t) {
    if (a.ckpt && t % kGlrGroup == 0) a.ckpt[(size_t)(t / kGlrGroup) * a.D + c] = s;
    const Gate k = glr_gate<RAW>(Elt<G>::to_f32(g[(size_t)t * a.gs]));
    const float u = Elt<T>::to_f32(x[(size_t)t * a.xs]);
    s = k.a * s + (CONVEX ? k.forget * u : u);
    h[(size_t)t * a.D] = Elt<T>::from_f32(s);
  }
  if (a.s_final) a.s_final[(size_t)n * a.D + c] = s;
}

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

template <typename T, typename G, bool RAW, bool CONVEX>
__global__ __launch_bounds__(kGlrThreads) void glr_step_kernel(GlrStepArgs a) {
  const int cols = (a.D + kGlrThreads - 1) / kGlrThreads;
  const int n = blockIdx.x / cols, c = blockIdx.x % cols * kGlrThreads + threadIdx.x;
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

// The kernel's instance for a form: K<T, G, RAW, CONVEX>.
#define HAGDN_GLR_FORM(K, grid, block, stream, args)                                                            \
  do {                                                                                                         \
    if (!f.bf16) HAGDN_GLR_TYPES(K, float, float, grid, block, stream, args);                                   \
    else if (f.gate_bf16) HAGDN_GLR_TYPES(K, bf16_t, bf16_t, grid, block, stream, args);                        \
    else HAGDN_GLR_TYPES(K, bf16_t, float, grid, block, stream, args);                                          \
  } while (0)
#define HAGDN_GLR_TYPES(K, T, G, grid, block, stream, args)                                                     \
  do {                                                                                                         \
    if (f.raw && f.convex) hipLaunchKernelGGL((K<T, G, true, true>), grid, block, 0, stream, args);             \
    else if (f.raw) hipLaunchKernelGGL((K<T, G, true, false>), grid, block, 0, stream, args);                   \
    else if (f.convex) hipLaunchKernelGGL((K<T, G, false, true>), grid, block, 0, stream, args);                \
    else hipLaunchKernelGGL((K<T, G, false, false>), grid, block, 0, stream, args);                             \
  } while (0)

hipError_t launch_glr_forward(const GlrArgs &a, const GlrForm &f, hipStream_t s) {
  const dim3 grid((unsigned)((size_t)a.N * ((a.D + kGlrThreads - 1) / kGlrThreads)));
  HAGDN_GLR_FORM(glr_forward_kernel, grid, dim3(kGlrThreads), s, a);
  return hipGetLastError();
}

hipError_t launch_glr_backward(const GlrArgs &a, const GlrForm &f, hipStream_t s) {
  const dim3 grid((unsigned)((size_t)a.N * ((a.D + kGlrThreads - 1) / kGlrThreads)));
  HAGDN_GLR_FORM(glr_backward_kernel, grid, dim3(kGlrThreads), s, a);
  return hipGetLastError();
}

hipError_t launch_glr_step(const GlrStepArgs &a, const GlrForm &f, hipStream_t s) {
  const dim3 grid((unsigned)((size_t)a.N * ((a.D + kGlrThreads - 1) / kGlrThreads)));
  HAGDN_GLR_FORM(glr_step_kernel, grid, dim3(kGlrThreads), s, a);
  return hipGetLastError();
}

}  // namespace hagdn

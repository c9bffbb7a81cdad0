// k8_norms.hip -- the norms before and after a block, fused with the residual
// stream's scaled add (add_norm) and with the mixer's output gate (gate_norm),
// and their backward passes.
//
// One workgroup per row; the backward kernels' workgroups take rows in turn and
// each keeps its own partial sums of the weights' gradients, which a second
// kernel adds in a fixed order.
#include "device.h"
#include "layer.h"

namespace hagdn {

constexpr int kNormThreads = 256;
constexpr unsigned kMaxGrid = 1 << 20;  // workgroups: a launch holds fewer than 2^32 threads

template <int K> __device__ __forceinline__ void block_sums(float (&v)[K]) {
  __shared__ float s[kNormThreads / 64][K];
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = wave_sum(v[k]);
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int k = 0; k < K; ++k) s[threadIdx.x >> 6][k] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) {
    v[k] = 0.f;
    for (int w = 0; w < kNormThreads / 64; ++w) v[k] += s[w][k];
  }
  __syncthreads();
}

template <typename T, typename R> __global__ __launch_bounds__(kNormThreads) void add_norm_kernel(AddNormArgs a) {
  for (size_t t = blockIdx.x; t < (size_t)a.T; t += gridDim.x) {
  const T *x = static_cast<const T *>(a.x) + t * a.xs;
  const R *res = a.res ? static_cast<const R *>(a.res) + t * a.rs : nullptr;
  const float inv = 1.f / (float)a.D;
  float rx = 1.f;
  if (a.post) {
    float v[1] = {0.f};
    for (int c = threadIdx.x; c < a.D; c += kNormThreads) {
      const float u = Elt<T>::to_f32(x[c]);
      v[0] += u * u;
    }
    block_sums(v);
    rx = 1.f / sqrtf(v[0] * inv + a.eps);
  }
  auto stream = [&](int c) {  // r' = r + s u
    const float u = Elt<T>::to_f32(x[c]) * (a.post ? rx * a.post[c] : 1.f);
    const float s = a.scale_vec ? a.scale_vec[c] : a.scale;
    return (res ? Elt<R>::to_f32(res[c]) : 0.f) + s * u;
  };
  float v[1] = {0.f};
  for (int c = threadIdx.x; c < a.D; c += kNormThreads) {
    const float r = stream(c);
    v[0] += r * r;
  }
  block_sums(v);
  const float rr = 1.f / sqrtf(v[0] * inv + a.eps);
  for (int c = threadIdx.x; c < a.D; c += kNormThreads) {
    const float r = stream(c);
    static_cast<T *>(a.y)[t * a.D + c] = Elt<T>::from_f32(r * rr * a.w[c]);
    if (a.res_out) static_cast<R *>(a.res_out)[t * a.D + c] = Elt<R>::from_f32(r);
  }
  }
}

template <typename T, typename R>
__global__ __launch_bounds__(kNormThreads) void add_norm_backward_kernel(AddNormArgs a) {
  const float inv = 1.f / (float)a.D;
  const int outs = 1 + (a.dscale != nullptr) + (a.dpost != nullptr);
  float *pw = a.partial + (size_t)blockIdx.x * outs * a.D, *ps = pw + a.D, *pp = a.dscale ? ps + a.D : ps;
  for (int i = threadIdx.x; i < outs * a.D; i += kNormThreads) pw[i] = 0.f;
  __syncthreads();
  for (size_t t = blockIdx.x; t < (size_t)a.T; t += gridDim.x) {
    const T *x = a.x ? static_cast<const T *>(a.x) + t * a.xs : nullptr;
    const T *dy = static_cast<const T *>(a.dy) + t * a.dys;
    const R *res = static_cast<const R *>(a.res) + t * a.rs;
    const R *din = a.dres ? static_cast<const R *>(a.dres) + t * a.drs : nullptr;
    float v[3] = {0.f, 0.f, 0.f};  // sums of r'^2, r' w dy, x^2
    for (int c = threadIdx.x; c < a.D; c += kNormThreads) {
      const float r = Elt<R>::to_f32(res[c]);
      v[0] += r * r;
      v[1] += r * a.w[c] * Elt<T>::to_f32(dy[c]);
      if (a.post) v[2] += Elt<T>::to_f32(x[c]) * Elt<T>::to_f32(x[c]);
    }
    block_sums(v);
    const float rr = 1.f / sqrtf(v[0] * inv + a.eps), m = rr * rr * v[1] * inv;
    const float rx = 1.f / sqrtf(v[2] * inv + a.eps);
    auto total = [&](int c) {  // the gradient of r'
      const float d = rr * (a.w[c] * Elt<T>::to_f32(dy[c]) - Elt<R>::to_f32(res[c]) * m);
      return din ? Elt<R>::to_f32(din[c]) + d : d;
    };
    auto scale = [&](int c) { return a.scale_vec ? a.scale_vec[c] : a.scale; };
    float mx = 0.f;
    if (a.post) {
      float q[1] = {0.f};
      for (int c = threadIdx.x; c < a.D; c += kNormThreads)
        q[0] += Elt<T>::to_f32(x[c]) * a.post[c] * scale(c) * total(c);
      block_sums(q);
      mx = rx * rx * q[0] * inv;
    }
    for (int c = threadIdx.x; c < a.D; c += kNormThreads) {
      const float d = total(c), du = scale(c) * d, xn = x ? Elt<T>::to_f32(x[c]) * (a.post ? rx : 1.f) : 0.f;
      pw[c] += Elt<T>::to_f32(dy[c]) * Elt<R>::to_f32(res[c]) * rr;
      if (a.dscale) ps[c] += d * xn * (a.post ? a.post[c] : 1.f);
      if (a.dpost) pp[c] += du * xn;
      const float dx = a.post ? rx * (a.post[c] * du - Elt<T>::to_f32(x[c]) * mx) : du;
      static_cast<T *>(a.dx)[t * a.D + c] = Elt<T>::from_f32(dx);
      if (a.dres_out) static_cast<R *>(a.dres_out)[t * a.D + c] = Elt<R>::from_f32(d);
    }
    __syncthreads();
  }
}

// out[c] = the sum over the parts of partial[part][c], c < cols; the columns
// [k D, (k + 1) D) go to the k-th of up to three gradients.
__global__ __launch_bounds__(kNormThreads) void sum_parts_kernel(const float *partial, int parts, int cols, int D,
                                                                 float *o0, float *o1, float *o2) {
  const int c = blockIdx.x * kNormThreads + threadIdx.x;
  if (c >= cols) return;
  float s = 0.f;
  for (int p = 0; p < parts; ++p) s += partial[(size_t)p * cols + c];
  (c < D ? o0 : c < 2 * D ? o1 : o2)[c % D] = s;
}

static hipError_t sum_parts(const float *partial, int parts, int D, float *o0, float *o1, float *o2, hipStream_t s) {
  const int cols = D * (1 + (o1 != nullptr) + (o2 != nullptr));
  hipLaunchKernelGGL(sum_parts_kernel, dim3((cols + kNormThreads - 1) / kNormThreads), dim3(kNormThreads), 0, s, partial,
                     parts, cols, D, o0, o1, o2);
  return hipGetLastError();
}

// act(z) and its derivative.
__device__ __forceinline__ void activation(bool silu, float z, float &f, float &df) {
  const float s = sigmoid(z);
  f = silu ? z * s : s;
  df = silu ? s * (1.f + z * (1.f - s)) : s * (1.f - s);
}

template <typename T> __global__ __launch_bounds__(kNormThreads) void gate_norm_kernel(GateNormArgs a) {
  for (size_t row = blockIdx.x; row < (size_t)a.T * a.H; row += gridDim.x) {
  const size_t t = row / a.H;
  const int h = (int)(row % a.H);
  const T *o = static_cast<const T *>(a.o) + t * a.os + (size_t)h * a.d;
  const T *z = static_cast<const T *>(a.z) + t * a.zs + (size_t)h * a.d;
  float v[1] = {0.f};
  for (int c = threadIdx.x; c < a.d; c += kNormThreads) v[0] += Elt<T>::to_f32(o[c]) * Elt<T>::to_f32(o[c]);
  block_sums(v);
  const float r = 1.f / sqrtf(v[0] / (float)a.d + a.eps);
  for (int c = threadIdx.x; c < a.d; c += kNormThreads) {
    float f, df;
    activation(a.silu, Elt<T>::to_f32(z[c]), f, df);
    static_cast<T *>(a.y)[row * a.d + c] = Elt<T>::from_f32(Elt<T>::to_f32(o[c]) * r * a.w[c] * f);
  }
  }
}

template <typename T> __global__ __launch_bounds__(kNormThreads) void gate_norm_backward_kernel(GateNormArgs a) {
  float *pw = a.partial + (size_t)blockIdx.x * a.d;
  for (int i = threadIdx.x; i < a.d; i += kNormThreads) pw[i] = 0.f;
  __syncthreads();
  for (size_t row = blockIdx.x; row < (size_t)a.T * a.H; row += gridDim.x) {
    const size_t t = row / a.H, hd = (row % a.H) * a.d;
    const T *o = static_cast<const T *>(a.o) + t * a.os + hd, *z = static_cast<const T *>(a.z) + t * a.zs + hd;
    const T *dy = static_cast<const T *>(a.dy) + t * a.dys + hd;
    float v[2] = {0.f, 0.f};  // sums of o^2, o w dn
    for (int c = threadIdx.x; c < a.d; c += kNormThreads) {
      float f, df;
      activation(a.silu, Elt<T>::to_f32(z[c]), f, df);
      const float x = Elt<T>::to_f32(o[c]);
      v[0] += x * x;
      v[1] += x * a.w[c] * Elt<T>::to_f32(dy[c]) * f;
    }
    block_sums(v);
    const float r = 1.f / sqrtf(v[0] / (float)a.d + a.eps), m = r * r * v[1] / (float)a.d;
    for (int c = threadIdx.x; c < a.d; c += kNormThreads) {
      float f, df;
      activation(a.silu, Elt<T>::to_f32(z[c]), f, df);
      const float x = Elt<T>::to_f32(o[c]), g = Elt<T>::to_f32(dy[c]), dn = g * f;
      static_cast<T *>(a.dout)[row * a.d + c] = Elt<T>::from_f32(r * (a.w[c] * dn - x * m));
      static_cast<T *>(a.dz)[row * a.d + c] = Elt<T>::from_f32(g * x * r * a.w[c] * df);
      pw[c] += dn * x * r;
    }
    __syncthreads();
  }
}

int norm_parts(long rows, int cus) {
  const long most = 4L * (cus > 0 ? cus : 256);
  return (int)(rows < 1 ? 1 : rows < most ? rows : most);
}

#define HAGDN_NORM_TYPES(K, grid)                                                                          \
  do {                                                                                                     \
    if (!bf16) hipLaunchKernelGGL((K<float, float>), grid, dim3(kNormThreads), 0, s, a);                   \
    else if (res_bf16) hipLaunchKernelGGL((K<bf16_t, bf16_t>), grid, dim3(kNormThreads), 0, s, a);         \
    else hipLaunchKernelGGL((K<bf16_t, float>), grid, dim3(kNormThreads), 0, s, a);                        \
  } while (0)

hipError_t launch_add_norm(const AddNormArgs &a, bool bf16, bool res_bf16, hipStream_t s) {
  HAGDN_NORM_TYPES(add_norm_kernel, dim3(a.T < kMaxGrid ? a.T : kMaxGrid));
  return hipGetLastError();
}

hipError_t launch_add_norm_backward(const AddNormArgs &a, bool bf16, bool res_bf16, hipStream_t s) {
  HAGDN_NORM_TYPES(add_norm_backward_kernel, dim3(a.parts));
  hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : sum_parts(a.partial, a.parts, a.D, a.dw, a.dscale ? a.dscale : a.dpost,
                                         a.dscale ? a.dpost : nullptr, s);
}

hipError_t launch_gate_norm(const GateNormArgs &a, bool bf16, hipStream_t s) {
  const size_t rows = (size_t)a.T * a.H;
  const dim3 grid((unsigned)(rows < kMaxGrid ? rows : kMaxGrid));
  if (bf16) hipLaunchKernelGGL(gate_norm_kernel<bf16_t>, grid, dim3(kNormThreads), 0, s, a);
  else hipLaunchKernelGGL(gate_norm_kernel<float>, grid, dim3(kNormThreads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_gate_norm_backward(const GateNormArgs &a, bool bf16, hipStream_t s) {
  if (bf16) hipLaunchKernelGGL(gate_norm_backward_kernel<bf16_t>, dim3(a.parts), dim3(kNormThreads), 0, s, a);
  else hipLaunchKernelGGL(gate_norm_backward_kernel<float>, dim3(a.parts), dim3(kNormThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : sum_parts(a.partial, a.parts, a.d, a.dw, nullptr, nullptr, s);
}

}  // namespace hagdn

// k8_norms.hip -- the norms before and after a block, fused with the residual
// stream's scaled add (add_norm) and with the mixer's output gate (gate_norm),
// and their backward passes.  RMS norms: norm(v) = v rstd(v), rstd = (mean v^2 + eps)^-1/2.
//
// All are bound by HBM: some 10 to 25 operations an element against 6 to 20 bytes.  So
// every operand is loaded once, 16 bytes a lane, and a row stays in the registers of the
// lanes that share it from its loads to its stores.  A row of n 16-byte chunks has
// 16 to 1024 lanes (forward_rows): up to a wave each lane holds one chunk, then up to four
// per lane, so that rows to 2048 bf16 elements need no barrier at all; longer ones one
// barrier per sum.  The sums of the backward passes are taken together in one round: the
// second norm's, which depends on the first's result, is linear in it.
//
// The weights' gradients sum over rows.  Each lane adds up its own elements of all the
// rows it meets, a workgroup's row groups meet in LDS at the end, the workgroups' sums
// in a second kernel; every order is fixed, so the results repeat bit for bit.
#include "device.h"
#include "layer.h"

namespace hagdn {

// ------------------------------------------------------------------ row access
// VE neighbouring elements in fp32, loaded and stored as a vector at the element's
// alignment (a column slice may start anywhere).
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

template <typename T, int VE> struct Raw {  // VE elements as they lie in memory
  T v[VE];
  __device__ void load(const T *p) {
#pragma unroll
    for (int i = 0; i < VE; ++i) v[i] = p[i];
  }
  __device__ float get(int i) const { return Elt<T>::to_f32(v[i]); }
};
template <> struct Raw<bf16_t, 8> {
  u32x4 v;
  __device__ void load(const bf16_t *p) { v = *reinterpret_cast<const u32x4_any *>(p); }
  __device__ float get(int i) const { return __uint_as_float(i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16); }
};
template <> struct Raw<float, 4> {
  f32x4 v;
  __device__ void load(const float *p) { v = *reinterpret_cast<const f32x4_any *>(p); }
  __device__ float get(int i) const { return v[i]; }
};
template <> struct Raw<float, 8> {
  f32x4 v[2];
  __device__ void load(const float *p) {
    v[0] = *reinterpret_cast<const f32x4_any *>(p);
    v[1] = *reinterpret_cast<const f32x4_any *>(p + 4);
  }
  __device__ float get(int i) const { return v[i >> 2][i & 3]; }
};
template <int VE> __device__ __forceinline__ void store_vec(bf16_t *p, const float (&v)[VE]) {
  if constexpr (VE == 8) {
    u32x4_any u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = (uint32_t)f32_to_bf16(v[2 * i]) | (uint32_t)f32_to_bf16(v[2 * i + 1]) << 16;
    *reinterpret_cast<u32x4_any *>(p) = u;
  } else {
    *p = f32_to_bf16(v[0]);
  }
}
template <int VE> __device__ __forceinline__ void store_vec(float *p, const float (&v)[VE]) {
  if constexpr (VE == 1) {
    *p = v[0];
  } else {
#pragma unroll
    for (int i = 0; i < VE; i += 4) {
      f32x4_any u;
#pragma unroll
      for (int j = 0; j < 4; ++j) u[j] = v[i + j];
      *reinterpret_cast<f32x4_any *>(p + i) = u;
    }
  }
}

// A lane's chunk of rows of d elements (d >= VE): elements at .. at + VE - 1, of which
// the first `skip` belong to the lane before (the last chunk of a row is moved back to
// end with it) or, skip = VE, all of them (no chunk left).
template <int VE> struct Chunk {
  int at, skip;
  __device__ Chunk() {}
  __device__ Chunk(int e0, int d) {
    at = min(e0, d - VE);
    skip = min(e0 - at, VE);
  }
  template <typename T> __device__ Raw<T, VE> fetch(const T *row) const {
    Raw<T, VE> r;
    r.load(row + at);
    return r;
  }
  // In fp32; elements that are another lane's come as zeros.
  template <typename T> __device__ void open(const Raw<T, VE> &r, float (&v)[VE]) const {
#pragma unroll
    for (int j = 0; j < VE; ++j) v[j] = r.get(j);
    if (skip > 0) {
#pragma unroll
      for (int j = 0; j < VE; ++j) v[j] = j < skip ? 0.f : v[j];
    }
  }
  template <typename T> __device__ void load(const T *row, float (&v)[VE]) const { open(fetch(row), v); }
  template <typename T> __device__ void store(T *row, const float (&v)[VE]) const {
    if (skip == 0) {
      store_vec<VE>(row + at, v);
    } else {
#pragma unroll
      for (int j = 0; j < VE; ++j)
        if (j >= skip) row[at + j] = Elt<T>::from_f32(v[j]);
    }
  }
};

// ---------------------------------------------------------------------- row sums
// Sums over the LANES lanes of a row (lanes are a power of two); every lane gets them.
// Rows of more than a wave pass through LDS, in alternating buffers, so that a row's
// single barrier also guards the one before last.
template <int CTRL> __device__ __forceinline__ float dpp_add(float x) {
  return x + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xf, 0xf, true));
}
template <int LANES> __device__ __forceinline__ float lanes_sum(float x) {
  x = dpp_add<0xb1>(x);   // lanes 1, 0, 3, 2
  x = dpp_add<0x4e>(x);   // lanes 2, 3, 0, 1
  x = dpp_add<0x141>(x);  // 8 lanes mirrored
  x = dpp_add<0x140>(x);  // 16 lanes mirrored
  if constexpr (LANES >= 32) x += __shfl_xor(x, 16);
  if constexpr (LANES >= 64) x += __shfl_xor(x, 32);
  return x;
}
template <int LANES> constexpr int row_threads() { return LANES > 256 ? LANES : 256; }  // of a workgroup
template <int LANES, int K> struct RowSums {
  static constexpr int kWaves = LANES / 64;
  float (*buf)[row_threads<LANES>() / 64][K];  // [2]
  int turn = 0;
  __device__ void operator()(float (&v)[K]) {
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = lanes_sum<LANES>(v[k]);
    if constexpr (kWaves > 1) {
      const int wave = threadIdx.x >> 6;
      if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) buf[turn][wave][k] = v[k];
      __syncthreads();
#pragma unroll
      for (int k = 0; k < K; ++k) {
        v[k] = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v[k] += buf[turn][threadIdx.x / LANES * kWaves + w][k];
      }
      turn ^= 1;
    }
  }
};
#define HAGDN_ROW_SUMS(name, LANES, K)                              \
  __shared__ float name##_buf[2][row_threads<LANES>() / 64][K];     \
  RowSums<LANES, K> name{name##_buf}

__device__ __forceinline__ float rstd(float sum, float inv, float eps) { return 1.f / sqrtf(sum * inv + eps); }

// ------------------------------------------------------------------ partial sums
// Adds a workgroup's row groups' sums in LDS and writes them to out[0 .. d): lane lr of
// the GROUPS groups of LANES lanes holds acc[C][VE] of its chunks.
template <int VE, int C, int LANES, int GROUPS>
__device__ __forceinline__ void write_partial(const float (&acc)[C][VE], const Chunk<VE> (&ch)[C], float *out,
                                              float (&lds)[GROUPS > 1 ? GROUPS * LANES : 1]) {
  const int group = threadIdx.x / LANES, lr = threadIdx.x % LANES;
#pragma unroll
  for (int j = 0; j < C; ++j)
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      float v = acc[j][e];
      if constexpr (GROUPS > 1) {
        __syncthreads();
        lds[threadIdx.x] = v;
        __syncthreads();
        if (group == 0) {
          v = 0.f;
#pragma unroll
          for (int g = 0; g < GROUPS; ++g) v += lds[g * LANES + lr];
        }
      }
      if (group == 0 && e >= ch[j].skip) out[ch[j].at + e] = v;
    }
}

constexpr int kSumThreads = 1024, kSumCols = 16;

// The sum over the parts of partial[part][c], c < cols; the columns [k D, (k + 1) D) go
// to the k-th of up to three gradients.  16 columns a workgroup, 64 lanes to each.
__global__ __launch_bounds__(kSumThreads) void sum_parts_kernel(const float *partial, int parts, int cols, int D, float *o0,
                                                                float *o1, float *o2) {
  __shared__ float s[kSumThreads / 64][kSumCols];
  const int c = blockIdx.x * kSumCols + threadIdx.x % kSumCols;
  float v = 0.f;
  if (c < cols)
    for (int p = threadIdx.x / kSumCols; p < parts; p += kSumThreads / kSumCols) v += partial[(size_t)p * cols + c];
  v += __shfl_xor(v, 16);
  v += __shfl_xor(v, 32);
  if ((threadIdx.x & 63) < kSumCols) s[threadIdx.x >> 6][threadIdx.x & 63] = v;
  __syncthreads();
  if (threadIdx.x >= kSumCols || c >= cols) return;
  v = 0.f;
#pragma unroll
  for (int w = 0; w < kSumThreads / 64; ++w) v += s[w][threadIdx.x];
  (c < D ? o0 : c < 2 * D ? o1 : o2)[c % D] = v;
}

static hipError_t sum_parts(const float *partial, int parts, int D, float *o0, float *o1, float *o2, hipStream_t s) {
  const int cols = D * (1 + (o1 != nullptr) + (o2 != nullptr));
  hipLaunchKernelGGL(sum_parts_kernel, dim3((cols + kSumCols - 1) / kSumCols), dim3(kSumThreads), 0, s, partial, parts, cols,
                     D, o0, o1, o2);
  return hipGetLastError();
}

// ---------------------------------------------------------------------- add_norm
template <typename T, typename R, int VE, int LANES, int C>
__global__ __launch_bounds__(row_threads<LANES>()) void add_norm_kernel(AddNormArgs a) {
  constexpr int kRows = row_threads<LANES>() / LANES;
  HAGDN_ROW_SUMS(sums, LANES, 1);
  const float inv = 1.f / (float)a.D;
  Chunk<VE> ch[C];
#pragma unroll
  for (int j = 0; j < C; ++j) ch[j] = Chunk<VE>((j * LANES + threadIdx.x % LANES) * VE, a.D);
  for (long row = (long)blockIdx.x * kRows + threadIdx.x / LANES; row < a.T; row += (long)gridDim.x * kRows) {
    const T *x = static_cast<const T *>(a.x) + row * a.xs;
    float u[C][VE], r[C][VE], w[VE], v[1];
#pragma unroll
    for (int j = 0; j < C; ++j) {
      ch[j].load(x, u[j]);
      if (a.res) {
        ch[j].load(static_cast<const R *>(a.res) + row * a.rs, r[j]);
      } else {
#pragma unroll
        for (int e = 0; e < VE; ++e) r[j][e] = 0.f;
      }
    }
    if (a.post) {
      v[0] = 0.f;
#pragma unroll
      for (int j = 0; j < C; ++j)
#pragma unroll
        for (int e = 0; e < VE; ++e) v[0] += u[j][e] * u[j][e];
      sums(v);
      const float rx = rstd(v[0], inv, a.eps);
#pragma unroll
      for (int j = 0; j < C; ++j) {
        ch[j].load(a.post, w);
#pragma unroll
        for (int e = 0; e < VE; ++e) u[j][e] *= rx * w[e];
      }
    }
    v[0] = 0.f;
#pragma unroll
    for (int j = 0; j < C; ++j) {
      if (a.scale_vec) {
        ch[j].load(a.scale_vec, w);
      } else {
#pragma unroll
        for (int e = 0; e < VE; ++e) w[e] = a.scale;
      }
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        r[j][e] += w[e] * u[j][e];
        v[0] += r[j][e] * r[j][e];
      }
    }
    sums(v);
    const float rr = rstd(v[0], inv, a.eps);
#pragma unroll
    for (int j = 0; j < C; ++j) {
      if (a.res_out) ch[j].store(static_cast<R *>(a.res_out) + row * a.D, r[j]);
      ch[j].load(a.w, w);
#pragma unroll
      for (int e = 0; e < VE; ++e) r[j][e] *= rr * w[e];
      ch[j].store(static_cast<T *>(a.y) + row * a.D, r[j]);
    }
  }
}

// With D the gradient of r', m = mean(r' w dy) and q = mean(x post s D):
//   D = dres + rr (w dy - r' rr^2 m),   dx = rx (post s D - x rx^2 q).
// q is taken from D's three terms' own sums, so that one round of sums serves the row.
// READS_X: a scale vector or post_weight is there.
template <typename T, typename R, int VE, int LANES, int C, bool READS_X>
__global__ __launch_bounds__(row_threads<LANES>(), 4) void add_norm_backward_kernel(AddNormArgs a) {
  constexpr int kRows = row_threads<LANES>() / LANES, kSums = READS_X ? 6 : 2;
  HAGDN_ROW_SUMS(sums, LANES, kSums);
  __shared__ float lds[kRows > 1 ? kRows * LANES : 1];
  const float inv = 1.f / (float)a.D;
  Chunk<VE> ch[C];
  float aw[C][VE], as[C][VE], ap[C][VE];
#pragma unroll
  for (int j = 0; j < C; ++j) {
    ch[j] = Chunk<VE>((j * LANES + threadIdx.x % LANES) * VE, a.D);
#pragma unroll
    for (int e = 0; e < VE; ++e) aw[j][e] = as[j][e] = ap[j][e] = 0.f;
  }
  // the loop's bounds are those of the workgroup's first row: all lanes take every turn.
  // A row's operands are fetched while the one before is worked on.
  const long step = (long)gridDim.x * kRows, own = threadIdx.x / LANES;
  Raw<R, VE> fr[C], fd[C];
  Raw<T, VE> fg[C], fx[C];
  auto fetch = [&](long row) {
    row = min(row, (long)a.T - 1);
#pragma unroll
    for (int j = 0; j < C; ++j) {
      fr[j] = ch[j].fetch(static_cast<const R *>(a.res) + row * a.rs);
      fg[j] = ch[j].fetch(static_cast<const T *>(a.dy) + row * a.dys);
      if (a.dres) fd[j] = ch[j].fetch(static_cast<const R *>(a.dres) + row * a.drs);
      if constexpr (READS_X) fx[j] = ch[j].fetch(static_cast<const T *>(a.x) + row * a.xs);
    }
  };
  if (a.T > 0) fetch((long)blockIdx.x * kRows + own);
  for (long first = (long)blockIdx.x * kRows; first < a.T; first += step) {
    const long row = first + own;
    const bool live = row < a.T;
    float x[C][VE], r[C][VE], g[C][VE], d[C][VE];  // x, r', dy then w dy, dres then D
    float v[kSums] = {};
#pragma unroll
    for (int j = 0; j < C; ++j) {
      ch[j].open(fr[j], r[j]);
      ch[j].open(fg[j], g[j]);
      if (a.dres) ch[j].open(fd[j], d[j]);
      if constexpr (READS_X) ch[j].open(fx[j], x[j]);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        if (!a.dres) d[j][e] = 0.f;
        if (!live) g[j][e] = d[j][e] = 0.f;
      }
    }
    if (first + step < a.T) fetch(row + step);
#pragma unroll
    for (int j = 0; j < C; ++j) {
      float w[VE], s[VE], p[VE];
      ch[j].load(a.w, w);
      if constexpr (READS_X) {
        if (a.scale_vec) ch[j].load(a.scale_vec, s);
        if (a.post) ch[j].load(a.post, p);
      }
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float wg = w[e] * g[j][e];
        v[0] += r[j][e] * r[j][e];
        v[1] += r[j][e] * wg;
        if constexpr (READS_X) {
          const float ps = (a.post ? p[e] : 1.f) * (a.scale_vec ? s[e] : a.scale), xs = x[j][e] * ps;
          v[2] += x[j][e] * x[j][e];
          v[3] += xs * d[j][e];
          v[4] += xs * wg;
          v[5] += xs * r[j][e];
        }
      }
    }
    sums(v);
    const float rr = rstd(v[0], inv, a.eps), m = rr * rr * rr * v[1] * inv;
    float rx = 1.f, q = 0.f;
    if constexpr (READS_X) {
      if (a.post) {
        rx = rstd(v[2], inv, a.eps);
        q = rx * rx * (v[3] + rr * v[4] - m * v[5]) * inv;
      }
    }
#pragma unroll
    for (int j = 0; j < C; ++j) {
      float w[VE], s[VE], p[VE];
      ch[j].load(a.w, w);
      if constexpr (READS_X) {
        if (a.scale_vec) ch[j].load(a.scale_vec, s);
        if (a.post) ch[j].load(a.post, p);
      }
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        aw[j][e] += g[j][e] * (r[j][e] * rr);
        d[j][e] += rr * (w[e] * g[j][e]) - m * r[j][e];
        if constexpr (READS_X) {
          const float xn = x[j][e] * rx, se = a.scale_vec ? s[e] : a.scale;
          const float du = se * d[j][e];
          if (live) {
            as[j][e] += d[j][e] * xn * (a.post ? p[e] : 1.f);
            ap[j][e] += du * xn;
          }
          x[j][e] = a.post ? rx * (p[e] * du - x[j][e] * q) : du;
        } else {
          g[j][e] = a.scale * d[j][e];
        }
      }
      if (live) {
        if (a.dres_out) ch[j].store(static_cast<R *>(a.dres_out) + row * a.D, d[j]);
        ch[j].store(static_cast<T *>(a.dx) + row * a.D, READS_X ? x[j] : g[j]);
      }
    }
  }
  const int outs = 1 + (a.dscale != nullptr) + (a.dpost != nullptr);
  float *out = a.partial + (size_t)blockIdx.x * outs * a.D;
  write_partial<VE, C, LANES, kRows>(aw, ch, out, lds);
  if constexpr (READS_X) {
    if (a.dscale) write_partial<VE, C, LANES, kRows>(as, ch, out += a.D, lds);
    if (a.dpost) write_partial<VE, C, LANES, kRows>(ap, ch, out += a.D, lds);
  }
}

// --------------------------------------------------------------------- gate_norm
// act(z) and its derivative, from e^-z: 1 / (1 + e^-z) is 0 where that overflows.
__device__ __forceinline__ void activation(bool silu, float z, float &f, float &df) {
  const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504f));
  f = silu ? z * s : s;
  df = silu ? s * (1.f + z * (1.f - s)) : s * (1.f - s);
}

// Where a row (token, head) of a tensor [T, H, d] with a token stride begins.
__device__ __forceinline__ long head_row(uint32_t row, int H, int d, long stride) {
  if (stride == (long)H * d) return (long)row * d;
  const uint32_t t = row / (uint32_t)H;
  return (long)t * stride + (long)(row - t * (uint32_t)H) * d;
}

template <typename T, int VE, int LANES, int C>
__global__ __launch_bounds__(row_threads<LANES>()) void gate_norm_kernel(GateNormArgs a) {
  constexpr int kRows = row_threads<LANES>() / LANES;
  HAGDN_ROW_SUMS(sums, LANES, 1);
  const float inv = 1.f / (float)a.d;
  const long rows = (long)a.T * a.H;
  Chunk<VE> ch[C];
#pragma unroll
  for (int j = 0; j < C; ++j) ch[j] = Chunk<VE>((j * LANES + threadIdx.x % LANES) * VE, a.d);
  for (long row = (long)blockIdx.x * kRows + threadIdx.x / LANES; row < rows; row += (long)gridDim.x * kRows) {
    const T *o = static_cast<const T *>(a.o) + head_row((uint32_t)row, a.H, a.d, a.os);
    const T *zr = static_cast<const T *>(a.z) + head_row((uint32_t)row, a.H, a.d, a.zs);
    float x[C][VE], z[C][VE], w[VE], v[1] = {0.f};
#pragma unroll
    for (int j = 0; j < C; ++j) {
      ch[j].load(o, x[j]);
      ch[j].load(zr, z[j]);
    }
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
      for (int e = 0; e < VE; ++e) v[0] += x[j][e] * x[j][e];
    sums(v);
    const float r = rstd(v[0], inv, a.eps);
#pragma unroll
    for (int j = 0; j < C; ++j) {
      ch[j].load(a.w, w);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        float f, df;
        activation(a.silu, z[j][e], f, df);
        x[j][e] *= r * w[e] * f;
      }
      ch[j].store(static_cast<T *>(a.y) + row * a.d, x[j]);
    }
  }
}

template <typename T, int VE, int LANES, int C>
__global__ __launch_bounds__(row_threads<LANES>(), 4) void gate_norm_backward_kernel(GateNormArgs a) {
  constexpr int kRows = row_threads<LANES>() / LANES;
  HAGDN_ROW_SUMS(sums, LANES, 2);
  __shared__ float lds[kRows > 1 ? kRows * LANES : 1];
  const float inv = 1.f / (float)a.d;
  const long rows = (long)a.T * a.H;
  Chunk<VE> ch[C];
  float aw[C][VE];
#pragma unroll
  for (int j = 0; j < C; ++j) {
    ch[j] = Chunk<VE>((j * LANES + threadIdx.x % LANES) * VE, a.d);
#pragma unroll
    for (int e = 0; e < VE; ++e) aw[j][e] = 0.f;
  }
  // the loop's bounds are those of the workgroup's first row: all lanes take every turn.
  // A row's operands are fetched while the one before is worked on.
  const long step = (long)gridDim.x * kRows, own = threadIdx.x / LANES;
  Raw<T, VE> fx[C], fz[C], fg[C];
  auto fetch = [&](long row) {
    const uint32_t r = (uint32_t)min(row, rows - 1);
    const T *o = static_cast<const T *>(a.o) + head_row(r, a.H, a.d, a.os);
    const T *z = static_cast<const T *>(a.z) + head_row(r, a.H, a.d, a.zs);
    const T *dy = static_cast<const T *>(a.dy) + head_row(r, a.H, a.d, a.dys);
#pragma unroll
    for (int j = 0; j < C; ++j) {
      fx[j] = ch[j].fetch(o);
      fz[j] = ch[j].fetch(z);
      fg[j] = ch[j].fetch(dy);
    }
  };
  if (rows > 0) fetch((long)blockIdx.x * kRows + own);
  for (long first = (long)blockIdx.x * kRows; first < rows; first += step) {
    const long row = first + own;
    const bool live = row < rows;
    float x[C][VE], z[C][VE], g[C][VE], v[2] = {0.f, 0.f};  // o, z then dz's factor, dy then dn
#pragma unroll
    for (int j = 0; j < C; ++j) {
      ch[j].open(fx[j], x[j]);
      ch[j].open(fz[j], z[j]);
      ch[j].open(fg[j], g[j]);
    }
    if (first + step < rows) fetch(row + step);
#pragma unroll
    for (int j = 0; j < C; ++j) {
      float w[VE];
      ch[j].load(a.w, w);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        float f, df;
        activation(a.silu, z[j][e], f, df);
        z[j][e] = g[j][e] * w[e] * df;
        g[j][e] = live ? g[j][e] * f : 0.f;
        v[0] += x[j][e] * x[j][e];
        v[1] += x[j][e] * w[e] * g[j][e];
      }
    }
    sums(v);
    const float r = rstd(v[0], inv, a.eps), m = r * r * r * v[1] * inv;
#pragma unroll
    for (int j = 0; j < C; ++j) {
      float w[VE], dn[VE];
      ch[j].load(a.w, w);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float n = x[j][e] * r;
        aw[j][e] += g[j][e] * n;
        z[j][e] *= n;
        dn[e] = r * (w[e] * g[j][e]) - m * x[j][e];
      }
      if (live) {
        ch[j].store(static_cast<T *>(a.dout) + row * a.d, dn);
        ch[j].store(static_cast<T *>(a.dz) + row * a.d, z[j]);
      }
    }
  }
  write_partial<VE, C, LANES, kRows>(aw, ch, a.partial + (size_t)blockIdx.x * a.d, lds);
}

// -------------------------------------------------------------------- launches
// The lanes of a row of d elements and the chunks of each, K::go<VE, LANES, C>; V is the
// vector's elements (16 bytes of the operands' type).
template <int V, typename K> static hipError_t forward_rows(int d, const K &k) {
  const int n = (d + V - 1) / V;
  if (d < V) return k.template go<1, 16, 1>();
  if (n <= 16) return k.template go<V, 16, 1>();
  if (n <= 32) return k.template go<V, 32, 1>();
  if (n <= 64) return k.template go<V, 64, 1>();
  if (n <= 128) return k.template go<V, 64, 2>();
  if (n <= 256) return k.template go<V, 64, 4>();
  if (n <= 512) return k.template go<V, 256, 2>();
  if (n <= 1024) return k.template go<V, 256, 4>();
  if constexpr (V == 4)
    if (n > 2048) return k.template go<V, 1024, 4>();
  return k.template go<V, 1024, 2>();
}
// Backward passes keep sums of their own beside the row, so eight elements a lane (of the
// widest rows 16) and a barrier a row beyond 512 elements.
template <int V, typename K> static hipError_t backward_rows(int d, const K &k) {
  constexpr int C = 8 / V;
  if (d < V) return k.template go<1, 16, 1>();
  if (d <= 128) return k.template go<V, 16, C>();
  if (d <= 256) return k.template go<V, 32, C>();
  if (d <= 512) return k.template go<V, 64, C>();
  if (d <= 1024) return k.template go<V, 128, C>();
  if (d <= 2048) return k.template go<V, 256, C>();
  if (d <= 4096) return k.template go<V, 512, C>();
  if (d <= 8192) return k.template go<V, 1024, C>();
  return k.template go<V, 1024, 2 * C>();
}

// Workgroups for `rows` rows, `per` of them each at a time; forward passes.
static unsigned norm_grid(long rows, int per) {
  const long groups = (rows + per - 1) / per;
  return (unsigned)(groups < (1l << 20) ? groups : 1l << 20);
}

template <typename T, typename R> struct AddNorm {
  const AddNormArgs &a;
  hipStream_t s;
  template <int VE, int LANES, int C> hipError_t go() const {
    hipLaunchKernelGGL((add_norm_kernel<T, R, VE, LANES, C>), dim3(norm_grid(a.T, row_threads<LANES>() / LANES)),
                       dim3(row_threads<LANES>()), 0, s, a);
    return hipGetLastError();
  }
};
template <typename T, typename R> struct AddNormBackward {
  const AddNormArgs &a;
  hipStream_t s;
  template <int VE, int LANES, int C> hipError_t go() const {
    const dim3 grid(a.parts), block(row_threads<LANES>());
    if (a.post || a.scale_vec) hipLaunchKernelGGL((add_norm_backward_kernel<T, R, VE, LANES, C, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((add_norm_backward_kernel<T, R, VE, LANES, C, false>), grid, block, 0, s, a);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : sum_parts(a.partial, a.parts, a.D, a.dw, a.dscale ? a.dscale : a.dpost,
                                           a.dscale ? a.dpost : nullptr, s);
  }
};
template <typename T> struct GateNorm {
  const GateNormArgs &a;
  hipStream_t s;
  template <int VE, int LANES, int C> hipError_t go() const {
    hipLaunchKernelGGL((gate_norm_kernel<T, VE, LANES, C>), dim3(norm_grid((long)a.T * a.H, row_threads<LANES>() / LANES)),
                       dim3(row_threads<LANES>()), 0, s, a);
    return hipGetLastError();
  }
};
template <typename T> struct GateNormBackward {
  const GateNormArgs &a;
  hipStream_t s;
  template <int VE, int LANES, int C> hipError_t go() const {
    hipLaunchKernelGGL((gate_norm_backward_kernel<T, VE, LANES, C>), dim3(a.parts), dim3(row_threads<LANES>()), 0, s, a);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : sum_parts(a.partial, a.parts, a.d, a.dw, nullptr, nullptr, s);
  }
};

hipError_t launch_add_norm(const AddNormArgs &a, bool bf16, bool res_bf16, hipStream_t s) {
  if (!bf16) return forward_rows<4>(a.D, AddNorm<float, float>{a, s});
  return res_bf16 ? forward_rows<8>(a.D, AddNorm<bf16_t, bf16_t>{a, s}) : forward_rows<8>(a.D, AddNorm<bf16_t, float>{a, s});
}

hipError_t launch_add_norm_backward(const AddNormArgs &a, bool bf16, bool res_bf16, hipStream_t s) {
  if (!bf16) return backward_rows<4>(a.D, AddNormBackward<float, float>{a, s});
  return res_bf16 ? backward_rows<8>(a.D, AddNormBackward<bf16_t, bf16_t>{a, s})
                  : backward_rows<8>(a.D, AddNormBackward<bf16_t, float>{a, s});
}

hipError_t launch_gate_norm(const GateNormArgs &a, bool bf16, hipStream_t s) {
  return bf16 ? forward_rows<8>(a.d, GateNorm<bf16_t>{a, s}) : forward_rows<4>(a.d, GateNorm<float>{a, s});
}

hipError_t launch_gate_norm_backward(const GateNormArgs &a, bool bf16, hipStream_t s) {
  return bf16 ? backward_rows<8>(a.d, GateNormBackward<bf16_t>{a, s}) : backward_rows<4>(a.d, GateNormBackward<float>{a, s});
}

}  // namespace hagdn

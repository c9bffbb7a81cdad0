// k8_norms.hip -- the norms before and after a block, fused with the residual
// stream's scaled add (add_norm) and with the mixer's output gate (gate_norm),
// and their backward passes.  RMS norms: norm(v) = v rstd(v), rstd = (mean v^2 + eps)^-1/2.
//
// All are bound by HBM: some 10 to 25 operations an element against 6 to 20 bytes.  So
// every operand is loaded once, 16 bytes a lane, and a row stays in the registers of the
// lanes that share it from its loads to its stores.  A row of n 16-byte chunks has
// 8 to 1024 lanes (norm_rows); those of more than a wave meet in LDS, with one barrier a
// round of sums.  The sums of the backward passes are taken together in one round: the
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
  __device__ void clear(int i) { v[i] = T(0); }
  __device__ void keep_packed() {}
};
template <> struct Raw<bf16_t, 8> {
  u32x4 v;
  __device__ void load(const bf16_t *p) { v = *reinterpret_cast<const u32x4_any *>(p); }
  __device__ float get(int i) const { return __uint_as_float(i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16); }
  __device__ void clear(int i) { v[i >> 1] &= i & 1 ? 0x0000ffffu : 0xffff0000u; }
  // Makes the compiler unpack the elements anew from here on rather than hold them in
  // fp32, in twice the registers, since their last use.
  __device__ void keep_packed() {
#ifdef __HIP_DEVICE_COMPILE__
    asm("" : "+v"(v));
#endif
  }
};
template <> struct Raw<float, 4> {
  f32x4 v;
  __device__ void load(const float *p) { v = *reinterpret_cast<const f32x4_any *>(p); }
  __device__ float get(int i) const { return v[i]; }
  __device__ void clear(int i) { v[i] = 0.f; }
  __device__ void keep_packed() {}
};
template <> struct Raw<float, 8> {
  f32x4 v[2];
  __device__ void load(const float *p) {
    v[0] = *reinterpret_cast<const f32x4_any *>(p);
    v[1] = *reinterpret_cast<const f32x4_any *>(p + 4);
  }
  __device__ float get(int i) const { return v[i >> 2][i & 3]; }
  __device__ void clear(int i) { v[i >> 2][i & 3] = 0.f; }
  __device__ void keep_packed() {}
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
  template <typename T> __device__ void fetch(const T *row, Raw<T, VE> &r) const { r.load(row + at); }
  // Clears the elements that are another lane's (those before `skip`; n = VE: all).
  template <typename T> __device__ static void clear(Raw<T, VE> &r, int n) {
    if (n > 0) {
#pragma unroll
      for (int j = 0; j < VE; ++j)
        if (j < n) r.clear(j);
    }
  }
  template <typename T> __device__ void load(const T *row, float (&v)[VE]) const {
    Raw<T, VE> r;
    fetch(row, r);
    clear(r, skip);
#pragma unroll
    for (int j = 0; j < VE; ++j) v[j] = r.get(j);
  }
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
  x = dpp_add<0xb1>(x);                             // lanes 1, 0, 3, 2
  if constexpr (LANES >= 4) x = dpp_add<0x4e>(x);   // lanes 2, 3, 0, 1
  if constexpr (LANES >= 8) x = dpp_add<0x141>(x);  // 8 lanes mirrored
  if constexpr (LANES >= 16) x = dpp_add<0x140>(x);  // 16 lanes mirrored
  if constexpr (LANES >= 32) x += __shfl_xor(x, 16);
  if constexpr (LANES >= 64) x += __shfl_xor(x, 32);
  return x;
}
// THREADS: of the workgroup, whose rows all take their barriers together.
template <int LANES, int THREADS, int K> struct RowSums {
  static constexpr int kWaves = LANES / 64;
  float (*buf)[THREADS / 64][K];  // [2]
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
      const int first = threadIdx.x / LANES * kWaves;
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] = lanes_sum<kWaves>(buf[turn][first + threadIdx.x % kWaves][k]);
      turn ^= 1;
    }
  }
};
#define HAGDN_ROW_SUMS(name, LANES, THREADS, K)           \
  __shared__ float name##_buf[2][(THREADS) / 64][K];      \
  RowSums<LANES, THREADS, K> name{name##_buf}

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

// Threads of a workgroup: rows of up to a wave need no barrier, and short workgroups end
// apart; in the backward passes more rows together mean fewer partial sums.
template <int LANES> constexpr int forward_threads() { return LANES > 256 ? LANES : 256; }
template <int LANES> constexpr int backward_threads() { return LANES > 512 ? LANES : 512; }
// Rows that a group of lanes takes through one round of sums in add_norm's backward: two,
// where a row's way through its waves is long and both rows' operands are bf16 (8192 rows
// of 2048 39 us against 41, with both vectors 49 against 51; 500 rows 14 against 16).  A
// stream in fp32 loses by it (55 against 53, 66 against 64), all in fp32 spills (58
// against 45); within one wave, up to 512 values a row, it makes no difference.
template <typename T, typename R, int LANES> constexpr int rows_per_turn() {
  return sizeof(T) == 2 && sizeof(R) == 2 && LANES >= 128 && LANES <= 512 ? 2 : 1;
}

// ---------------------------------------------------------------------- add_norm
// One read of x and the stream, one write of y and the stream.  32768 rows of 2048 in
// bf16 95 us, 5.6 TB/s; 4096 of them 16 us, with the stream in fp32 17; one row 2.1 us.
template <typename T, typename R, int VE, int LANES, int C>
__global__ __launch_bounds__(forward_threads<LANES>()) void add_norm_kernel(AddNormArgs a) {
  constexpr int kThreads = forward_threads<LANES>(), kRows = kThreads / LANES;
  HAGDN_ROW_SUMS(sums, LANES, kThreads, 1);
  const float inv = 1.f / (float)a.D;
  Chunk<VE> ch[C];
#pragma unroll
  for (int j = 0; j < C; ++j) ch[j] = Chunk<VE>((j * LANES + threadIdx.x % LANES) * VE, a.D);
  // the loop's bounds are those of the workgroup's first row: all lanes take every turn
  for (long first = (long)blockIdx.x * kRows; first < a.T; first += (long)gridDim.x * kRows) {
    const bool live = first + threadIdx.x / LANES < a.T;
    const long row = live ? first + threadIdx.x / LANES : a.T - 1;
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
      if (a.res_out && live) ch[j].store(static_cast<R *>(a.res_out) + row * a.D, r[j]);
      ch[j].load(a.w, w);
#pragma unroll
      for (int e = 0; e < VE; ++e) r[j][e] *= rr * w[e];
      if (live) ch[j].store(static_cast<T *>(a.y) + row * a.D, r[j]);
    }
  }
}

// With D the gradient of r', n = r' rr and xn = x rx the normed rows:
//   D = dres + rr (w dy - n m),    m = mean(n w dy),
//   dx = rx (post s D - xn q),     q = mean(xn post s D).
// No power of rr or rx is formed by itself, which would leave fp32's range long before
// the results do.  q is taken from D's three terms' own sums, so that one round of sums
// serves the row.
// The operands stay as they were loaded (bf16 ones two to a register), the weights in
// registers for all of the workgroup's rows.  READS_X: a scale vector or post_weight is
// there.  8192 rows of 2048 in bf16 with both 48 us, 4.2 TB/s, of which 5 the sum over the
// workgroups; without them 38 us, 4.4 TB/s.  2000 rows of 8192 68 us with both, 44 without;
// of 16384, where a lane has two chunks and 1024 lanes leave it 128 registers, 400 (half a
// KiB a lane spilled) and 82.  Bound by the rows' way through their sums and barrier, which
// eight waves a CU overlap in part: at 8192 x 2048 sixteen, which spill, took 98 us; with one
// row a turn 51, and the operands of two or three rows fetched ahead no less.
template <typename T, typename R, int VE, int LANES, int C, bool READS_X>
__global__ __launch_bounds__(backward_threads<LANES>(),
                             LANES > 512 || (!READS_X && rows_per_turn<T, R, LANES>() == 1) ? 4 : 2)
void add_norm_backward_kernel(AddNormArgs a) {
  constexpr int kThreads = backward_threads<LANES>(), kRows = kThreads / LANES, kSums = READS_X ? 6 : 2;
  constexpr int P = rows_per_turn<T, R, LANES>();
  HAGDN_ROW_SUMS(sums, LANES, kThreads, P * kSums);
  __shared__ float lds[kRows > 1 ? kRows * LANES : 1];
  const float inv = 1.f / (float)a.D;
  Chunk<VE> ch[C];
  float aw[C][VE], as[C][VE], ap[C][VE];  // the weights' gradients
  float w[C][VE], s[C][VE], post[C][VE];  // weight, scale, post_weight
#pragma unroll
  for (int j = 0; j < C; ++j) {
    ch[j] = Chunk<VE>((j * LANES + threadIdx.x % LANES) * VE, a.D);
#pragma unroll
    for (int e = 0; e < VE; ++e) aw[j][e] = as[j][e] = ap[j][e] = 0.f;
  }
#pragma unroll
  for (int j = 0; j < C; ++j) {
    ch[j].load(a.w, w[j]);
#pragma unroll
    for (int e = 0; e < VE; ++e) s[j][e] = a.scale, post[j][e] = 1.f;
    if (READS_X && a.scale_vec) ch[j].load(a.scale_vec, s[j]);
    if (READS_X && a.post) ch[j].load(a.post, post[j]);
  }
  // the loop's bounds are those of the workgroup's first row: all lanes take every turn.
  // The next turn's operands are fetched while one is worked on.
  const long step = (long)gridDim.x * kRows * P, own = threadIdx.x / LANES;
  Raw<R, VE> nr[P][C], nd[P][C];
  Raw<T, VE> ng[P][C], nx[P][C];
  auto fetch = [&](long first) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const long row = min(first + p * kRows + own, (long)a.T - 1);
#pragma unroll
      for (int j = 0; j < C; ++j) {
        ch[j].fetch(static_cast<const R *>(a.res) + row * a.rs, nr[p][j]);
        ch[j].fetch(static_cast<const T *>(a.dy) + row * a.dys, ng[p][j]);
        if (a.dres) ch[j].fetch(static_cast<const R *>(a.dres) + row * a.drs, nd[p][j]);
        if constexpr (READS_X) ch[j].fetch(static_cast<const T *>(a.x) + row * a.xs, nx[p][j]);
      }
    }
  };
  if (a.T > 0) fetch((long)blockIdx.x * kRows * P);
  for (long first = (long)blockIdx.x * kRows * P; first < a.T; first += step) {
    Raw<R, VE> r[P][C], d[P][C];  // r', dres
    Raw<T, VE> g[P][C], x[P][C];  // dy, x
    float v[P * kSums] = {};
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const bool live = first + p * kRows + own < a.T;
#pragma unroll
      for (int j = 0; j < C; ++j) {
        r[p][j] = nr[p][j], g[p][j] = ng[p][j], d[p][j] = nd[p][j];
        if constexpr (READS_X) x[p][j] = nx[p][j];
        Chunk<VE>::clear(r[p][j], ch[j].skip);
        if constexpr (READS_X) Chunk<VE>::clear(x[p][j], ch[j].skip);
        Chunk<VE>::clear(g[p][j], live ? ch[j].skip : VE);  // a row past the end adds nothing
        Chunk<VE>::clear(d[p][j], live && a.dres ? ch[j].skip : VE);
      }
    }
    if (first + step < a.T) fetch(first + step);
#pragma unroll
    for (int p = 0; p < P; ++p) {
      float *s6 = v + p * kSums;
#pragma unroll
      for (int j = 0; j < C; ++j)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const float re = r[p][j].get(e), wg = w[j][e] * g[p][j].get(e);
          s6[0] += re * re;
          s6[1] += re * wg;
          if constexpr (READS_X) {
            const float xe = x[p][j].get(e), xs = xe * (post[j][e] * s[j][e]);
            s6[2] += xe * xe;
            s6[3] += xs * d[p][j].get(e);
            s6[4] += xs * wg;
            s6[5] += xs * re;
          }
        }
    }
    sums(v);
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const long row = first + p * kRows + own;
      const float *s6 = v + p * kSums;
      const float rr = rstd(s6[0], inv, a.eps), m = rr * s6[1] * inv;
      float rx = 1.f, q = 0.f;
      if constexpr (READS_X) {
        if (a.post) {
          rx = rstd(s6[2], inv, a.eps);
          q = rx * (s6[3] + rr * (s6[4] - m * (rr * s6[5]))) * inv;
        }
      }
#pragma unroll
      for (int j = 0; j < C; ++j) {
        float out[VE], dx[VE];
        r[p][j].keep_packed();
        g[p][j].keep_packed();
        d[p][j].keep_packed();
        if constexpr (READS_X) x[p][j].keep_packed();
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const float n = r[p][j].get(e) * rr, ge = g[p][j].get(e);
          aw[j][e] += ge * n;
          out[e] = d[p][j].get(e) + rr * (w[j][e] * ge - m * n);
          const float du = s[j][e] * out[e];
          if constexpr (READS_X) {
            const float xn = x[p][j].get(e) * rx;
            as[j][e] += out[e] * xn * post[j][e];
            ap[j][e] += du * xn;
            dx[e] = rx * (post[j][e] * du - xn * q);
          } else {
            dx[e] = du;
          }
        }
        if (row < a.T) {
          if (a.dres_out) ch[j].store(static_cast<R *>(a.dres_out) + row * a.D, out);
          ch[j].store(static_cast<T *>(a.dx) + row * a.D, dx);
        }
      }
    }
  }
  const bool alone = gridDim.x == 1;  // its sums are the gradients
  const int outs = 1 + (a.dscale != nullptr) + (a.dpost != nullptr);
  float *out = a.partial + (size_t)blockIdx.x * outs * a.D;
  write_partial<VE, C, LANES, kRows>(aw, ch, alone ? a.dw : out, lds);
  if constexpr (READS_X) {
    if (a.dscale) write_partial<VE, C, LANES, kRows>(as, ch, alone ? a.dscale : out += a.D, lds);
    if (a.dpost) write_partial<VE, C, LANES, kRows>(ap, ch, alone ? a.dpost : out += a.D, lds);
  }
}

// --------------------------------------------------------------------- gate_norm
// act(z) and its derivative, from t = e^-z: s = 1 / (1 + t) is 0 where t overflows.  Its
// complement is t s, since 1 - s would cancel for open gates; the minimum, which passes
// over a NaN, makes it 1 where t s is infinity times 0.
__device__ __forceinline__ void activation(bool silu, float z, float &f, float &df) {
  const float t = __builtin_amdgcn_exp2f(z * -1.44269504f), s = __builtin_amdgcn_rcpf(1.f + t);
  const float rest = fminf(t * s, 1.f);
  f = silu ? z * s : s;
  df = f * rest + (silu ? s : 0.f);  // s (1 + z (1 - s)), or s (1 - s)
}

// Where a row (token, head) of a tensor [T, H, d] with a token stride begins.
__device__ __forceinline__ long head_row(uint32_t row, int H, int d, long stride) {
  if (stride == (long)H * d) return (long)row * d;
  const uint32_t t = row / (uint32_t)H;
  return (long)t * stride + (long)(row - t * (uint32_t)H) * d;
}

// 32768 tokens x 16 heads of 128 in bf16 73 us, 5.5 TB/s.
template <typename T, int VE, int LANES, int C>
__global__ __launch_bounds__(forward_threads<LANES>()) void gate_norm_kernel(GateNormArgs a) {
  constexpr int kThreads = forward_threads<LANES>(), kRows = kThreads / LANES;
  HAGDN_ROW_SUMS(sums, LANES, kThreads, 1);
  const float inv = 1.f / (float)a.d;
  const long rows = (long)a.T * a.H;
  Chunk<VE> ch[C];
#pragma unroll
  for (int j = 0; j < C; ++j) ch[j] = Chunk<VE>((j * LANES + threadIdx.x % LANES) * VE, a.d);
  // the loop's bounds are those of the workgroup's first row: all lanes take every turn
  for (long first = (long)blockIdx.x * kRows; first < rows; first += (long)gridDim.x * kRows) {
    const bool live = first + threadIdx.x / LANES < rows;
    const long row = live ? first + threadIdx.x / LANES : rows - 1;
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
      if (live) ch[j].store(static_cast<T *>(a.y) + row * a.d, x[j]);
    }
  }
}

// With n = o r and dn = dy act(z): do = r (w dn - n mean(n w dn)), dz = dy w n act'(z),
// dw = sum dn n.  8192 tokens x 32 heads of 128 in bf16 67 us, 5.0 TB/s.
template <typename T, int VE, int LANES, int C>
__global__ __launch_bounds__(backward_threads<LANES>(), LANES > 512 || sizeof(T) == 2 ? 4 : 3) void gate_norm_backward_kernel(
    GateNormArgs a) {
  constexpr int kThreads = backward_threads<LANES>(), kRows = kThreads / LANES;
  HAGDN_ROW_SUMS(sums, LANES, kThreads, 2);
  __shared__ float lds[kRows > 1 ? kRows * LANES : 1];
  const float inv = 1.f / (float)a.d;
  const long rows = (long)a.T * a.H;
  Chunk<VE> ch[C];
  float aw[C][VE], w[C][VE];
#pragma unroll
  for (int j = 0; j < C; ++j) {
    ch[j] = Chunk<VE>((j * LANES + threadIdx.x % LANES) * VE, a.d);
    ch[j].load(a.w, w[j]);
#pragma unroll
    for (int e = 0; e < VE; ++e) aw[j][e] = 0.f;
  }
  // the loop's bounds are those of the workgroup's first row: all lanes take every turn.
  // A row's operands are fetched while the one before is worked on.
  const long step = (long)gridDim.x * kRows, own = threadIdx.x / LANES;
  Raw<T, VE> nx[C], nz[C], ng[C];
  auto fetch = [&](long row) {
    const uint32_t r = (uint32_t)min(row, rows - 1);
    const T *o = static_cast<const T *>(a.o) + head_row(r, a.H, a.d, a.os);
    const T *z = static_cast<const T *>(a.z) + head_row(r, a.H, a.d, a.zs);
    const T *dy = static_cast<const T *>(a.dy) + head_row(r, a.H, a.d, a.dys);
#pragma unroll
    for (int j = 0; j < C; ++j) {
      ch[j].fetch(o, nx[j]);
      ch[j].fetch(z, nz[j]);
      ch[j].fetch(dy, ng[j]);
    }
  };
  if (rows > 0) fetch((long)blockIdx.x * kRows + own);
  for (long first = (long)blockIdx.x * kRows; first < rows; first += step) {
    const long row = first + own;
    const bool live = row < rows;
    Raw<T, VE> x[C];
    float z[C][VE], g[C][VE], v[2] = {0.f, 0.f};  // dy w act'(z), dn
#pragma unroll
    for (int j = 0; j < C; ++j) {
      x[j] = nx[j];
      Raw<T, VE> dy = ng[j];
      Chunk<VE>::clear(x[j], ch[j].skip);
      Chunk<VE>::clear(dy, live ? ch[j].skip : VE);  // a row past the end adds nothing
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        float f, df;
        activation(a.silu, nz[j].get(e), f, df);
        z[j][e] = dy.get(e) * w[j][e] * df;
        g[j][e] = dy.get(e) * f;
      }
    }
    if (first + step < rows) fetch(row + step);
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float xe = x[j].get(e);
        v[0] += xe * xe;
        v[1] += xe * (w[j][e] * g[j][e]);
      }
    sums(v);
    const float r = rstd(v[0], inv, a.eps), m = r * v[1] * inv;
#pragma unroll
    for (int j = 0; j < C; ++j) {
      float dx[VE];
      x[j].keep_packed();
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float n = x[j].get(e) * r;
        aw[j][e] += g[j][e] * n;
        z[j][e] *= n;
        dx[e] = r * (w[j][e] * g[j][e] - m * n);
      }
      if (live) {
        ch[j].store(static_cast<T *>(a.dout) + row * a.d, dx);
        ch[j].store(static_cast<T *>(a.dz) + row * a.d, z[j]);
      }
    }
  }
  write_partial<VE, C, LANES, kRows>(aw, ch, gridDim.x == 1 ? a.dw : a.partial + (size_t)blockIdx.x * a.d, lds);
}

// -------------------------------------------------------------------- launches
// The lanes of a row of d elements and the chunks of each, K::go<VE, LANES, C>; V is the
// vector's elements (16 bytes of the operands' type).  One chunk a lane, in the backward
// passes eight elements, wherever 1024 lanes hold the row: rows of 2048 bf16 elements on
// one wave with four chunks a lane, which need no barrier, took 115 us instead of 98
// (32768 of them, add_norm).
template <int V, int C, typename K> static hipError_t norm_rows(int d, const K &k) {
  constexpr int E = V * C;
  if (d < V) return k.template go<1, 8, 1>();
  if (d <= 8 * E) return k.template go<V, 8, C>();
  if (d <= 16 * E) return k.template go<V, 16, C>();
  if (d <= 32 * E) return k.template go<V, 32, C>();
  if (d <= 64 * E) return k.template go<V, 64, C>();
  if (d <= 128 * E) return k.template go<V, 128, C>();
  if (d <= 256 * E) return k.template go<V, 256, C>();
  if (d <= 512 * E) return k.template go<V, 512, C>();
  if (d <= 1024 * E) return k.template go<V, 1024, C>();
  if constexpr (1024 * E * 2 < kMaxNormDim)
    if (d > 1024 * E * 2) return k.template go<V, 1024, 4 * C>();
  return k.template go<V, 1024, 2 * C>();
}

// Workgroups for `rows` rows, `per` of them each at a time; forward passes.
static unsigned norm_grid(long rows, int per) {
  const long groups = (rows + per - 1) / per;
  return (unsigned)(groups < (1l << 20) ? groups : 1l << 20);
}

// Workgroups of a backward pass, `per` rows at a time each: at most a.parts, never one
// without rows, and one alone, which needs no second kernel, for what two would do.
static int norm_parts_used(long rows, int per, int parts) {
  const long groups = (rows + per - 1) / per;
  return groups <= 2 ? 1 : (int)(groups < parts ? groups : parts);
}

template <typename T, typename R> struct AddNorm {
  const AddNormArgs &a;
  hipStream_t s;
  template <int VE, int LANES, int C> hipError_t go() const {
    hipLaunchKernelGGL((add_norm_kernel<T, R, VE, LANES, C>), dim3(norm_grid(a.T, forward_threads<LANES>() / LANES)),
                       dim3(forward_threads<LANES>()), 0, s, a);
    return hipGetLastError();
  }
};
template <typename T, typename R> struct AddNormBackward {
  const AddNormArgs &a;
  hipStream_t s;
  template <int VE, int LANES, int C> hipError_t go() const {
    const int parts = norm_parts_used(a.T, backward_threads<LANES>() / LANES * rows_per_turn<T, R, LANES>(),
                                       a.parts);
    const dim3 grid(parts), block(backward_threads<LANES>());
    if (a.post || a.scale_vec) hipLaunchKernelGGL((add_norm_backward_kernel<T, R, VE, LANES, C, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((add_norm_backward_kernel<T, R, VE, LANES, C, false>), grid, block, 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || parts == 1) return e;
    return sum_parts(a.partial, parts, a.D, a.dw, a.dscale ? a.dscale : a.dpost, a.dscale ? a.dpost : nullptr, s);
  }
};
template <typename T> struct GateNorm {
  const GateNormArgs &a;
  hipStream_t s;
  template <int VE, int LANES, int C> hipError_t go() const {
    hipLaunchKernelGGL((gate_norm_kernel<T, VE, LANES, C>), dim3(norm_grid((long)a.T * a.H, forward_threads<LANES>() / LANES)),
                       dim3(forward_threads<LANES>()), 0, s, a);
    return hipGetLastError();
  }
};
template <typename T> struct GateNormBackward {
  const GateNormArgs &a;
  hipStream_t s;
  template <int VE, int LANES, int C> hipError_t go() const {
    const int parts = norm_parts_used((long)a.T * a.H, backward_threads<LANES>() / LANES, a.parts);
    hipLaunchKernelGGL((gate_norm_backward_kernel<T, VE, LANES, C>), dim3(parts), dim3(backward_threads<LANES>()), 0, s, a);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || parts == 1 ? e : sum_parts(a.partial, parts, a.d, a.dw, nullptr, nullptr, s);
  }
};

hipError_t launch_add_norm(const AddNormArgs &a, bool bf16, bool res_bf16, hipStream_t s) {
  if (!bf16) return norm_rows<4, 1>(a.D, AddNorm<float, float>{a, s});
  return res_bf16 ? norm_rows<8, 1>(a.D, AddNorm<bf16_t, bf16_t>{a, s}) : norm_rows<8, 1>(a.D, AddNorm<bf16_t, float>{a, s});
}

hipError_t launch_add_norm_backward(const AddNormArgs &a, bool bf16, bool res_bf16, hipStream_t s) {
  if (!bf16) return norm_rows<4, 2>(a.D, AddNormBackward<float, float>{a, s});
  return res_bf16 ? norm_rows<8, 1>(a.D, AddNormBackward<bf16_t, bf16_t>{a, s})
                  : norm_rows<8, 1>(a.D, AddNormBackward<bf16_t, float>{a, s});
}

hipError_t launch_gate_norm(const GateNormArgs &a, bool bf16, hipStream_t s) {
  return bf16 ? norm_rows<8, 1>(a.d, GateNorm<bf16_t>{a, s}) : norm_rows<4, 1>(a.d, GateNorm<float>{a, s});
}

hipError_t launch_gate_norm_backward(const GateNormArgs &a, bool bf16, hipStream_t s) {
  return bf16 ? norm_rows<8, 1>(a.d, GateNormBackward<bf16_t>{a, s}) : norm_rows<4, 2>(a.d, GateNormBackward<float>{a, s});
}

}  // namespace hagdn

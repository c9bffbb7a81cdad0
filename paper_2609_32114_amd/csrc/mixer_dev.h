// mixer_dev.h -- device parts shared by the short convolution and the selective scan:
// activations, elements at any alignment, and the walk over packed sequences.
#pragma once

#include "device.h"
#include "glr.h"  // row access
#include "mixer.h"
#include "prefill.h"

namespace hagdn {

constexpr float kLog2e = 1.44269504f;

// 1 / (1 + e^-v) by the hardware's 2^x and reciprocal: an ulp each, and |v| 2^-24 of the
// exponent's product.  Below v = -87, where it is under the least normal number, it is 0.
__device__ __forceinline__ float logistic(float v) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * v));
}
__device__ __forceinline__ float silu(float v) { return v * logistic(v); }
// The derivative of silu from its logistic s: s (1 + v (1 - s)).  What 1 - s loses where s is near
// one is |v| 2^-24 of the result.
__device__ __forceinline__ float silu_slope(float v, float s) { return s * __builtin_fmaf(v, 1.f - s, 1.f); }

// log(1 + e^v) = max(v, 0) + log1p(t), t = e^-|v|.  With w = 1 + t rounded, log1p(t) is log w and
// what w lost of t (over w, which is one wherever that counts).  The hardware's logarithm keeps
// its digits near one: at most 1.8 ulp, measured over every seventh t from 2^-30 to 1, so that
// small results, steps of 1e-3 and less, keep theirs.
__device__ __forceinline__ float softplus(float v) {
  const float t = __builtin_amdgcn_exp2f(-__builtin_fabsf(v) * kLog2e), w = 1.f + t;
  return __builtin_fmaf(__builtin_amdgcn_logf(w), 0.693147182f, t - (w - 1.f)) + __builtin_fmaxf(v, 0.f);  // (a NaN comes through t)
}

// V consecutive elements, aligned as one of them is.
template <typename T, int V> struct __attribute__((packed, aligned(sizeof(T)))) Pack {
  T v[V];
};
template <typename T, int V> __device__ __forceinline__ Pack<T, V> load_pack(const void *base, size_t at) {
  return *reinterpret_cast<const Pack<T, V> *>(static_cast<const T *>(base) + at);
}
template <typename T, int V> __device__ __forceinline__ void store_pack(void *base, size_t at, const Pack<T, V> &p) {
  *reinterpret_cast<Pack<T, V> *>(static_cast<T *>(base) + at) = p;
}

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// The sequence offsets, in LDS where up to kCheckInPlace sequences' fit: a sequence's end costs
// a wave some 100 ns from there and a microsecond from memory.
struct Offsets32 {
  const int32_t *cu;  // null: one sequence of all tokens
  int N, T;
  const HAGDN_LDS int32_t *lds;
  __device__ int operator[](int i) const { return uniform(lane_value(i)); }
  __device__ int lane_value(int i) const {
    if (N <= kCheckInPlace) return lds[i];
    return cu[i];
  }
};
// Fills the LDS copy and says whether cu[0 .. N] are the offsets of N sequences over T tokens:
// asked here, where the call's first workgroup tells the host (unless status is null), or by the
// kernel before.  The whole workgroup calls.
__device__ __forceinline__ bool stage_offsets(const int32_t *cu, int N, int T, int *status, int32_t (&lds)[kCheckInPlace + 1],
                                              Offsets32 &o) {
  o = {cu, N, T, (const HAGDN_LDS int32_t *)lds};
  if (cu && N > kCheckInPlace) return uniform(*status) == 0;
  bool ok = true;
  if (cu) {
    for (int i = threadIdx.x; i <= N; i += blockDim.x) lds[i] = cu[i];
    __syncthreads();
    int bad = 0;
    for (int i = threadIdx.x; i < N; i += blockDim.x) bad |= lds[i] > lds[i + 1];
    if (threadIdx.x == 0) bad |= lds[0] != 0 || lds[N] != T;
    ok = !__syncthreads_or(bad);
  }
  if (status && blockIdx.x == 0 && threadIdx.x == 0) *status = ok ? 0 : kDevBadSeqlens;
  return ok;
}

// The sequence that a token belongs to, followed from one token to the next by a whole
// wave.  The offsets must have been checked.
struct Cursor {
  Offsets32 cu;
  int seq, start, end;  // uniform over the wave
  // The sequence of token t < T.  Each round of the search the lanes divide the range by 64.
  __device__ Cursor(const Offsets32 &o, int t) : cu(o), seq(0), start(0), end(o.T) {
    if (!cu.cu) return;
    int lo = 0, len = cu.N;  // the last sequence that starts at or before t is in [lo, lo + len)
    const int lane = lane_id();
    while (len > 1) {
      const int step = (len + 63) / 64;
      const long at = (long)lane * step;
      const bool below = at < len && cu.lane_value(lo + (int)at) <= t;
      const int count = __popcll(__ballot(below));
      const int skip = count > 1 ? (count - 1) * step : 0;
      lo += skip;
      len = min(step, len - skip);
    }
    seq = uniform(lo);
    start = cu[seq];
    end = cu[seq + 1];
  }
  // To the sequence of the token after this one's last (which must exist).
  __device__ void next() {
    start = end;
    do {
      ++seq;
      end = cu[seq + 1];
    } while (end == start);
  }
  // To the sequence of the token before this one's first (which must exist).
  __device__ void previous() {
    end = start;
    do {
      --seq;
      start = cu[seq];
    } while (end == start);
  }
};

// Calls f(n) for each sequence without tokens (all of them where the offsets are
// malformed); the whole wave calls.
template <typename F> __device__ __forceinline__ void for_empty(const int32_t *cu, int N, int T, bool ok, F f) {
  for (long base = 0; base < N; base += 64) {
    const long n = base + lane_id();
    const bool empty = n < N && (!ok || (cu ? cu[n] == cu[n + 1] : T == 0));
    for (uint64_t left = __ballot(empty); left; left &= left - 1) f((int)base + __builtin_ctzll(left));
  }
}

}  // namespace hagdn

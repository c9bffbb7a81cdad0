// glr.h -- shared parts of the gated linear recurrence's kernels: the gate, vector
// access to rows of any alignment, the sequences that meet a run of tokens, and the
// scan over tiles.
//
// The scan.  Over any run of tokens the state goes through an affine map, h_out =
// A h_in + B per channel, and maps compose; a run with a sequence's first token in it
// gives h_out = B whatever comes in (a reset).  The packed tokens are cut into tiles
// whose elements stay in the registers of one workgroup from their only load to the
// result's store, so that every input is read once:
//   1. each wave forms the map of its few tokens, and the waves' maps meet in LDS;
//   2. wave 0 composes them, publishes the tile's map, and follows the maps of the
//      tiles before it back to the nearest state that is known whole, folds forward
//      from there, and publishes the state its own tile leaves;
//   3. each wave folds the maps of the waves before it onto that state and goes over
//      its tokens again, from registers.
// Workgroups take the tiles of their 64 channels in order from a counter, so a tile's
// predecessors have all been taken by workgroups that run or have ended, and every wait
// ends.  (Lanes past the last channel follow a channel of their own column: glr_channel.
// One counter for the whole call costs some 33 ns a tile: 8192 tiles 272 us.)
// The state is always folded forward from a whole one through the same fused products,
// so that its bits do not depend on how far back that one was: results repeat exactly.
// A wait is bounded all the same (kLookLimit, HAGDN_DEV_WAIT_TIMEOUT).
// The backward pass runs the same scan from the last tile to the first.
#pragma once

#include "device.h"
#include "layer.h"
#include "prefill.h"

namespace hagdn {

// ---------------------------------------------------------------------- the gate
struct Gate {
  float a, forget;  // decay e^g, and 1 - a
};

// RAW: g holds a raw value r, the log-gate being -softplus(r): a = 1 / (1 + e^r) and
// 1 - a = 1 / (1 + e^-r), both from e^-|r| so that nothing overflows and neither
// loses digits.  Else a = e^g, and 1 - a = -g (1 + g/2 (1 + g/3 (...))) near zero,
// where 1 - e^g would cancel: the series' first seven terms, whose remainder is
// under 2^-25 of the sum for |g| <= 0.35.
// The exponential is the hardware's 2^x of one product: its relative error is
// |g| 2^-24 from the product and an ulp of its own, which a, falling as e^g, hides.
template <bool RAW> __device__ __forceinline__ Gate glr_gate(float g) {
  constexpr float kLog2e = 1.44269504f;
  Gate k;
  if constexpr (RAW) {
    const float t = __builtin_amdgcn_exp2f(-__builtin_fabsf(g) * kLog2e);
    const float r = __builtin_amdgcn_rcpf(1.f + t), tr = t * r;
    k.a = g > 0.f ? tr : r;
    k.forget = g > 0.f ? r : tr;
  } else {
    k.a = __builtin_amdgcn_exp2f(g * kLog2e);
    float p = 1.f + g * (1.f / 7.f);
    p = 1.f + g * (1.f / 6.f) * p;
    p = 1.f + g * (1.f / 5.f) * p;
    p = 1.f + g * (1.f / 4.f) * p;
    p = 1.f + g * (1.f / 3.f) * p;
    p = 1.f + g * (1.f / 2.f) * p;
    k.forget = __builtin_fabsf(g) <= 0.35f ? -g * p : 1.f - k.a;
  }
  return k;
}

// ------------------------------------------------------------------- row access
// Accesses have a uniform row (a pair of scalar registers) and a lane's 32-bit offset as
// their address.  The empty statements keep the compiler from adding the two first and
// holding every row's sum in a pair of vector registers.
#ifdef __HIP_DEVICE_COMPILE__
#define HAGDN_GLOBAL __attribute__((address_space(1)))
#define HAGDN_LDS __attribute__((address_space(3)))
#define HAGDN_SCALAR(p) asm("" : "+s"(p))
#define HAGDN_VECTOR(v) asm("" : "+v"(v))
#else  // the compiler's host pass only parses device code
#define HAGDN_GLOBAL
#define HAGDN_LDS
#define HAGDN_SCALAR(p)
#define HAGDN_VECTOR(v)
#endif
// Where element c of a row lies.
template <typename T> __device__ __forceinline__ HAGDN_GLOBAL T *in_row(T *row, uint32_t c) {
  HAGDN_GLOBAL char *p = (HAGDN_GLOBAL char *)row;
  uint32_t offset = c * (uint32_t)sizeof(T);
  HAGDN_SCALAR(p);
  HAGDN_VECTOR(offset);
  return (HAGDN_GLOBAL T *)(p + offset);
}
// Element c of one row after another, `stride` elements apart (which may be negative).
template <typename T> struct Rows {
  HAGDN_GLOBAL char *p;
  long step;
  uint32_t offset;
  __device__ Rows(T *row, long stride, uint32_t c)
      : p((HAGDN_GLOBAL char *)row), step(stride * (long)sizeof(T)), offset(c * (uint32_t)sizeof(T)) {
    HAGDN_SCALAR(p);
  }
  __device__ HAGDN_GLOBAL T *here() {
    HAGDN_VECTOR(offset);
    return (HAGDN_GLOBAL T *)(p + offset);
  }
  __device__ void advance() {
    p += step;
    HAGDN_SCALAR(p);
  }
};

// --------------------------------------------------------------- sequences' ends
// Whether cu[0 .. N] are the offsets of N sequences over T tokens; every thread of
// the workgroup takes part and gets the answer.
__device__ __forceinline__ bool glr_seqlens_ok(const int32_t *cu, int N, int T) {
  if (!cu) return true;
  int bad = 0;
  for (int i = threadIdx.x; i < N; i += blockDim.x) bad |= cu[i] > cu[i + 1];
  if (threadIdx.x == 0) bad |= cu[0] != 0 || cu[N] != T;
  return !__syncthreads_or(bad);
}

// The sequence offsets, in LDS where they fit: a wave looks its tokens' sequences up while
// its rows are on their way, and loads from memory would have to wait for those (loads
// return in order): the backward pass of a packed batch of eight, 34800 x 2048 tokens, took
// 251 us from memory and 241 from LDS, at the time.
// The copy stands one entry further on, below a sentinel, so that no address formed on
// the way to the entry before a sequence's lies below the array.  The pointers keep their
// address spaces: a generic one to both would be a flat access, whose base may not
// leave LDS even where its offset leads back.
constexpr int kLdsOffsets = 1024;
struct Offsets {
  const HAGDN_GLOBAL int32_t *cu;  // null: one sequence of all tokens
  int N;
  const HAGDN_LDS int32_t *lds;
  __device__ int operator[](int i) const {
    if (N < kLdsOffsets) return lds[i + 1];
    return cu[i];
  }
};
// Fills the LDS copy; the caller's next barrier makes it whole.
__device__ __forceinline__ Offsets stage_offsets(const int32_t *cu, int N, int32_t (&lds)[kLdsOffsets + 1]) {
  if (cu && N < kLdsOffsets)
    for (int i = threadIdx.x; i <= N + 1; i += blockDim.x) lds[i] = i == 0 ? -1 : cu[i - 1];
  return {(const HAGDN_GLOBAL int32_t *)cu, N, (const HAGDN_LDS int32_t *)lds};
}

// The first and last tokens of sequences among a wave's tokens [t0, t0 + L), as bit
// masks, and the sequences' numbers in LDS.
template <int L> struct Marks {
  uint32_t first, last;  // uniform over the wave
  bool many;             // more than one sequence in the call
  const int *ids;        // [2 L]: of the sequence that starts, ends at token t0 + i
  __device__ int starts(int i) const { return many ? __builtin_amdgcn_readfirstlane(ids[i]) : 0; }
  __device__ int ends(int i) const { return many ? __builtin_amdgcn_readfirstlane(ids[L + i]) : 0; }
};

// Finds them.  The 64 lanes probe the offsets together: each round of the search divides
// the range by 64, then one look at the offsets from there on (more if tens of empty
// sequences lie there) marks every boundary.  No index or mark leaves its range
// whatever they hold.
template <int L> __device__ __forceinline__ Marks<L> find_marks(const Offsets &cu, int T, long t0, int (&ids)[2 * L]) {
  const int lane = lane_id(), N = cu.N;
  Marks<L> m{0, 0, cu.cu != nullptr, ids};
  if (t0 >= T) return m;
  if (!m.many) {
    m.first = t0 == 0;
    m.last = t0 + L >= T ? 1u << (int)(T - 1 - t0) : 0;
    return m;
  }
  int lo = 0, len = N;  // the last sequence that starts at or before t0 is in [lo, lo + len)
  while (len > 1) {
    const int step = (len + 63) / 64, at = lane * step;
    const bool below = at < len && cu[lo + at] <= t0;
    const int count = __popcll(__ballot(below));
    const int skip = count > 1 ? (count - 1) * step : 0;
    lo += skip;
    len = min(step, len - skip);
  }
  if (lane < 2 * L) ids[lane] = -1;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  for (long base = lo; base <= N; base += 64) {
    const int s = (int)min(base + lane, (long)N + 1);  // N < 2^31 - 1
    bool past = true;
    if (s <= N) {
      const long v = cu[s], i = v - t0;
      if (s < N && cu[s + 1] > v && i >= 0 && i < L) ids[i] = s;
      if (s > 0 && cu[s - 1] < v && i >= 1 && i <= L) ids[L + i - 1] = s - 1;
      past = i > L;
    }
    if (__any(past)) break;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  const bool set = lane < 2 * L && ids[lane] >= 0;
  const uint64_t bits = __ballot(set);
  m.first = (uint32_t)(bits & ((1ull << L) - 1));
  m.last = (uint32_t)(bits >> L) & (uint32_t)((1ull << L) - 1);
  return m;
}

// out[n] = in[n] (null: 0) for the sequences without tokens (all of them if !ok), in
// channel c.
__device__ __forceinline__ void pass_empty(const int32_t *cu, int N, int T, bool ok, const float *in, float *out, int D,
                                           uint32_t c) {
  if (!out) return;
  const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6, lane = lane_id();
  for (long base = (long)wave * 64; base < N; base += waves * 64) {
    const long n = base + lane;
    const bool empty = n < N && (!ok || (cu ? cu[n] == cu[n + 1] : T == 0));
    for (uint64_t left = __ballot(empty); left; left &= left - 1) {
      const size_t at = (size_t)(base + __builtin_ctzll(left)) * D + c;
      if (c < (uint32_t)D) out[at] = in ? in[at] : 0.f;
    }
  }
}

// ------------------------------------------------------------ states between tiles
// One 64-bit word per tile and channel, written and read whole (its halves cannot
// part, so no fence orders them).  Low half: B, or the state that the tile leaves.  High
// half, A being a product of e^g and so never negative:
//   kNoWord   nothing yet (the whole word has all bits set; glr_setup_kernel)
//   kState    the low half is the state
//   else      A, the tile's map
constexpr uint32_t kNoWord = 0xffffffffu, kState = 0x80000000u;
constexpr int kLookLimit = 1 << 20;    // looks before a wait is given up, about a second

__device__ __forceinline__ void publish(uint64_t *row, uint32_t c, uint32_t high, float low) {
  __hip_atomic_store(in_row(row, c), (uint64_t)high << 32 | __float_as_uint(low), __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void publish_map(uint64_t *row, uint32_t c, float A, float B) {
  publish(row, c, __float_as_uint(A) & 0x7fffffffu, B);  // a NaN keeps no sign
}

// One look at the K tiles nearest to one, for one channel a lane: near is the first, dir
// the way to those further off, of which there are `left`, near included.  If some
// tile's state is known whole and every map between is too, the state that enters.
template <int K>
__device__ __forceinline__ bool look(uint64_t *words, int D, uint32_t c, long near, int dir, long left, float &s) {
  uint64_t w[K];
#pragma unroll
  for (int k = 0; k < K; ++k)
    w[k] = __hip_atomic_load(in_row(words + (size_t)(near + dir * (k < left ? k : left - 1)) * D, c), __ATOMIC_RELAXED,
                             __HIP_MEMORY_SCOPE_AGENT);
  int found = -1;
  bool open = true;  // every tile so far has its word
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const uint32_t high = (uint32_t)(w[k] >> 32);
    if (found < 0 && open && __all(high == kState)) found = k;
    open &= (bool)__all(high != kNoWord);
  }
  if (found < 0) return false;
#pragma unroll
  for (int k = K - 1; k >= 0; --k)
    if (k <= found) {
      const uint32_t high = (uint32_t)(w[k] >> 32);
      const float low = __uint_as_float((uint32_t)w[k]);
      s = high == kState ? low : __builtin_fmaf(__uint_as_float(high), s, low);
    }
  return true;
}

// The state that enters a tile.  The whole wave calls.  Mostly one of the nearest tiles'
// states is there when its turn comes; where a call has few channels its tiles all wait
// for each other, and a wider look, which costs no more time, moves the states on by
// more tiles at once.
__device__ __forceinline__ float look_back(uint64_t *words, int D, uint32_t c, long near, int dir, long left, int *status) {
  float s = 0.f;
  if (look<4>(words, D, c, near, dir, left, s)) return s;
  for (int looks = 0; looks < kLookLimit; ++looks) {
    if (look<8>(words, D, c, near, dir, left, s)) return s;
    __builtin_amdgcn_s_sleep(1);
  }
  if (lane_id() == 0) atomicMax(status, kDevWaitTimeout);
  return 0.f;
}

// The next tile of a column of 64 channels.  A tile is worked on as soon as it is taken:
// workgroups that take one ahead, to hide the counter's latency, hold up those that took
// later ones (packed batch of eight, 34800 x 2048 tokens, 147 us instead of 131).
__device__ __forceinline__ uint32_t take_tile(const GlrArgs &a, uint32_t col) {
  return atomicAdd(a.counters + (size_t)col * kGlrCounterStride, 1u);
}

// The instance of a launcher for a call's form: Launch<T, G>::go<RAW, CONVEX>(a, s).
template <template <typename, typename> class Launch, typename A>
hipError_t glr_dispatch(const A &a, const GlrForm &f, hipStream_t s) {
  auto forms = [&](auto types) {
    using K = decltype(types);
    if (f.raw) return f.convex ? K::template go<true, true>(a, s) : K::template go<true, false>(a, s);
    return f.convex ? K::template go<false, true>(a, s) : K::template go<false, false>(a, s);
  };
  if (!f.bf16) return forms(Launch<float, float>());
  return f.gate_bf16 ? forms(Launch<bf16_t, bf16_t>()) : forms(Launch<bf16_t, float>());
}

// Compute units, and a call's tiles of `tokens` tokens x 64 channels.
inline long glr_cus(const GlrArgs &a) { return a.cus > 0 ? a.cus : 256; }
inline long glr_tiles(const GlrArgs &a, long tokens) { return ((long)a.T + tokens - 1) / tokens * (((long)a.D + 63) / 64); }

// Clears the words and the counter, checks the offsets, writes the status.
hipError_t launch_glr_setup(const GlrArgs &, size_t words, uint32_t cols, hipStream_t);

}  // namespace hagdn

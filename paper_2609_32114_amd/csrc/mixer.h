// mixer.h -- arguments and launchers of the short causal convolution (k9_conv.hip), the
// selective state space scan (k10_ssm.hip, k11_ssm_backward.hip) and the copies between
// rows of state pools (k12_pool.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "layer.h"

namespace hagdn {

constexpr size_t kMixerHeader = 256;  // workspace bytes before anything else: the status word
// Offsets of up to this many sequences are checked by every workgroup that needs to know;
// more are checked once, by a kernel of their own.
constexpr int kCheckInPlace = 512;

// ------------------------------------------------------- short causal convolution
constexpr int kMinTaps = 2, kMaxTaps = 8;

struct ConvArgs {
  const void *x, *dy;     // rows of D channels, strides below (in elements)
  long xs, dys;
  const float *w, *b;     // [D, W]; [D] or null
  const void *w0;         // [N, W - 1, D] windows before the sequences, or null: zeros
  const void *dfinal;     // [N, W - 1, D] or null
  const int32_t *cu;      // [N + 1] or null: one sequence
  int N, T, D, W;
  bool silu;
  void *y, *w_final;      // [T, D]; [N, W - 1, D] or null
  void *dx, *dw0;         // [T, D]; [N, W - 1, D] or null
  float *dw, *db;         // [D, W]; [D] or null
  int *status;
  float *partial;         // [parts][W + 1][D]
  int parts;              // runs of tokens whose sums of the weights' gradients stand apart
  int run;                // tokens of a run
};

struct ConvStepArgs {
  const void *x;
  long xs;
  const float *w, *b;
  void *state;            // [num_slots, W - 1, D]
  const int32_t *slots;
  int num_slots, N, D, W;
  bool silu;
  void *y;
};

hipError_t launch_conv_forward(const ConvArgs &, bool bf16, hipStream_t);
hipError_t launch_conv_backward(const ConvArgs &, bool bf16, hipStream_t);
hipError_t launch_conv_step(const ConvStepArgs &, bool bf16, hipStream_t);
// Writes whether cu[0 .. N] are the offsets of N sequences over T tokens to *status.
hipError_t launch_check_offsets(const int32_t *cu, int N, int T, int *status, hipStream_t);

// The backward pass's runs of tokens: a wave goes over one run of 256 channels (of 64 in calls
// below 256 channels).
inline int conv_run(int T, int D, int cus) {
  const long cols = ((long)D + 255) / 256, waves = 16l * (cus > 0 ? cus : 256);
  const long run = ((long)T * cols + waves - 1) / waves;
  return (int)(run < 16 ? 16 : run < T || T < 16 ? run : T);  // (a run of all tokens may pass 31 bits)
}
// The forward pass's: two waves a SIMD, but runs long enough beside the rows that they
// read a second time.
inline int conv_forward_run(int T, int D, int cus) {
  const long cols = ((long)D + 255) / 256, waves = 8l * (cus > 0 ? cus : 256);
  const long run = ((long)T * cols + waves - 1) / waves;
  return (int)(run < 8 ? 8 : run > 64 ? 64 : (run + 7) / 8 * 8);
}
inline int conv_parts(int T, int D, int cus) {
  const int run = conv_run(T, D, cus);
  return T > 0 ? (T - 1) / run + 1 : 1;
}

// ----------------------------------------------------- selective state space scan
constexpr int kMaxStates = 64;
// States a channel as the kernels hold them: the next of 16, 32 and 64.
inline int ssm_padded(int S) { return S <= 16 ? 16 : S <= 32 ? 32 : 64; }
// Tokens between two saved states of the scan (hagdn.h, ssm_prefill).
constexpr int kSsmGroup = 16;

struct SsmArgs {
  const void *x, *dt, *z, *B, *C, *dy;  // rows of D channels (B, C: of G x S), strides below; z may be null
  long xs, dts, zs, Bs, Cs, dys;
  const float *A, *skip, *bias;         // [D, S]; [D] or null
  const float *s0, *dfinal;             // [N, D, S] or null
  const int32_t *cu;
  int N, T, D, S, G;
  bool raw;                             // dt + bias goes through the softplus
  void *y;                              // [T, D]
  float *s_final;                       // [N, D, S] or null
  float *ckpt;                          // [ceil(T / group), padded S, D] or null
  void *dx, *ddt, *dz, *dB, *dC;        // [T, D], .., [T, G, S]
  float *dA, *dskip, *dbias, *ds0;
  // workspace
  int *status;
  float *maps;                          // [chunks][padded S][D]: what a chunk leaves of nothing, then what enters it
  float *sums;                          // [chunks][D]: its step sizes' sum
  int *resets;                          // [chunks]: whether a sequence starts (backward: ends) in it
  float *dbc;                           // [teams of a group][T][G][2][padded S]: sums of dB and dC over channels
  float *dweights;                      // [chunks][padded S + 2][D]: sums of dA, dskip and dbias over a chunk
  int chunk, chunks;                    // tokens of a chunk
};

struct SsmStepArgs {
  const void *x, *dt, *z, *B, *C;
  long xs, dts, zs, Bs, Cs;
  const float *A, *skip, *bias;
  float *state;                         // [num_slots, D, S]
  const int32_t *slots;
  int num_slots, N, D, S, G;
  bool raw;
  void *y;
};

// Columns of 64 channels of a group of channels, the waves of a workgroup, which have a column
// each and share B and C (one where a group has fewer than four columns: the others would
// only wait), and workgroups that a group's columns take.
inline long ssm_columns(int D, int G) { return ((long)D / G + 63) / 64; }
inline int ssm_waves(int D, int G) { return ssm_columns(D, G) < 4 ? 1 : 4; }
inline long ssm_teams(int D, int G) { return (ssm_columns(D, G) + ssm_waves(D, G) - 1) / ssm_waves(D, G); }

// Tokens of a chunk, which a workgroup goes over.  The scan is bound by its arithmetic, so that
// every CU should get as many workgroups as the others: one round of what can be resident (by
// registers and LDS), or in calls where a chunk would pass 512 tokens as few rounds as keep it
// below.  (17401 x 2048 tokens in 68 chunks of 256, 2.1 workgroups a CU: outputs 203 us, backward
// 913; in chunks of 136 and 272 149 and 632 to 666.)  Calls of up to 64 tokens of 16 states are one
// chunk, which needs one launch instead of three.
inline int ssm_chunk(int T, int D, int S, int G, int cus, bool backward) {
  const auto over = [](long a, long b) { return (a + b - 1) / b; };
  const int padded = ssm_padded(S);
  const bool one = ssm_waves(D, G) == 1;
  const int resident = !backward ? (one ? 16 : 4) : padded == 16 ? (one ? 8 : 2) : padded == 32 ? (one ? 6 : 2) : one ? 3 : 1;
  const long slots = (cus > 0 ? cus : 256) * (long)resident;
  const long total = (long)T * ssm_teams(D, G) * G, rounds = over(total + 1, slots * 512);
  const int unit = backward ? kSsmGroup : 8, least = (long)T * padded <= 1024 ? 64 : 16;
  const long chunk = over(over(total, slots * rounds), unit) * unit;
  return (int)(chunk < least ? least : chunk);
}

hipError_t launch_ssm_forward(const SsmArgs &, bool bf16, bool dt_bf16, hipStream_t);
hipError_t launch_ssm_backward(const SsmArgs &, bool bf16, bool dt_bf16, hipStream_t);
hipError_t launch_ssm_step(const SsmStepArgs &, bool bf16, bool dt_bf16, hipStream_t);
// Shared by both directions: what enters each chunk from what each leaves of nothing.
hipError_t launch_ssm_carry(const SsmArgs &, bool backward, hipStream_t);

// ------------------------------------------------------------------- state pools
// Device status (hagdn_device_code) of a fork that found too few free slots.
constexpr int kDevPoolFull = 3;
constexpr int kPoolsPerLaunch = 64;
constexpr int kMaxPools = 1024;
constexpr int kMaxPoolSlots = 1 << 20;    // of a plan (fork, compact)
constexpr int kMaxMovesInPlace = 8192;    // rows of a copy within pools
struct Pool {
  void *to;
  const void *from;
  uint64_t units;  // of a row
  int unit;        // bytes of an access: 16, 8, 4, 2 or 1, what rows and pointers are aligned to
};
struct PoolCopyArgs {
  Pool pools[kPoolsPerLaunch];
  int count;                // of pools
  const int32_t *dst, *src;  // rows, or null: entry i is row i
  int n, dst_rows, src_rows;
  const int *moves;         // null, or {number of moves, dst, src, dst, src, ..}: instead of the tables
};
struct PoolPlanArgs {
  const int32_t *slots, *parents;  // [N], [M] (fork)
  int32_t *out;                    // [M] (fork), [N] (compact)
  int N, M, num_slots;
  int *status;
  int *moves;                      // {count, dst, src, ..}
  int *mark;                       // [num_slots]
};
hipError_t launch_pool_copy(const PoolCopyArgs &, bool in_place, int cus, hipStream_t);
hipError_t launch_pool_fork_plan(const PoolPlanArgs &, hipStream_t);
hipError_t launch_pool_compact_plan(const PoolPlanArgs &, hipStream_t);

}  // namespace hagdn

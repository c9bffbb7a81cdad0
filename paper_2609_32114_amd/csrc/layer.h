// layer.h -- arguments and launchers of the operators around the delta-rule
// layers: the gated linear recurrence (k6_glr.hip, k7_glr_backward.hip) and the
// norms before and after a block (k8_norms.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace hagdn {

// Records the message of a failed call for hagdn_last_error; returns code (api.cpp).
int set_error(int code, const char *msg);
// Compute units of the current device (0 if it cannot be queried) (api.cpp).
int device_cus();

// Tokens between two saved states of the recurrence (hagdn.h, glr_prefill).
constexpr int kGlrGroup = 128;

// One sequence's token range is [cu[n], cu[n+1]); cu == nullptr: N = 1, [0, T).
struct GlrArgs {
  const void *x, *g, *dh;  // rows of D channels, strides below (in elements)
  long xs, gs, dhs;
  const float *s0, *dfinal;  // [N, D] or null
  const int32_t *cu;
  int N, T, D;
  void *h, *dx, *dg;       // [T, D], contiguous
  float *s_final, *ds0;    // [N, D] or null
  float *ckpt;             // [ceil(T / kGlrGroup), D] states before each group's first token, or null
  int cus;                 // compute units of the device
  // workspace: the device status word, a tile counter per 64 channels, and a word per
  // tile and channel (glr.h)
  int *status;
  uint32_t *counters;
  uint64_t *words;
};

// The smallest tile of a call that has several, in tokens (calls of up to 64 tokens take one
// of 64); a call of one tile needs no words.
constexpr int kGlrLeastTile = 128;
constexpr size_t kGlrHeader = 256;          // bytes before the counters
constexpr size_t kGlrCounterStride = 32;    // counters lie in memory lines of their own
inline size_t glr_counter_bytes(int D) { return ((size_t)D + 63) / 64 * kGlrCounterStride * sizeof(uint32_t); }

// The channel a lane of the scan works on.  Lanes past the last channel, which store and
// publish nothing, follow a channel of their own column of 64 (the last one), so that a
// tile waits for tiles of its own column only.  at: 64 column + lane; D >= 1.
__host__ __device__ inline uint32_t glr_channel(uint32_t at, uint32_t D) { return at < D ? at : D - 1; }

struct GlrStepArgs {
  const void *x, *g;
  long xs, gs;
  float *state;
  const int32_t *slots;
  int num_slots, N, D;
  void *h;
};

// How the gate and the input weight are formed (hagdn.h, glr_prefill).
struct GlrForm {
  bool bf16, gate_bf16, raw, convex;
};

hipError_t launch_glr_forward(const GlrArgs &, const GlrForm &, hipStream_t);
hipError_t launch_glr_backward(const GlrArgs &, const GlrForm &, hipStream_t);
hipError_t launch_glr_step(const GlrStepArgs &, const GlrForm &, hipStream_t);

struct AddNormArgs {
  const void *x, *res, *dy, *dres;  // rows of D, strides below (in elements); res, dres may be null
  long xs, rs, dys, drs;
  const float *w, *post, *scale_vec;
  float scale, eps;
  int T, D;
  void *y, *res_out;         // forward, contiguous
  void *dx, *dres_out;       // backward, contiguous
  float *dw, *dscale, *dpost;  // [D]; the last two or null
  float *partial;            // workspace: [parts][1 + vector + post][D]
  int parts;
};

struct GateNormArgs {
  const void *o, *z, *dy;  // [T, H, d], token strides below (in elements)
  long os, zs, dys;
  const float *w;
  float eps;
  int T, H, d;
  bool silu;               // else sigmoid
  void *y, *dout, *dz;     // contiguous
  float *dw;
  float *partial;          // workspace: [parts][d]
  int parts;
};

hipError_t launch_add_norm(const AddNormArgs &, bool bf16, bool res_bf16, hipStream_t);
hipError_t launch_add_norm_backward(const AddNormArgs &, bool bf16, bool res_bf16, hipStream_t);
hipError_t launch_gate_norm(const GateNormArgs &, bool bf16, hipStream_t);
hipError_t launch_gate_norm_backward(const GateNormArgs &, bool bf16, hipStream_t);

// Elements of a norm's row at most.
constexpr int kMaxNormDim = 16384;
// Workgroups that share the rows of a backward norm, each with its own partial sums of
// the weights' gradients: one a CU.  With two the rows flow no faster and the sums are
// twice as many (add_norm, 8192 rows of 2048 with both vectors 57 us instead of 50;
// gate_norm, 8192 x 32 heads of 128 72 instead of 67).
inline int norm_parts(long rows, int cus) {
  const long most = cus > 0 ? cus : 256;
  return (int)(rows < 1 ? 1 : rows < most ? rows : most);
}

}  // namespace hagdn

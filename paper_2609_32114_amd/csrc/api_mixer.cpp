// api_mixer.cpp -- the C ABI of the short convolution, the selective scan and the state
// pools (include/hagdn.h): host-side argument checks, then the launches on the caller's
// stream.  No allocation, no synchronisation, no pointer retained after return.
#include <hip/hip_runtime.h>

#include <stdarg.h>
#include <stdio.h>

#include "hagdn.h"
#include "mixer.h"
#include "prefill.h"

namespace {

int fail(int code, const char *fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return hagdn::set_error(code, buf);
}

int done(hipError_t e) {
  return e == hipSuccess ? HAGDN_OK : fail(HAGDN_EHIP, "HIP error: %s", hipGetErrorString(e));
}

// A device buffer argument: its name, whether it must not be NULL, its alignment, and its
// extent in bytes for the check of overlaps (0: not known here).
struct Buf {
  const void *p;
  const char *name;
  bool required;
  size_t align, bytes;
};
template <size_t N> int check_buffers(const Buf (&bs)[N]) {
  for (const Buf &b : bs) {
    if (b.required && !b.p) return fail(HAGDN_EINVAL, "NULL required pointer %s", b.name);
    if ((uintptr_t)b.p % b.align) return fail(HAGDN_EINVAL, "%s must be %zu-byte aligned", b.name, b.align);
  }
  return HAGDN_OK;
}
bool overlap(const void *a, size_t na, const void *b, size_t nb) {
  const uintptr_t p = (uintptr_t)a, q = (uintptr_t)b;
  return p && q && na && nb && (p >= q ? p - q < nb : q - p < na);
}
// Outputs (the workspace among them) against inputs and each other.
template <size_t NO, size_t NI> int check_overlaps(const Buf (&outs)[NO], const Buf (&ins)[NI]) {
  for (size_t i = 0; i < NO; ++i) {
    for (const Buf &b : ins)
      if (overlap(outs[i].p, outs[i].bytes, b.p, b.bytes)) return fail(HAGDN_EINVAL, "%s overlaps %s", outs[i].name, b.name);
    for (size_t j = i + 1; j < NO; ++j)
      if (overlap(outs[i].p, outs[i].bytes, outs[j].p, outs[j].bytes))
        return fail(HAGDN_EINVAL, "%s overlaps %s", outs[i].name, outs[j].name);
  }
  return HAGDN_OK;
}

struct Stride {
  int64_t s;
  const char *name;
};
template <size_t N> int check_strides(const Stride (&ss)[N]) {
  for (const Stride &a : ss)
    if (a.s < 0 || a.s > 0x7fffffff)
      return fail(HAGDN_EINVAL, "%s must be in [0, 2^31) (got %lld)", a.name, (long long)a.s);
  return HAGDN_OK;
}

size_t esize(int dtype) { return dtype == HAGDN_BF16 ? 2 : 4; }
// Bytes from the first to the last of `rows` rows of `cols` elements.
size_t extent(int rows, int64_t stride, size_t cols, int dtype) {
  if (rows < 1) return 0;
  const size_t n = (size_t)(rows - 1) * (size_t)stride + cols;  // below 2^63
  return n >> 60 ? SIZE_MAX : n * esize(dtype);
}

int query_cus() {
  const int n = hagdn::device_cus();
  return n > 0 ? n : 256;  // no device: sizes as for an MI355X
}

size_t pad256(size_t n) { return (n + 255) / 256 * 256; }

// Token numbers, and those of the rows that kernels look ahead for, fit 31 bits.
constexpr int kMaxTokens = 0x7fff0000;
int check_tokens(int T) {
  if (T < 0) return fail(HAGDN_EINVAL, "T_total must be >= 0 (got %d)", T);
  if (T > kMaxTokens) return fail(HAGDN_EUNSUPPORTED, "T_total > %d unsupported (got %d)", kMaxTokens, T);
  return HAGDN_OK;
}

// --------------------------------------------------------------- convolution
int check_conv(int T, int D, int W, int dtype, int activation) {
  if (int rc = check_tokens(T)) return rc;
  if (D < 1) return fail(HAGDN_EINVAL, "D must be >= 1 (got %d)", D);
  if (D > (1 << 28)) return fail(HAGDN_EUNSUPPORTED, "D > 2^28 unsupported");
  if (W < hagdn::kMinTaps || W > hagdn::kMaxTaps)
    return fail(HAGDN_EUNSUPPORTED, "W must be in [%d, %d] (got %d)", hagdn::kMinTaps, hagdn::kMaxTaps, W);
  if (dtype != HAGDN_F32 && dtype != HAGDN_BF16) return fail(HAGDN_EUNSUPPORTED, "dtype %d unsupported", dtype);
  if (activation != HAGDN_ACT_SILU && activation != HAGDN_ACT_NONE)
    return fail(HAGDN_EINVAL, "unknown activation %d", activation);
  return HAGDN_OK;
}

int check_sequences(const int32_t *cu, int N) {
  if (N < 1) return fail(HAGDN_EINVAL, "N must be >= 1 (got %d)", N);
  if (!cu && N != 1) return fail(HAGDN_EINVAL, "cu_seqlens may be NULL for one sequence only (N = %d)", N);
  return HAGDN_OK;
}

size_t conv_bytes(int T, int D, int W, bool backward) {
  if (!backward) return hagdn::kMixerHeader;
  return hagdn::kMixerHeader + (size_t)hagdn::conv_parts(T, D, query_cus()) * (W + 1) * (size_t)D * sizeof(float);
}

int check_workspace(const void *ws, size_t bytes, size_t need) {
  if (!ws) return fail(HAGDN_EINVAL, "NULL required pointer workspace");
  if ((uintptr_t)ws % 16) return fail(HAGDN_EINVAL, "workspace must be 16-byte aligned");
  if (bytes < need) return fail(HAGDN_EWORKSPACE, "workspace too small: %zu bytes, need %zu", bytes, need);
  return HAGDN_OK;
}

// ---------------------------------------------------------------------- scan
int check_ssm(int T, int D, int S, int G, int dtype, int dt_dtype, int pre) {
  if (int rc = check_tokens(T)) return rc;
  if (D < 1) return fail(HAGDN_EINVAL, "D must be >= 1 (got %d)", D);
  if (D > (1 << 28)) return fail(HAGDN_EUNSUPPORTED, "D > 2^28 unsupported");
  if (S < 1) return fail(HAGDN_EINVAL, "S must be >= 1 (got %d)", S);
  if (S > hagdn::kMaxStates) return fail(HAGDN_EUNSUPPORTED, "S > %d unsupported (got %d)", hagdn::kMaxStates, S);
  if (G < 1 || D % G) return fail(HAGDN_EINVAL, "G must divide D (got %d and %d)", G, D);
  if (dtype != HAGDN_F32 && dtype != HAGDN_BF16) return fail(HAGDN_EUNSUPPORTED, "dtype %d unsupported", dtype);
  if (dt_dtype != HAGDN_F32 && !(dt_dtype == HAGDN_BF16 && dtype == HAGDN_BF16))
    return fail(HAGDN_EUNSUPPORTED, "dt dtype %d unsupported with dtype %d", dt_dtype, dtype);
  if (pre & ~hagdn::kPreGateSoftplus) return fail(HAGDN_EINVAL, "unsupported preprocessing flags 0x%x", pre);
  return HAGDN_OK;
}

// A call's chunks and the places of its workspace's parts (forward: the first three).
struct SsmPlan {
  int chunk, chunks;
  size_t maps, sums, resets, dbc, dweights, bytes;
  bool fits;  // below 2^62 bytes: what stands above is not wrapped
};
SsmPlan ssm_plan(int T, int D, int S, int G, bool backward) {
  SsmPlan p = {};
  const size_t np = hagdn::ssm_padded(S);
  p.chunk = hagdn::ssm_chunk(T, D, S, G, query_cus(), backward);
  p.chunks = T > 0 ? (T - 1) / p.chunk + 1 : 1;
  const size_t between = p.chunks > 1 ? p.chunks : 0;  // one chunk leaves nothing to another
  size_t at = hagdn::kMixerHeader;
  p.fits = true;
  const auto take = [&](size_t rows, size_t cols) {  // fp32 values
    size_t n;
    const size_t here = at;
    p.fits = p.fits && !__builtin_mul_overflow(rows, cols * 4, &n) && n < (size_t)1 << 62;
    if (p.fits) at += pad256(n);
    p.fits = p.fits && at < (size_t)1 << 62;
    return here;
  };
  p.maps = take(between, np * D);
  p.sums = take(between, D);
  p.resets = take(between, 1);
  if (backward) {
    p.dbc = take((size_t)hagdn::ssm_teams(D, G) * T, 2 * np * G);
    p.dweights = take(p.chunks, (np + 2) * D);
  }
  p.bytes = at;
  return p;
}
int check_fits(const SsmPlan &p, int T, int D, int S, int G) {
  return p.fits ? HAGDN_OK : fail(HAGDN_EINVAL, "sizes too large for a workspace (%d x %d x %d, %d groups)", T, D, S, G);
}

int check_ssm_call(const int32_t *cu, int N, int T, int D, int S, int G, int dtype, int dt_dtype, int pre,
                   const float *dt_bias, const void *ws, size_t ws_bytes, bool backward, SsmPlan *plan) {
  if (int rc = check_sequences(cu, N)) return rc;
  if (int rc = check_ssm(T, D, S, G, dtype, dt_dtype, pre)) return rc;
  if ((size_t)N * (size_t)D * (size_t)S >= 0x7fffffffu) return fail(HAGDN_EINVAL, "N x D x S too large (%d x %d x %d)", N, D, S);
  if (dt_bias && !pre) return fail(HAGDN_EINVAL, "dt_bias needs HAGDN_PRE_GATE_SOFTPLUS");
  *plan = ssm_plan(T, D, S, G, backward);
  if (int rc = check_fits(*plan, T, D, S, G)) return rc;
  return check_workspace(ws, ws_bytes, plan->bytes);
}

void set_plan(hagdn::SsmArgs *a, const SsmPlan &p, void *ws) {
  char *w = static_cast<char *>(ws);
  a->chunk = p.chunk;
  a->chunks = p.chunks;
  a->status = reinterpret_cast<int *>(w);
  a->maps = reinterpret_cast<float *>(w + p.maps);
  a->sums = reinterpret_cast<float *>(w + p.sums);
  a->resets = reinterpret_cast<int *>(w + p.resets);
  a->dbc = reinterpret_cast<float *>(w + p.dbc);
  a->dweights = reinterpret_cast<float *>(w + p.dweights);
}

// --------------------------------------------------------------------- pools
int check_pools(void *const *pools, const size_t *row_bytes, int num_pools) {
  if (num_pools < 1 || num_pools > hagdn::kMaxPools)
    return fail(HAGDN_EINVAL, "num_pools must be in [1, %d] (got %d)", hagdn::kMaxPools, num_pools);
  if (!pools || !row_bytes) return fail(HAGDN_EINVAL, "NULL required pointer pools or row_bytes");
  for (int p = 0; p < num_pools; ++p) {
    if (!pools[p]) return fail(HAGDN_EINVAL, "NULL required pointer pools[%d]", p);
    if (row_bytes[p] < 1 || row_bytes[p] >> 40) return fail(HAGDN_EINVAL, "row_bytes[%d] out of range (%zu)", p, row_bytes[p]);
  }
  return HAGDN_OK;
}

// No two of the pools overlap, and no pool overlaps a source.  (Checked in the order of
// their addresses: a heap on the stack, for up to 2048 ranges.)
struct Range {
  uintptr_t at;
  size_t bytes;
  bool source;
};
bool ranges_disjoint(Range *r, int n) {
  // heap sort by address
  const auto sift = [&](int root, int end) {
    for (int child; (child = 2 * root + 1) < end; root = child) {
      if (child + 1 < end && r[child].at < r[child + 1].at) ++child;
      if (r[root].at >= r[child].at) return;
      const Range t = r[root];
      r[root] = r[child];
      r[child] = t;
    }
  };
  for (int i = n / 2 - 1; i >= 0; --i) sift(i, n);
  for (int end = n - 1; end > 0; --end) {
    const Range t = r[0];
    r[0] = r[end];
    r[end] = t;
    sift(0, end);
  }
  uintptr_t pool_end = 0, source_end = 0;  // of those before
  for (int i = 0; i < n; ++i) {
    if (r[i].at < pool_end || (!r[i].source && r[i].at < source_end)) return false;
    uintptr_t &end = r[i].source ? source_end : pool_end;
    const uintptr_t e = r[i].at + r[i].bytes;
    if (e > end) end = e;
  }
  return true;
}

int check_ranges(void *const *pools, const void *const *sources, const size_t *row_bytes, int num_pools, int dst_rows,
                 int src_rows) {
  Range r[2 * hagdn::kMaxPools];
  int n = 0;
  for (int p = 0; p < num_pools; ++p) {
    size_t bytes;
    const int most = sources && src_rows > dst_rows ? src_rows : dst_rows;
    if (__builtin_mul_overflow(row_bytes[p], (size_t)most, &bytes) || bytes >> 62)
      return fail(HAGDN_EINVAL, "pools[%d] too large (%d rows of %zu bytes)", p, most, row_bytes[p]);
    r[n++] = {(uintptr_t)pools[p], row_bytes[p] * (size_t)dst_rows, false};
    if (sources) r[n++] = {(uintptr_t)sources[p], row_bytes[p] * (size_t)src_rows, true};
  }
  return ranges_disjoint(r, n) ? HAGDN_OK : fail(HAGDN_EINVAL, "pools overlap each other or a source");
}

// The copies of all pools, in launches of up to kPoolsPerLaunch pools.
int launch_copies(hagdn::PoolCopyArgs a, void *const *pools, const void *const *sources, const size_t *row_bytes,
                  int num_pools, bool in_place, hipStream_t s) {
  const int cus = query_cus();
  for (int base = 0; base < num_pools; base += hagdn::kPoolsPerLaunch) {
    a.count = num_pools - base < hagdn::kPoolsPerLaunch ? num_pools - base : hagdn::kPoolsPerLaunch;
    for (int p = 0; p < a.count; ++p) {
      void *to = pools[base + p];
      const void *from = sources ? sources[base + p] : to;
      const size_t row = row_bytes[base + p];
      const uintptr_t bits = (uintptr_t)to | (uintptr_t)from | (uintptr_t)row;
      const int unit = bits % 16 == 0 ? 16 : bits % 8 == 0 ? 8 : bits % 4 == 0 ? 4 : bits % 2 == 0 ? 2 : 1;
      a.pools[p] = {to, from, row / unit, unit};
    }
    if (hipError_t e = hagdn::launch_pool_copy(a, in_place, cus, s)) return done(e);
  }
  return HAGDN_OK;
}

size_t plan_bytes(int num_slots) { return hagdn::kMixerHeader + ((size_t)1 + 3 * (size_t)num_slots) * sizeof(int); }

int check_plan(void *const *pools, const size_t *row_bytes, int num_pools, int num_slots, const void *ws, size_t ws_bytes) {
  if (int rc = check_pools(pools, row_bytes, num_pools)) return rc;
  if (num_slots < 1) return fail(HAGDN_EINVAL, "num_slots must be >= 1 (got %d)", num_slots);
  if (num_slots > hagdn::kMaxPoolSlots)
    return fail(HAGDN_EUNSUPPORTED, "num_slots > %d unsupported (got %d)", hagdn::kMaxPoolSlots, num_slots);
  if (int rc = check_ranges(pools, nullptr, row_bytes, num_pools, num_slots, 0)) return rc;
  return check_workspace(ws, ws_bytes, plan_bytes(num_slots));
}

// A plan's tables (in entries of 4 bytes) and workspace against the pools, and the workspace against
// the tables.
template <size_t N>
int check_plan_overlaps(void *const *pools, const size_t *row_bytes, int num_pools, int num_slots, const Buf (&tables)[N],
                        const void *ws) {
  const size_t need = plan_bytes(num_slots);
  for (int p = 0; p < num_pools; ++p) {
    const size_t bytes = row_bytes[p] * (size_t)num_slots;
    for (const Buf &t : tables)
      if (overlap(t.p, t.bytes, pools[p], bytes)) return fail(HAGDN_EINVAL, "%s overlaps pools[%d]", t.name, p);
    if (overlap(ws, need, pools[p], bytes)) return fail(HAGDN_EINVAL, "workspace overlaps pools[%d]", p);
  }
  for (const Buf &t : tables)
    if (overlap(ws, need, t.p, t.bytes)) return fail(HAGDN_EINVAL, "workspace overlaps %s", t.name);
  return HAGDN_OK;
}

hagdn::PoolPlanArgs plan_args(const int32_t *slots, int N, int num_slots, int32_t *out, void *ws) {
  hagdn::PoolPlanArgs a = {};
  a.slots = slots; a.N = N; a.num_slots = num_slots; a.out = out;
  a.status = static_cast<int *>(ws);
  a.moves = reinterpret_cast<int *>(static_cast<char *>(ws) + hagdn::kMixerHeader);
  a.mark = a.moves + 1 + 2 * (size_t)num_slots;
  return a;
}

}  // namespace

extern "C" {

size_t hagdn_conv_workspace_size(int T_total, int D, int W, int backward) {
  if (check_conv(T_total, D, W, HAGDN_F32, HAGDN_ACT_NONE) != HAGDN_OK) return 0;
  return conv_bytes(T_total, D, W, backward != 0);
}

int hagdn_conv_prefill(const void *x, int64_t x_stride, const float *weight, const float *bias, const void *w0,
                       const int32_t *cu_seqlens, int N, int T_total, int D, int W, int dtype, int activation, void *y,
                       void *w_final, void *workspace, size_t workspace_bytes, void *stream) {
  if (int rc = check_sequences(cu_seqlens, N)) return rc;
  if (int rc = check_conv(T_total, D, W, dtype, activation)) return rc;
  if (workspace || N > hagdn::kCheckInPlace)
    if (int rc = check_workspace(workspace, workspace_bytes, conv_bytes(T_total, D, W, false))) return rc;
  const Stride ss[] = {{x_stride, "x_stride"}};
  if (int rc = check_strides(ss)) return rc;
  const bool tok = T_total > 0;
  const size_t e = esize(dtype), windows = (size_t)N * (W - 1) * D * e;
  const Buf ins[] = {{x, "x", tok, e, extent(T_total, x_stride, D, dtype)}, {w0, "w0", false, e, windows},
                     {weight, "weight", true, 4, (size_t)D * W * 4}, {bias, "bias", false, 4, (size_t)D * 4},
                     {cu_seqlens, "cu_seqlens", false, 4, ((size_t)N + 1) * 4}};
  const Buf outs[] = {{y, "y", tok, e, extent(T_total, D, D, dtype)}, {w_final, "w_final", false, e, windows},
                      {workspace, "workspace", false, 16, conv_bytes(T_total, D, W, false)}};
  if (int rc = check_buffers(ins)) return rc;
  if (int rc = check_buffers(outs)) return rc;
  if (int rc = check_overlaps(outs, ins)) return rc;
  hagdn::ConvArgs a = {};
  a.x = x; a.xs = x_stride; a.w = weight; a.b = bias; a.w0 = w0; a.cu = cu_seqlens; a.N = N; a.T = T_total; a.D = D; a.W = W;
  a.silu = activation == HAGDN_ACT_SILU; a.y = y; a.w_final = w_final; a.status = static_cast<int *>(workspace);
  a.run = hagdn::conv_forward_run(T_total, D, query_cus());
  return done(hagdn::launch_conv_forward(a, dtype == HAGDN_BF16, static_cast<hipStream_t>(stream)));
}

int hagdn_conv_backward(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, const float *weight,
                        const float *bias, const void *w0, const void *dfinal, const int32_t *cu_seqlens, int N,
                        int T_total, int D, int W, int dtype, int activation, void *dx, float *dweight, float *dbias,
                        void *dw0, void *workspace, size_t workspace_bytes, void *stream) {
  if (int rc = check_sequences(cu_seqlens, N)) return rc;
  if (int rc = check_conv(T_total, D, W, dtype, activation)) return rc;
  if (int rc = check_workspace(workspace, workspace_bytes, conv_bytes(T_total, D, W, true))) return rc;
  const Stride ss[] = {{dy_stride, "dy_stride"}, {x_stride, "x_stride"}};
  if (int rc = check_strides(ss)) return rc;
  const bool tok = T_total > 0;
  const size_t e = esize(dtype), windows = (size_t)N * (W - 1) * D * e;
  const Buf ins[] = {{dy, "dy", tok, e, extent(T_total, dy_stride, D, dtype)}, {x, "x", tok, e, extent(T_total, x_stride, D, dtype)},
                     {w0, "w0", false, e, windows}, {dfinal, "dfinal", false, e, windows},
                     {weight, "weight", true, 4, (size_t)D * W * 4}, {bias, "bias", false, 4, (size_t)D * 4},
                     {cu_seqlens, "cu_seqlens", false, 4, ((size_t)N + 1) * 4}};
  const Buf outs[] = {{dx, "dx", tok, e, extent(T_total, D, D, dtype)}, {dweight, "dweight", true, 4, (size_t)D * W * 4},
                      {dbias, "dbias", bias != nullptr, 4, (size_t)D * 4}, {dw0, "dw0", false, e, windows},
                      {workspace, "workspace", true, 16, conv_bytes(T_total, D, W, true)}};
  if (int rc = check_buffers(ins)) return rc;
  if (int rc = check_buffers(outs)) return rc;
  if (int rc = check_overlaps(outs, ins)) return rc;
  hagdn::ConvArgs a = {};
  a.dy = dy; a.dys = dy_stride; a.x = x; a.xs = x_stride; a.w = weight; a.b = bias; a.w0 = w0; a.dfinal = dfinal;
  a.cu = cu_seqlens; a.N = N; a.T = T_total; a.D = D; a.W = W; a.silu = activation == HAGDN_ACT_SILU;
  a.dx = dx; a.dw = dweight; a.db = bias ? dbias : nullptr; a.dw0 = dw0; a.status = static_cast<int *>(workspace);
  a.partial = reinterpret_cast<float *>(static_cast<char *>(workspace) + hagdn::kMixerHeader);
  a.run = hagdn::conv_run(T_total, D, query_cus());
  a.parts = hagdn::conv_parts(T_total, D, query_cus());
  return done(hagdn::launch_conv_backward(a, dtype == HAGDN_BF16, static_cast<hipStream_t>(stream)));
}

int hagdn_conv_decode(const void *x, int64_t x_stride, const float *weight, const float *bias, void *state,
                      const int32_t *slots, int num_slots, int N, int D, int W, int dtype, int activation, void *y,
                      void *stream) {
  if (N < 0) return fail(HAGDN_EINVAL, "N must be >= 0 (got %d)", N);
  if (int rc = check_conv(0, D, W, dtype, activation)) return rc;
  if ((size_t)N * (size_t)D >= 0x7fffffffu) return fail(HAGDN_EINVAL, "N x D too large (%d x %d)", N, D);
  const Stride ss[] = {{x_stride, "x_stride"}};
  if (int rc = check_strides(ss)) return rc;
  if (N == 0) return HAGDN_OK;
  if (!slots) num_slots = N;
  if (num_slots < 1) return fail(HAGDN_EINVAL, "num_slots must be >= 1 (got %d)", num_slots);
  const size_t e = esize(dtype);
  const Buf ins[] = {{x, "x", true, e, extent(N, x_stride, D, dtype)}, {weight, "weight", true, 4, (size_t)D * W * 4},
                     {bias, "bias", false, 4, (size_t)D * 4}, {slots, "slots", false, 4, (size_t)N * 4}};
  const Buf outs[] = {{y, "y", true, e, extent(N, D, D, dtype)},
                      {state, "state", true, e, (size_t)num_slots * (W - 1) * D * e}};
  if (int rc = check_buffers(ins)) return rc;
  if (int rc = check_buffers(outs)) return rc;
  if (int rc = check_overlaps(outs, ins)) return rc;
  hagdn::ConvStepArgs a = {};
  a.x = x; a.xs = x_stride; a.w = weight; a.b = bias; a.state = state; a.slots = slots; a.num_slots = num_slots;
  a.N = N; a.D = D; a.W = W; a.silu = activation == HAGDN_ACT_SILU; a.y = y;
  return done(hagdn::launch_conv_step(a, dtype == HAGDN_BF16, static_cast<hipStream_t>(stream)));
}

size_t ssm_workspace_size(int T_total, int D, int S, int G, int backward) {
  if (check_ssm(T_total, D, S, G, HAGDN_F32, HAGDN_F32, 0) != HAGDN_OK) return 0;
  const SsmPlan p = ssm_plan(T_total, D, S, G, backward != 0);
  return check_fits(p, T_total, D, S, G) == HAGDN_OK ? p.bytes : 0;
}

size_t ssm_checkpoints_size(int T_total, int D, int S) {
  if (check_ssm(T_total, D, S, 1, HAGDN_F32, HAGDN_F32, 0) != HAGDN_OK) return 0;
  return ((size_t)T_total + hagdn::kSsmGroup - 1) / hagdn::kSsmGroup * hagdn::ssm_padded(S) * (size_t)D;
}

int ssm_prefill(const void *x, int64_t x_stride, const void *dt, int64_t dt_stride, const float *A, const void *B,
                int64_t B_stride, const void *C, int64_t C_stride, const float *skip, const void *z, int64_t z_stride,
                const float *dt_bias, const float *s0, const int32_t *cu_seqlens, int N, int T_total, int D, int S, int G,
                int dtype, int dt_dtype, int pre, void *y, float *s_final, float *checkpoints, void *workspace,
                size_t workspace_bytes, void *stream) {
  SsmPlan plan;
  if (int rc = check_ssm_call(cu_seqlens, N, T_total, D, S, G, dtype, dt_dtype, pre, dt_bias, workspace, workspace_bytes, false,
                              &plan))
    return rc;
  const Stride ss[] = {{x_stride, "x_stride"}, {dt_stride, "dt_stride"}, {B_stride, "B_stride"}, {C_stride, "C_stride"},
                       {z_stride, "z_stride"}};
  if (int rc = check_strides(ss)) return rc;
  const bool tok = T_total > 0;
  const size_t e = esize(dtype), states = (size_t)N * D * S * 4, gs = (size_t)G * S;
  const Buf ins[] = {{x, "x", tok, e, extent(T_total, x_stride, D, dtype)},
                     {dt, "dt", tok, esize(dt_dtype), extent(T_total, dt_stride, D, dt_dtype)},
                     {A, "A", true, 4, (size_t)D * S * 4},
                     {B, "B", tok, e, extent(T_total, B_stride, gs, dtype)},
                     {C, "C", tok, e, extent(T_total, C_stride, gs, dtype)},
                     {skip, "skip", false, 4, (size_t)D * 4},
                     {z, "z", false, e, extent(T_total, z_stride, D, dtype)},
                     {dt_bias, "dt_bias", false, 4, (size_t)D * 4},
                     {s0, "s0", false, 4, states},
                     {cu_seqlens, "cu_seqlens", false, 4, ((size_t)N + 1) * 4}};
  const Buf outs[] = {{y, "y", tok, e, extent(T_total, D, D, dtype)},
                      {s_final, "s_final", false, 4, states},
                      {checkpoints, "checkpoints", false, 4, ssm_checkpoints_size(T_total, D, S) * 4},
                      {workspace, "workspace", true, 16, plan.bytes}};
  if (int rc = check_buffers(ins)) return rc;
  if (int rc = check_buffers(outs)) return rc;
  if (int rc = check_overlaps(outs, ins)) return rc;
  hagdn::SsmArgs a = {};
  a.x = x; a.xs = x_stride; a.dt = dt; a.dts = dt_stride; a.A = A; a.B = B; a.Bs = B_stride; a.C = C; a.Cs = C_stride;
  a.skip = skip; a.z = z; a.zs = z_stride; a.bias = dt_bias; a.s0 = s0; a.cu = cu_seqlens;
  a.N = N; a.T = T_total; a.D = D; a.S = S; a.G = G; a.raw = pre != 0;
  a.y = y; a.s_final = s_final; a.ckpt = checkpoints;
  set_plan(&a, plan, workspace);
  return done(hagdn::launch_ssm_forward(a, dtype == HAGDN_BF16, dt_dtype == HAGDN_BF16, static_cast<hipStream_t>(stream)));
}

int ssm_backward(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, const void *dt, int64_t dt_stride,
                 const float *A, const void *B, int64_t B_stride, const void *C, int64_t C_stride, const float *skip,
                 const void *z, int64_t z_stride, const float *dt_bias, const float *checkpoints, const float *s0,
                 const float *dfinal, const int32_t *cu_seqlens, int N, int T_total, int D, int S, int G, int dtype,
                 int dt_dtype, int pre, void *dx, void *ddt, float *dA, void *dB, void *dC, float *dskip, void *dz,
                 float *d_dt_bias, float *ds0, void *workspace, size_t workspace_bytes, void *stream) {
  SsmPlan plan;
  if (int rc = check_ssm_call(cu_seqlens, N, T_total, D, S, G, dtype, dt_dtype, pre, dt_bias, workspace, workspace_bytes, true,
                              &plan))
    return rc;
  const Stride ss[] = {{dy_stride, "dy_stride"}, {x_stride, "x_stride"}, {dt_stride, "dt_stride"},
                       {B_stride, "B_stride"}, {C_stride, "C_stride"}, {z_stride, "z_stride"}};
  if (int rc = check_strides(ss)) return rc;
  const bool tok = T_total > 0;
  const size_t e = esize(dtype), states = (size_t)N * D * S * 4, gs = (size_t)G * S;
  const Buf ins[] = {{dy, "dy", tok, e, extent(T_total, dy_stride, D, dtype)},
                     {x, "x", tok, e, extent(T_total, x_stride, D, dtype)},
                     {dt, "dt", tok, esize(dt_dtype), extent(T_total, dt_stride, D, dt_dtype)},
                     {A, "A", true, 4, (size_t)D * S * 4},
                     {B, "B", tok, e, extent(T_total, B_stride, gs, dtype)},
                     {C, "C", tok, e, extent(T_total, C_stride, gs, dtype)},
                     {skip, "skip", false, 4, (size_t)D * 4},
                     {z, "z", false, e, extent(T_total, z_stride, D, dtype)},
                     {dt_bias, "dt_bias", false, 4, (size_t)D * 4},
                     {checkpoints, "checkpoints", tok, 4, ssm_checkpoints_size(T_total, D, S) * 4},
                     {s0, "s0", false, 4, states},
                     {dfinal, "dfinal", false, 4, states},
                     {cu_seqlens, "cu_seqlens", false, 4, ((size_t)N + 1) * 4}};
  const size_t rows = extent(T_total, D, D, dtype), bc = (size_t)T_total * gs * e;
  const Buf outs[] = {{dx, "dx", tok, e, rows},
                      {ddt, "ddt", tok, esize(dt_dtype), extent(T_total, D, D, dt_dtype)},
                      {dA, "dA", true, 4, (size_t)D * S * 4},
                      {dB, "dB", tok, e, bc},
                      {dC, "dC", tok, e, bc},
                      {dskip, "dskip", skip != nullptr, 4, (size_t)D * 4},
                      {dz, "dz", tok && z != nullptr, e, rows},
                      {d_dt_bias, "d_dt_bias", dt_bias != nullptr, 4, (size_t)D * 4},
                      {ds0, "ds0", false, 4, states},
                      {workspace, "workspace", true, 16, plan.bytes}};
  if (int rc = check_buffers(ins)) return rc;
  if (int rc = check_buffers(outs)) return rc;
  if (int rc = check_overlaps(outs, ins)) return rc;
  hagdn::SsmArgs a = {};
  a.dy = dy; a.dys = dy_stride; a.x = x; a.xs = x_stride; a.dt = dt; a.dts = dt_stride; a.A = A; a.B = B; a.Bs = B_stride;
  a.C = C; a.Cs = C_stride; a.skip = skip; a.z = z; a.zs = z_stride; a.bias = dt_bias; a.s0 = s0; a.dfinal = dfinal;
  a.cu = cu_seqlens; a.N = N; a.T = T_total; a.D = D; a.S = S; a.G = G; a.raw = pre != 0;
  a.ckpt = const_cast<float *>(checkpoints);
  a.dx = dx; a.ddt = ddt; a.dA = dA; a.dB = dB; a.dC = dC; a.dskip = skip ? dskip : nullptr; a.dz = dz;
  a.dbias = dt_bias ? d_dt_bias : nullptr; a.ds0 = ds0;
  set_plan(&a, plan, workspace);
  return done(hagdn::launch_ssm_backward(a, dtype == HAGDN_BF16, dt_dtype == HAGDN_BF16, static_cast<hipStream_t>(stream)));
}

int ssm_decode(const void *x, int64_t x_stride, const void *dt, int64_t dt_stride, const float *A, const void *B,
               int64_t B_stride, const void *C, int64_t C_stride, const float *skip, const void *z, int64_t z_stride,
               const float *dt_bias, float *state, const int32_t *slots, int num_slots, int N, int D, int S, int G,
               int dtype, int dt_dtype, int pre, void *y, void *stream) {
  if (N < 0) return fail(HAGDN_EINVAL, "N must be >= 0 (got %d)", N);
  if (int rc = check_ssm(0, D, S, G, dtype, dt_dtype, pre)) return rc;
  if ((size_t)N * (size_t)D * (size_t)S >= 0x7fffffffu) return fail(HAGDN_EINVAL, "N x D x S too large (%d x %d x %d)", N, D, S);
  if (dt_bias && !pre) return fail(HAGDN_EINVAL, "dt_bias needs HAGDN_PRE_GATE_SOFTPLUS");
  const Stride ss[] = {{x_stride, "x_stride"}, {dt_stride, "dt_stride"}, {B_stride, "B_stride"}, {C_stride, "C_stride"},
                       {z_stride, "z_stride"}};
  if (int rc = check_strides(ss)) return rc;
  if (N == 0) return HAGDN_OK;
  if (!slots) num_slots = N;
  if (num_slots < 1) return fail(HAGDN_EINVAL, "num_slots must be >= 1 (got %d)", num_slots);
  const size_t e = esize(dtype), gs = (size_t)G * S;
  const Buf ins[] = {{x, "x", true, e, extent(N, x_stride, D, dtype)},
                     {dt, "dt", true, esize(dt_dtype), extent(N, dt_stride, D, dt_dtype)},
                     {A, "A", true, 4, (size_t)D * S * 4},
                     {B, "B", true, e, extent(N, B_stride, gs, dtype)},
                     {C, "C", true, e, extent(N, C_stride, gs, dtype)},
                     {skip, "skip", false, 4, (size_t)D * 4},
                     {z, "z", false, e, extent(N, z_stride, D, dtype)},
                     {dt_bias, "dt_bias", false, 4, (size_t)D * 4},
                     {slots, "slots", false, 4, (size_t)N * 4}};
  const Buf outs[] = {{y, "y", true, e, extent(N, D, D, dtype)}, {state, "state", true, 4, (size_t)num_slots * D * S * 4}};
  if (int rc = check_buffers(ins)) return rc;
  if (int rc = check_buffers(outs)) return rc;
  if (int rc = check_overlaps(outs, ins)) return rc;
  hagdn::SsmStepArgs a = {};
  a.x = x; a.xs = x_stride; a.dt = dt; a.dts = dt_stride; a.A = A; a.B = B; a.Bs = B_stride; a.C = C; a.Cs = C_stride;
  a.skip = skip; a.z = z; a.zs = z_stride; a.bias = dt_bias; a.state = state; a.slots = slots; a.num_slots = num_slots;
  a.N = N; a.D = D; a.S = S; a.G = G; a.raw = pre != 0; a.y = y;
  return done(hagdn::launch_ssm_step(a, dtype == HAGDN_BF16, dt_dtype == HAGDN_BF16, static_cast<hipStream_t>(stream)));
}

int hagdn_pool_copy(void *const *pools, const void *const *sources, const size_t *row_bytes, int num_pools,
                    const int32_t *dst_slots, const int32_t *src_slots, int n, int dst_rows, int src_rows, void *stream) {
  if (int rc = check_pools(pools, row_bytes, num_pools)) return rc;
  if (!sources) src_rows = dst_rows;
  if (n < 0 || dst_rows < 0 || src_rows < 0)
    return fail(HAGDN_EINVAL, "n, dst_rows and src_rows must be >= 0 (got %d, %d, %d)", n, dst_rows, src_rows);
  if (!sources && n > hagdn::kMaxMovesInPlace)
    return fail(HAGDN_EUNSUPPORTED, "n > %d unsupported without sources (got %d)", hagdn::kMaxMovesInPlace, n);
  if (sources)
    for (int p = 0; p < num_pools; ++p)
      if (!sources[p]) return fail(HAGDN_EINVAL, "NULL required pointer sources[%d]", p);
  const Buf tables[] = {{dst_slots, "dst_slots", false, 4, 0}, {src_slots, "src_slots", false, 4, 0}};
  if (int rc = check_buffers(tables)) return rc;
  if (int rc = check_ranges(pools, sources, row_bytes, num_pools, dst_rows, src_rows)) return rc;
  for (int p = 0; p < num_pools; ++p)
    for (const int32_t *t : {dst_slots, src_slots})
      if (overlap(pools[p], row_bytes[p] * (size_t)dst_rows, t, (size_t)n * 4)) return fail(HAGDN_EINVAL, "a table overlaps pools[%d]", p);
  if (n == 0 || dst_rows == 0) return HAGDN_OK;
  hagdn::PoolCopyArgs a = {};
  a.dst = dst_slots; a.src = src_slots; a.n = n; a.dst_rows = dst_rows; a.src_rows = src_rows;
  return launch_copies(a, pools, sources, row_bytes, num_pools, !sources, static_cast<hipStream_t>(stream));
}

size_t hagdn_pool_workspace_size(int num_slots) {
  if (num_slots < 1 || num_slots > hagdn::kMaxPoolSlots) {
    fail(HAGDN_EINVAL, "num_slots out of range (got %d)", num_slots);
    return 0;
  }
  return plan_bytes(num_slots);
}

int hagdn_pool_fork(void *const *pools, const size_t *row_bytes, int num_pools, const int32_t *slots, int N,
                    const int32_t *parents, int M, int num_slots, int32_t *new_slots, void *workspace,
                    size_t workspace_bytes, void *stream) {
  if (int rc = check_plan(pools, row_bytes, num_pools, num_slots, workspace, workspace_bytes)) return rc;
  if (N < 0 || M < 0) return fail(HAGDN_EINVAL, "N and M must be >= 0 (got %d, %d)", N, M);
  if (M > hagdn::kMaxPoolSlots) return fail(HAGDN_EUNSUPPORTED, "M > %d unsupported (got %d)", hagdn::kMaxPoolSlots, M);
  const Buf ins[] = {{slots, "slots", N > 0, 4, (size_t)N * 4}, {parents, "parents", M > 0, 4, (size_t)M * 4}};
  const Buf outs[] = {{new_slots, "new_slots", M > 0, 4, (size_t)M * 4}};
  if (int rc = check_buffers(ins)) return rc;
  if (int rc = check_buffers(outs)) return rc;
  if (int rc = check_overlaps(outs, ins)) return rc;
  const Buf tables[] = {ins[0], ins[1], outs[0]};
  if (int rc = check_plan_overlaps(pools, row_bytes, num_pools, num_slots, tables, workspace)) return rc;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  hagdn::PoolPlanArgs plan = plan_args(slots, N, num_slots, new_slots, workspace);
  plan.parents = parents;
  plan.M = M;
  if (hipError_t e = hagdn::launch_pool_fork_plan(plan, s)) return done(e);
  hagdn::PoolCopyArgs a = {};
  a.moves = plan.moves;
  a.n = M < num_slots ? M : num_slots;  // at most
  a.dst_rows = a.src_rows = num_slots;
  return a.n > 0 ? launch_copies(a, pools, nullptr, row_bytes, num_pools, false, s) : HAGDN_OK;
}

int hagdn_pool_compact(void *const *pools, const size_t *row_bytes, int num_pools, const int32_t *slots, int N,
                       int num_slots, int32_t *new_slots, void *workspace, size_t workspace_bytes, void *stream) {
  if (int rc = check_plan(pools, row_bytes, num_pools, num_slots, workspace, workspace_bytes)) return rc;
  if (N < 0) return fail(HAGDN_EINVAL, "N must be >= 0 (got %d)", N);
  if (N > hagdn::kMaxPoolSlots) return fail(HAGDN_EUNSUPPORTED, "N > %d unsupported (got %d)", hagdn::kMaxPoolSlots, N);
  const Buf tables[] = {{slots, "slots", N > 0, 4, (size_t)N * 4}, {new_slots, "new_slots", N > 0, 4, (size_t)N * 4}};
  if (int rc = check_buffers(tables)) return rc;
  if (new_slots != slots && overlap(new_slots, (size_t)N * 4, slots, (size_t)N * 4))
    return fail(HAGDN_EINVAL, "new_slots overlaps slots partly");
  if (int rc = check_plan_overlaps(pools, row_bytes, num_pools, num_slots, tables, workspace)) return rc;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const hagdn::PoolPlanArgs plan = plan_args(slots, N, num_slots, new_slots, workspace);
  if (hipError_t e = hagdn::launch_pool_compact_plan(plan, s)) return done(e);
  hagdn::PoolCopyArgs a = {};
  a.moves = plan.moves;
  a.n = N < num_slots / 2 ? N : num_slots / 2;  // at most: as many holes as states behind them
  a.dst_rows = a.src_rows = num_slots;
  return a.n > 0 ? launch_copies(a, pools, nullptr, row_bytes, num_pools, false, s) : HAGDN_OK;
}

}  // extern "C"

// api_layer.cpp -- the C ABI of the gated linear recurrence and the block norms
// (include/hagdn.h): host-side argument checks, then the launches on the caller's
// stream.  No allocation, no synchronisation, no pointer retained after return.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include "hagdn.h"
#include "layer.h"
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

bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }

// A device pointer argument: its name, whether it must not be NULL, its alignment.
struct Ptr {
  const void *p;
  const char *name;
  bool required;
  size_t align;
};
template <size_t N> int check_pointers(const Ptr (&ps)[N]) {
  for (const Ptr &a : ps) {
    if (a.required && !a.p) return fail(HAGDN_EINVAL, "NULL required pointer %s", a.name);
    if (!aligned(a.p, a.align)) return fail(HAGDN_EINVAL, "%s must be %zu-byte aligned", a.name, a.align);
  }
  return HAGDN_OK;
}

// Row strides in elements; below 2^31 so that row x stride stays far inside 64 bits.
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

int check_dtypes(int dtype, int other, const char *what) {
  if (dtype != HAGDN_F32 && dtype != HAGDN_BF16) return fail(HAGDN_EUNSUPPORTED, "dtype %d unsupported", dtype);
  if (other != HAGDN_F32 && !(other == HAGDN_BF16 && dtype == HAGDN_BF16))
    return fail(HAGDN_EUNSUPPORTED, "%s dtype %d unsupported with dtype %d", what, other, dtype);
  return HAGDN_OK;
}

size_t esize(int dtype) { return dtype == HAGDN_BF16 ? 2 : 4; }

// a and b, `bytes` each, overlap without being the same buffer.
bool partly_aliased(const void *a, const void *b, size_t bytes) {
  const char *p = static_cast<const char *>(a), *q = static_cast<const char *>(b);
  return p && q && p != q && p < q + bytes && q < p + bytes;
}

// ---------------------------------------------------------------- recurrence
int check_glr(int N, int T, int D, int dtype, int gate_dtype, int convex, int pre) {
  if (T < 0) return fail(HAGDN_EINVAL, "T_total must be >= 0 (got %d)", T);
  if (D < 1) return fail(HAGDN_EINVAL, "D must be >= 1 (got %d)", D);
  if (D > (1 << 28)) return fail(HAGDN_EUNSUPPORTED, "D > 2^28 unsupported");  // 32-bit offsets within a row
  if ((size_t)N * (size_t)D >= 0x7fffffffu) return fail(HAGDN_EINVAL, "N x D too large (%d x %d)", N, D);
  if (convex != 0 && convex != 1) return fail(HAGDN_EINVAL, "convex must be 0 or 1 (got %d)", convex);
  if (pre & ~hagdn::kPreGateSoftplus) return fail(HAGDN_EINVAL, "unsupported preprocessing flags 0x%x", pre);
  return check_dtypes(dtype, gate_dtype, "gate");
}

// Workspace of a call in either direction: the header and, where some tiles' words are
// needed, the counters and the words of the smallest tiles.
size_t glr_bytes(int T, int D) {
  const size_t tiles = ((size_t)T + hagdn::kGlrLeastTile - 1) / hagdn::kGlrLeastTile;
  return hagdn::kGlrHeader + (tiles > 1 ? hagdn::glr_counter_bytes(D) + tiles * (size_t)D * 8 : 0);  // below 2^60
}

// Sizes, the sequences and the workspace, shared by the forward and backward calls.
int check_glr_call(const int32_t *cu, int N, int T, int D, int dtype, int gate_dtype, int convex, int pre,
                   const void *ws, size_t ws_bytes) {
  if (N < 1) return fail(HAGDN_EINVAL, "N must be >= 1 (got %d)", N);
  if (int rc = check_glr(N, T, D, dtype, gate_dtype, convex, pre)) return rc;
  if (!cu && N != 1) return fail(HAGDN_EINVAL, "cu_seqlens may be NULL for one sequence only (N = %d)", N);
  const Ptr ps[] = {{cu, "cu_seqlens", false, 4}, {ws, "workspace", true, 16}};
  if (int rc = check_pointers(ps)) return rc;
  const size_t need = glr_bytes(T, D);
  if (ws_bytes < need) return fail(HAGDN_EWORKSPACE, "workspace too small: %zu bytes, need %zu", ws_bytes, need);
  return HAGDN_OK;
}

void set_workspace(hagdn::GlrArgs *a, void *ws) {
  char *p = static_cast<char *>(ws);
  a->cus = hagdn::device_cus();
  a->status = reinterpret_cast<int *>(p);
  a->counters = reinterpret_cast<uint32_t *>(p + hagdn::kGlrHeader);
  a->words = reinterpret_cast<uint64_t *>(p + hagdn::kGlrHeader + hagdn::glr_counter_bytes(a->D));
}

hagdn::GlrForm form(int dtype, int gate_dtype, int convex, int pre) {
  return {dtype == HAGDN_BF16, gate_dtype == HAGDN_BF16, (pre & hagdn::kPreGateSoftplus) != 0, convex != 0};
}

// --------------------------------------------------------------------- norms
using hagdn::kMaxNormDim;

int check_rows(int T, long per_token, int d, float eps) {
  if (T < 0) return fail(HAGDN_EINVAL, "T must be >= 0 (got %d)", T);
  if (d < 1) return fail(HAGDN_EINVAL, "rows must have at least one element (got %d)", d);
  if (d > kMaxNormDim) return fail(HAGDN_EUNSUPPORTED, "rows of more than %d elements unsupported (got %d)", kMaxNormDim, d);
  if (per_token < 1 || (size_t)per_token * (size_t)(T > 0 ? T : 1) > 0x7fffffffu)
    return fail(HAGDN_EINVAL, "head count out of range");
  if (!(eps >= 0.f) || !isfinite(eps)) return fail(HAGDN_EINVAL, "eps must be finite and >= 0");
  return HAGDN_OK;
}

size_t partial_bytes(long rows, int cols, int cus) {
  return (size_t)hagdn::norm_parts(rows, cus) * (size_t)cols * sizeof(float);
}

int query_cus() {
  const int n = hagdn::device_cus();
  return n > 0 ? n : 256;  // no device: sizes as for an MI355X
}

}  // namespace

extern "C" {

size_t glr_workspace_size(int T_total, int D) {
  if (check_glr(1, T_total, D, HAGDN_F32, HAGDN_F32, 0, 0) != HAGDN_OK) return 0;
  return glr_bytes(T_total, D);
}

int glr_prefill(const void *x, int64_t x_stride, const void *g, int64_t g_stride, const float *s0,
                const int32_t *cu_seqlens, int N, int T_total, int D, int dtype, int gate_dtype, int convex, int pre,
                void *h, float *s_final, float *checkpoints, void *workspace, size_t workspace_bytes, void *stream) {
  if (int rc = check_glr_call(cu_seqlens, N, T_total, D, dtype, gate_dtype, convex, pre, workspace, workspace_bytes))
    return rc;
  const bool tok = T_total > 0;
  const Ptr ps[] = {{x, "x", tok, esize(dtype)}, {g, "g", tok, esize(gate_dtype)}, {h, "h", tok, esize(dtype)},
                    {s0, "s0", false, 4}, {s_final, "s_final", false, 4}, {checkpoints, "checkpoints", false, 4}};
  if (int rc = check_pointers(ps)) return rc;
  const Stride ss[] = {{x_stride, "x_stride"}, {g_stride, "g_stride"}};
  if (int rc = check_strides(ss)) return rc;
  if (partly_aliased(s0, s_final, (size_t)N * D * 4)) return fail(HAGDN_EINVAL, "s_final overlaps s0 partly");
  hagdn::GlrArgs a = {};
  a.x = x; a.g = g; a.xs = x_stride; a.gs = g_stride; a.s0 = s0; a.cu = cu_seqlens;
  a.N = N; a.T = T_total; a.D = D; a.h = h; a.s_final = s_final; a.ckpt = checkpoints;
  set_workspace(&a, workspace);
  return done(hagdn::launch_glr_forward(a, form(dtype, gate_dtype, convex, pre), static_cast<hipStream_t>(stream)));
}

int glr_backward(const void *dh, int64_t dh_stride, const void *x, int64_t x_stride, const void *g, int64_t g_stride,
                 const float *checkpoints, const float *s0, const float *dfinal, const int32_t *cu_seqlens, int N,
                 int T_total, int D, int dtype, int gate_dtype, int convex, int pre, void *dx, void *dg, float *ds0,
                 void *workspace, size_t workspace_bytes, void *stream) {
  if (int rc = check_glr_call(cu_seqlens, N, T_total, D, dtype, gate_dtype, convex, pre, workspace, workspace_bytes))
    return rc;
  const bool tok = T_total > 0;
  const Ptr ps[] = {{dh, "dh", tok, esize(dtype)}, {x, "x", tok, esize(dtype)}, {g, "g", tok, esize(gate_dtype)},
                    {checkpoints, "checkpoints", tok, 4}, {dx, "dx", tok, esize(dtype)}, {dg, "dg", tok, esize(gate_dtype)},
                    {s0, "s0", false, 4}, {dfinal, "dfinal", false, 4}, {ds0, "ds0", false, 4}};
  if (int rc = check_pointers(ps)) return rc;
  const Stride ss[] = {{dh_stride, "dh_stride"}, {x_stride, "x_stride"}, {g_stride, "g_stride"}};
  if (int rc = check_strides(ss)) return rc;
  if (partly_aliased(dfinal, ds0, (size_t)N * D * 4)) return fail(HAGDN_EINVAL, "ds0 overlaps dfinal partly");
  hagdn::GlrArgs a = {};
  a.x = x; a.g = g; a.dh = dh; a.xs = x_stride; a.gs = g_stride; a.dhs = dh_stride; a.s0 = s0; a.dfinal = dfinal;
  a.cu = cu_seqlens; a.N = N; a.T = T_total; a.D = D; a.dx = dx; a.dg = dg; a.ds0 = ds0;
  a.ckpt = const_cast<float *>(checkpoints);
  set_workspace(&a, workspace);
  return done(hagdn::launch_glr_backward(a, form(dtype, gate_dtype, convex, pre), static_cast<hipStream_t>(stream)));
}

int glr_decode(const void *x, int64_t x_stride, const void *g, int64_t g_stride, float *state, const int32_t *slots,
               int num_slots, int N, int D, int dtype, int gate_dtype, int convex, int pre, void *h, void *stream) {
  if (N < 0) return fail(HAGDN_EINVAL, "N must be >= 0 (got %d)", N);
  if (int rc = check_glr(N, 0, D, dtype, gate_dtype, convex, pre)) return rc;
  if (N == 0) return HAGDN_OK;
  if (!slots) num_slots = N;
  if (num_slots < 1) return fail(HAGDN_EINVAL, "num_slots must be >= 1 (got %d)", num_slots);
  const Ptr ps[] = {{x, "x", true, esize(dtype)}, {g, "g", true, esize(gate_dtype)}, {state, "state", true, 4},
                    {h, "h", true, esize(dtype)}, {slots, "slots", false, 4}};
  if (int rc = check_pointers(ps)) return rc;
  const Stride ss[] = {{x_stride, "x_stride"}, {g_stride, "g_stride"}};
  if (int rc = check_strides(ss)) return rc;
  hagdn::GlrStepArgs a = {};
  a.x = x; a.g = g; a.xs = x_stride; a.gs = g_stride; a.state = state; a.slots = slots;
  a.num_slots = num_slots; a.N = N; a.D = D; a.h = h;
  return done(hagdn::launch_glr_step(a, form(dtype, gate_dtype, convex, pre), static_cast<hipStream_t>(stream)));
}

int hagdn_add_norm(const void *x, int64_t x_stride, const void *res, int64_t res_stride, const float *weight,
                   const float *post_weight, const float *scale_vec, float scale, float eps, int T, int D, int dtype,
                   int res_dtype, void *y, void *res_out, void *stream) {
  if (int rc = check_rows(T, 1, D, eps)) return rc;
  if (int rc = check_dtypes(dtype, res_dtype, "residual")) return rc;
  if (T == 0) return HAGDN_OK;
  const Ptr ps[] = {{x, "x", true, esize(dtype)}, {res, "res", false, esize(res_dtype)}, {weight, "weight", true, 4},
                    {post_weight, "post_weight", false, 4}, {scale_vec, "scale_vec", false, 4},
                    {y, "y", true, esize(dtype)}, {res_out, "res_out", false, esize(res_dtype)}};
  if (int rc = check_pointers(ps)) return rc;
  const Stride ss[] = {{x_stride, "x_stride"}, {res_stride, "res_stride"}};
  if (int rc = check_strides(ss)) return rc;
  if (res && res == res_out && T > 1 && res_stride != D) return fail(HAGDN_EINVAL, "res_out is res, which is not contiguous");
  hagdn::AddNormArgs a = {};
  a.x = x; a.xs = x_stride; a.res = res; a.rs = res_stride; a.w = weight; a.post = post_weight; a.scale_vec = scale_vec;
  a.scale = scale; a.eps = eps; a.T = T; a.D = D; a.y = y; a.res_out = res_out;
  return done(hagdn::launch_add_norm(a, dtype == HAGDN_BF16, res_dtype == HAGDN_BF16, static_cast<hipStream_t>(stream)));
}

size_t hagdn_add_norm_workspace_size(int T, int D, int has_scale_vec, int has_post) {
  if (check_rows(T, 1, D, 0.f) != HAGDN_OK) return 0;
  return partial_bytes(T, D * (1 + (has_scale_vec != 0) + (has_post != 0)), query_cus());
}

int hagdn_add_norm_backward(const void *dy, int64_t dy_stride, const void *dres, int64_t dres_stride, const void *res,
                            int64_t res_stride, const void *x, int64_t x_stride, const float *weight,
                            const float *post_weight, const float *scale_vec, float scale, float eps, int T, int D,
                            int dtype, int res_dtype, void *dx, void *dres_out, float *dweight, float *dscale,
                            float *dpost, void *workspace, size_t workspace_bytes, void *stream) {
  if (int rc = check_rows(T, 1, D, eps)) return rc;
  if (int rc = check_dtypes(dtype, res_dtype, "residual")) return rc;
  const bool tok = T > 0, vec = scale_vec != nullptr, post = post_weight != nullptr;
  const Ptr ps[] = {{dy, "dy", tok, esize(dtype)}, {dres, "dres", false, esize(res_dtype)},
                    {res, "res", tok, esize(res_dtype)}, {x, "x", tok && (vec || post), esize(dtype)},
                    {weight, "weight", true, 4}, {post_weight, "post_weight", false, 4},
                    {scale_vec, "scale_vec", false, 4}, {dx, "dx", tok, esize(dtype)},
                    {dres_out, "dres_out", false, esize(res_dtype)}, {dweight, "dweight", true, 4},
                    {dscale, "dscale", vec, 4}, {dpost, "dpost", post, 4}, {workspace, "workspace", true, 16}};
  if (int rc = check_pointers(ps)) return rc;
  const Stride ss[] = {{dy_stride, "dy_stride"}, {dres_stride, "dres_stride"}, {res_stride, "res_stride"},
                       {x_stride, "x_stride"}};
  if (int rc = check_strides(ss)) return rc;
  if (dres && dres == dres_out && T > 1 && dres_stride != D)
    return fail(HAGDN_EINVAL, "dres_out is dres, which is not contiguous");
  const int cus = query_cus();
  const size_t need = partial_bytes(T, D * (1 + vec + post), cus);
  if (workspace_bytes < need)
    return fail(HAGDN_EWORKSPACE, "workspace too small: %zu bytes, need %zu", workspace_bytes, need);
  hagdn::AddNormArgs a = {};
  a.dy = dy; a.dys = dy_stride; a.dres = dres; a.drs = dres_stride; a.res = res; a.rs = res_stride;
  a.x = vec || post ? x : nullptr; a.xs = x_stride;
  a.w = weight; a.post = post_weight; a.scale_vec = scale_vec; a.scale = scale; a.eps = eps; a.T = T; a.D = D;
  a.dx = dx; a.dres_out = dres_out; a.dw = dweight; a.dscale = vec ? dscale : nullptr; a.dpost = post ? dpost : nullptr;
  a.partial = static_cast<float *>(workspace); a.parts = hagdn::norm_parts(T, cus);
  return done(hagdn::launch_add_norm_backward(a, dtype == HAGDN_BF16, res_dtype == HAGDN_BF16,
                                              static_cast<hipStream_t>(stream)));
}

int hagdn_gate_norm(const void *o, int64_t o_stride, const void *z, int64_t z_stride, const float *weight, float eps,
                    int T, int H, int d, int dtype, int activation, void *y, void *stream) {
  if (int rc = check_rows(T, H, d, eps)) return rc;
  if (int rc = check_dtypes(dtype, HAGDN_F32, "weight")) return rc;
  if (activation != HAGDN_ACT_SILU && activation != HAGDN_ACT_SIGMOID)
    return fail(HAGDN_EINVAL, "unknown activation %d", activation);
  if (T == 0) return HAGDN_OK;
  const size_t e = esize(dtype);
  const Ptr ps[] = {{o, "o", true, e}, {z, "z", true, e}, {weight, "weight", true, 4}, {y, "y", true, e}};
  if (int rc = check_pointers(ps)) return rc;
  const Stride ss[] = {{o_stride, "o_stride"}, {z_stride, "z_stride"}};
  if (int rc = check_strides(ss)) return rc;
  hagdn::GateNormArgs a = {};
  a.o = o; a.os = o_stride; a.z = z; a.zs = z_stride; a.w = weight; a.eps = eps; a.T = T; a.H = H; a.d = d;
  a.silu = activation == HAGDN_ACT_SILU; a.y = y;
  return done(hagdn::launch_gate_norm(a, dtype == HAGDN_BF16, static_cast<hipStream_t>(stream)));
}

size_t hagdn_gate_norm_workspace_size(int T, int H, int d) {
  if (check_rows(T, H, d, 0.f) != HAGDN_OK) return 0;
  return partial_bytes((long)T * H, d, query_cus());
}

int hagdn_gate_norm_backward(const void *dy, int64_t dy_stride, const void *o, int64_t o_stride, const void *z,
                             int64_t z_stride, const float *weight, float eps, int T, int H, int d, int dtype,
                             int activation, void *d_o, void *d_z, float *dweight, void *workspace,
                             size_t workspace_bytes, void *stream) {
  if (int rc = check_rows(T, H, d, eps)) return rc;
  if (int rc = check_dtypes(dtype, HAGDN_F32, "weight")) return rc;
  if (activation != HAGDN_ACT_SILU && activation != HAGDN_ACT_SIGMOID)
    return fail(HAGDN_EINVAL, "unknown activation %d", activation);
  const size_t e = esize(dtype);
  const bool tok = T > 0;
  const Ptr ps[] = {{dy, "dy", tok, e}, {o, "o", tok, e}, {z, "z", tok, e}, {weight, "weight", true, 4},
                    {d_o, "d_o", tok, e}, {d_z, "d_z", tok, e}, {dweight, "dweight", true, 4},
                    {workspace, "workspace", true, 16}};
  if (int rc = check_pointers(ps)) return rc;
  const Stride ss[] = {{dy_stride, "dy_stride"}, {o_stride, "o_stride"}, {z_stride, "z_stride"}};
  if (int rc = check_strides(ss)) return rc;
  const int cus = query_cus();
  const size_t need = partial_bytes((long)T * H, d, cus);
  if (workspace_bytes < need)
    return fail(HAGDN_EWORKSPACE, "workspace too small: %zu bytes, need %zu", workspace_bytes, need);
  hagdn::GateNormArgs a = {};
  a.dy = dy; a.dys = dy_stride; a.o = o; a.os = o_stride; a.z = z; a.zs = z_stride; a.w = weight; a.eps = eps;
  a.T = T; a.H = H; a.d = d; a.silu = activation == HAGDN_ACT_SILU; a.dout = d_o; a.dz = d_z; a.dw = dweight;
  a.partial = static_cast<float *>(workspace); a.parts = hagdn::norm_parts((long)T * H, cus);
  return done(hagdn::launch_gate_norm_backward(a, dtype == HAGDN_BF16, static_cast<hipStream_t>(stream)));
}

}  // extern "C"

// C ABI of the sequence operators: argument validation and workspaces.  Every entry point
// validates on the host first and returns before enqueuing anything when an argument is wrong.
#include <cmath>
#include <cstdlib>
#include <utility>

#include "fdc.h"
#include "sequence.h"
#include "status.h"

using fdc::check_hip;
using fdc::fail;

namespace {

constexpr int64_t kMaxTokenStride = 1LL << 25;
constexpr int64_t kMaxElements = 1LL << 46;  // of a tensor, and of a batch stride: products stay far below 2^63

fdc_status check_dtype(int dtype) {
  if (dtype != FDC_F32 && dtype != FDC_BF16 && dtype != FDC_F16)
    return fail(FDC_EINVAL, "dtype must be FDC_F32, FDC_BF16 or FDC_F16 (got %d)", dtype);
  return FDC_OK;
}

// A [B][L][width] tensor: present (unless `optional`), strides in range, and an output's elements apart.
fdc_status check_tokens(const fdc_tokens &t, const char *name, int B, int L, int64_t width, bool output,
                        bool optional = false) {
  if (t.p == nullptr) return optional ? FDC_OK : fail(FDC_EINVAL, "%s is NULL", name);
  if (t.batch_stride < 0 || t.token_stride < 0)
    return fail(FDC_EINVAL, "%s: strides must not be negative (got %lld, %lld)", name, (long long)t.batch_stride,
                (long long)t.token_stride);
  if (t.token_stride >= kMaxTokenStride || t.batch_stride >= kMaxElements)
    return fail(FDC_EUNSUPPORTED, "%s: strides %lld, %lld too large", name, (long long)t.batch_stride,
                (long long)t.token_stride);
  if (output) {
    const int64_t inner = (int64_t)(L - 1) * t.token_stride + width, outer = (int64_t)(B - 1) * t.batch_stride + width;
    const bool tokens_in_batch = (L == 1 || t.token_stride >= width) && (B == 1 || t.batch_stride >= inner);
    const bool batch_in_token = (B == 1 || t.batch_stride >= width) && (L == 1 || t.token_stride >= outer);
    if (!tokens_in_batch && !batch_in_token)
      return fail(FDC_EINVAL, "%s is an output whose elements overlap (strides %lld, %lld)", name,
                  (long long)t.batch_stride, (long long)t.token_stride);
  }
  return FDC_OK;
}

// Whether the rows of an output (whose elements are apart) and of an input of the same strides share memory:
// some db * outer + dt * inner + dc, rows' distances and an element's within them, is the distance of the two.  With
// other strides only the same address is seen.  `same`: it is the input itself that is written.
struct Sharing {
  bool any, same;
};
Sharing sharing(const fdc_tokens &out, int64_t out_width, const fdc_tokens &in, int64_t in_width, int64_t B, int64_t L,
                size_t size) {
  if (out.p == nullptr || in.p == nullptr) return {false, false};
  if ((B > 1 && out.batch_stride != in.batch_stride) || (L > 1 && out.token_stride != in.token_stride))
    return {out.p == in.p, false};
  if (out.p == in.p) return {true, out_width == in_width};
  struct Axis {
    int64_t count, stride;
  } outer{B, out.batch_stride * (int64_t)size}, inner{L, out.token_stride * (int64_t)size};
  if (outer.count == 1 || (inner.count > 1 && inner.stride > outer.stride)) std::swap(outer, inner);
  // the (at most two) steps along an axis that leave less than its stride of a distance, either way
  auto any_step = [](const Axis &x, int64_t distance, auto &&rest_shares) {
    if (x.count == 1) return rest_shares(distance);
    const int64_t step = distance / x.stride, next = distance < 0 ? step - 1 : step + 1;
    return (std::abs(step) < x.count && rest_shares(distance - step * x.stride)) ||
           (std::abs(next) < x.count && rest_shares(distance - next * x.stride));
  };
  const int64_t distance = (int64_t)(reinterpret_cast<uintptr_t>(out.p) - reinterpret_cast<uintptr_t>(in.p));
  const bool any = any_step(outer, distance, [&](int64_t d) {
    return any_step(inner, d, [&](int64_t c) { return c < in_width * (int64_t)size && -c < out_width * (int64_t)size; });
  });
  return {any, false};
}

// `itself`: the output may be the whole of that input.
fdc_status check_apart(const fdc_tokens &out, const char *out_name, int64_t out_width, const fdc_tokens &in,
                       const char *in_name, int64_t in_width, int64_t B, int64_t L, int dtype, bool itself) {
  const Sharing sh = sharing(out, out_width, in, in_width, B, L, fdc::dtype_size(dtype));
  if (sh.any && !(itself && sh.same)) return fail(FDC_EINVAL, "%s shares memory with %s", out_name, in_name);
  return FDC_OK;
}

// The same of dense arrays.
fdc_status check_apart(const void *out, const void *in, size_t bytes, const char *what) {
  const uintptr_t o = reinterpret_cast<uintptr_t>(out), i = reinterpret_cast<uintptr_t>(in);
  if (out != nullptr && in != nullptr && o != i && o < i + bytes && i < o + bytes)
    return fail(FDC_EINVAL, "%s share memory in part", what);
  return FDC_OK;
}

fdc_status check_sizes(int B, int L, int D) {
  if (B < 1 || L < 1 || D < 1) return fail(FDC_EINVAL, "B, L and D must be positive (got %d, %d, %d)", B, L, D);
  if (B > 65535) return fail(FDC_EUNSUPPORTED, "B = %d exceeds 65535", B);
  if (D > (1 << 20)) return fail(FDC_EUNSUPPORTED, "D = %d exceeds 2^20", D);
  if (L > (1 << 28)) return fail(FDC_EUNSUPPORTED, "L = %d exceeds 2^28", L);
  return FDC_OK;
}

#define FDC_TRY(expr) \
  if (fdc_status st_ = (expr)) return st_

// ---- causal convolution ------------------------------------------------------
fdc_status check_conv_sizes(int dtype, int B, int L, int D, int n) {
  FDC_TRY(check_dtype(dtype));
  FDC_TRY(check_sizes(B, L, D));
  if (n < 1) return fail(FDC_EINVAL, "n must be positive (got %d)", n);
  if (n > fdc::kConvMaxTaps) return fail(FDC_EUNSUPPORTED, "n = %d taps: at most %d", n, fdc::kConvMaxTaps);
  // a sequence's threads in one grid dimension: at least 8 tokens and 4 channels each
  if (fdc::ceil_div(L, 8) * fdc::ceil_div(D, 4) >= (1LL << 32) - 256)
    return fail(FDC_EUNSUPPORTED, "L = %d times D = %d exceeds the launch limit", L, D);
  return FDC_OK;
}

fdc_status check_conv(const fdc_causal_conv_args *a) {
  if (a == nullptr) return fail(FDC_EINVAL, "arguments are NULL");
  FDC_TRY(check_conv_sizes(a->dtype, a->B, a->L, a->D, a->n));
  FDC_TRY(check_tokens(a->x, "x", a->B, a->L, a->D, false));
  if (!a->w) return fail(FDC_EINVAL, "w is NULL");
  return FDC_OK;
}

// ---- scan ----------------------------------------------------------------------
fdc_status check_scan_sizes(int B, int L, int D, int N, int G) {
  FDC_TRY(check_sizes(B, L, D));
  if (N < 1 || G < 1) return fail(FDC_EINVAL, "N and G must be positive (got %d, %d)", N, G);
  if (N > fdc::kScanMaxStates) return fail(FDC_EUNSUPPORTED, "N = %d states: at most %d", N, fdc::kScanMaxStates);
  if (D % G != 0) return fail(FDC_EINVAL, "D = %d is not a multiple of G = %d", D, G);
  if ((int64_t)B * D * N >= (1LL << 31) || (int64_t)B * L * G * N >= (1LL << 31))
    return fail(FDC_EUNSUPPORTED, "B D N or B L G N exceeds the launch limit (2^31)");
  return FDC_OK;
}

fdc_status check_scan(const fdc_scan_args *a, bool needs_y) {
  if (a == nullptr) return fail(FDC_EINVAL, "arguments are NULL");
  FDC_TRY(check_dtype(a->dtype));
  FDC_TRY(check_scan_sizes(a->B, a->L, a->D, a->N, a->G));
  FDC_TRY(check_tokens(a->x, "x", a->B, a->L, a->D, false));
  FDC_TRY(check_tokens(a->dt, "dt", a->B, a->L, a->D, false));
  FDC_TRY(check_tokens(a->gate, "gate", a->B, a->L, a->D, false, true));
  FDC_TRY(check_tokens(a->Bm, "Bm", a->B, a->L, (int64_t)a->G * a->N, false));
  FDC_TRY(check_tokens(a->Cm, "Cm", a->B, a->L, (int64_t)a->G * a->N, false));
  if (!a->A) return fail(FDC_EINVAL, "A is NULL");
  return needs_y ? check_tokens(a->y, "y", a->B, a->L, a->D, true) : FDC_OK;
}

// y may be x, dt or gate itself: the lanes that write a block of a channel's tokens have read it before.
fdc_status check_scan_apart(const fdc_scan_args *a) {
  const int64_t GN = (int64_t)a->G * a->N;
  FDC_TRY(check_apart(a->y, "y", a->D, a->x, "x", a->D, a->B, a->L, a->dtype, true));
  FDC_TRY(check_apart(a->y, "y", a->D, a->dt, "dt", a->D, a->B, a->L, a->dtype, true));
  FDC_TRY(check_apart(a->y, "y", a->D, a->gate, "gate", a->D, a->B, a->L, a->dtype, true));
  FDC_TRY(check_apart(a->y, "y", a->D, a->Bm, "Bm", GN, a->B, a->L, a->dtype, false));
  FDC_TRY(check_apart(a->y, "y", a->D, a->Cm, "Cm", GN, a->B, a->L, a->dtype, false));
  return check_apart(a->h_last, a->h0, (size_t)a->B * a->D * a->N * sizeof(float), "h_last and h0");
}

// ---- block norm ----------------------------------------------------------------
fdc_status check_row_stride(int64_t stride, int64_t R, int64_t width, const char *name, bool output) {
  if (stride < 0 || (output && R > 1 && stride < width))
    return fail(FDC_EINVAL, "%s: row stride %lld", name, (long long)stride);
  if (stride >= kMaxElements / R) return fail(FDC_EUNSUPPORTED, "%s: row stride %lld too large", name, (long long)stride);
  return FDC_OK;
}

fdc_status check_norm_sizes(int64_t R, int D) {
  if (R < 1 || D < 1) return fail(FDC_EINVAL, "R and D must be positive (got %lld, %d)", (long long)R, D);
  if (D > fdc::kNormMaxWidth) return fail(FDC_EUNSUPPORTED, "D = %d: at most %d", D, fdc::kNormMaxWidth);
  if (R > (1LL << 30)) return fail(FDC_EUNSUPPORTED, "R = %lld exceeds 2^30", (long long)R);
  return FDC_OK;
}

fdc_status check_norm(const fdc_block_norm_args *a) {
  if (a == nullptr) return fail(FDC_EINVAL, "arguments are NULL");
  FDC_TRY(check_dtype(a->dtype));
  FDC_TRY(check_norm_sizes(a->R, a->D));
  if (a->act < 0 || a->act > 2) return fail(FDC_EINVAL, "act must be 0, 1 or 2 (got %d)", a->act);
  if (!(a->eps > 0.f) || !std::isfinite(a->eps)) return fail(FDC_EINVAL, "eps must be positive (got %g)", (double)a->eps);
  if (!a->x) return fail(FDC_EINVAL, "x is NULL");
  if (!a->f && (a->gate || a->scale || a->w_post)) return fail(FDC_EINVAL, "gate, scale or w_post without f");
  FDC_TRY(check_row_stride(a->x_stride, a->R, a->D, "x", false));
  if (a->f) FDC_TRY(check_row_stride(a->f_stride, a->R, a->D, "f", false));
  if (a->gate) FDC_TRY(check_row_stride(a->gate_stride, a->R, a->D, "gate", false));
  return FDC_OK;
}

// ---- distillation ----------------------------------------------------------------
fdc_status check_distill_sizes(int dtype, int64_t R, int V) {
  FDC_TRY(check_dtype(dtype));
  if (R < 1 || V < 1) return fail(FDC_EINVAL, "R and V must be positive (got %lld, %d)", (long long)R, V);
  if (R >= (1LL << 26)) return fail(FDC_EUNSUPPORTED, "R = %lld: less than 2^26 are supported", (long long)R);
  if (V > (1 << 24)) return fail(FDC_EUNSUPPORTED, "V = %d exceeds 2^24", V);
  return FDC_OK;
}

fdc_status check_distill(const fdc_distill_args *a) {
  if (a == nullptr) return fail(FDC_EINVAL, "arguments are NULL");
  FDC_TRY(check_distill_sizes(a->dtype, a->R, a->V));
  if (a->K < 1) return fail(FDC_EINVAL, "K must be positive (got %d)", a->K);
  if (a->K > fdc::kDistillMaxTeacher) return fail(FDC_EUNSUPPORTED, "K = %d: at most %d", a->K, fdc::kDistillMaxTeacher);
  if (!(a->tau > 0.f) || !std::isfinite(a->tau)) return fail(FDC_EINVAL, "tau must be positive (got %g)", (double)a->tau);
  if (!(a->alpha >= 0.f && a->alpha <= 1.f)) return fail(FDC_EINVAL, "alpha must be in [0, 1] (got %g)", (double)a->alpha);
  if (!a->z || !a->idx || !a->teacher) return fail(FDC_EINVAL, "NULL tensor");
  return check_row_stride(a->z_stride, a->R, a->V, "z", false);
}

fdc_status check_ws(const void *ws, size_t got, size_t need, const char *what) {
  if (need > 0 && (!ws || got < need)) return fail(FDC_EWORKSPACE, "%s workspace: need %zu bytes, got %zu", what, need, got);
  if (need > 0 && (reinterpret_cast<uintptr_t>(ws) & 15)) return fail(FDC_EINVAL, "workspace must be 16-byte aligned");
  return FDC_OK;
}

}  // namespace

// ---------------------------------------------------------------------------
// causal convolution
// ---------------------------------------------------------------------------
fdc_status fdc_causal_conv_forward(const fdc_causal_conv_args *a, hipStream_t s) {
  FDC_TRY(check_conv(a));
  FDC_TRY(check_tokens(a->y, "y", a->B, a->L, a->D, true));
  // a run of tokens begins with rows in front of it, which another run's thread may have written by then
  FDC_TRY(check_apart(a->y, "y", a->D, a->x, "x", a->D, a->B, a->L, a->dtype, a->L == 1));
  FDC_TRY(check_apart(a->new_state, a->state, (size_t)a->B * (a->n - 1) * a->D * fdc::dtype_size(a->dtype),
                      "new_state and state"));
  return check_hip(fdc::launch_causal_conv_fwd(*a, s), "causal convolution");
}

fdc_status fdc_causal_conv_workspace_size(int dtype, int B, int L, int D, int n, size_t *bytes) {
  FDC_TRY(check_conv_sizes(dtype, B, L, D, n));
  if (!bytes) return fail(FDC_EINVAL, "bytes is NULL");
  *bytes = fdc::causal_conv_bwd_ws(dtype, B, L, D, n);
  return FDC_OK;
}

fdc_status fdc_causal_conv_backward(const fdc_causal_conv_args *a, fdc_tokens gy, fdc_tokens gx, float *gw,
                                    float *gbias, void *ws, size_t ws_bytes, hipStream_t s) {
  FDC_TRY(check_conv(a));
  FDC_TRY(check_tokens(gy, "gy", a->B, a->L, a->D, false));
  FDC_TRY(check_tokens(gx, "gx", a->B, a->L, a->D, true, true));
  if (!gx.p && !gw && !gbias) return FDC_OK;
  const size_t need = gw || gbias ? fdc::causal_conv_bwd_ws(a->dtype, a->B, a->L, a->D, a->n) : 0;
  FDC_TRY(check_ws(ws, ws_bytes, need, "causal convolution"));
  FDC_TRY(check_apart(gx, "gx", a->D, gy, "gy", a->D, a->B, a->L, a->dtype, a->L == 1));
  FDC_TRY(check_apart(gx, "gx", a->D, a->x, "x", a->D, a->B, a->L, a->dtype, a->L == 1));
  return check_hip(fdc::launch_causal_conv_bwd(*a, gy, gx, gw, gbias, static_cast<float *>(ws), s),
                   "causal convolution backward");
}

// ---------------------------------------------------------------------------
// selective scan
// ---------------------------------------------------------------------------
fdc_status fdc_scan_saved_size(int B, int L, int D, int N, size_t *bytes) {
  FDC_TRY(check_scan_sizes(B, L, D, N, 1));
  if (!bytes) return fail(FDC_EINVAL, "bytes is NULL");
  *bytes = fdc::scan_saved_floats(B, L, D, N) * sizeof(float);
  return FDC_OK;
}

fdc_status fdc_scan_workspace_size(int B, int L, int D, int N, int G, size_t *fwd_ws, size_t *bwd_ws) {
  FDC_TRY(check_scan_sizes(B, L, D, N, G));
  if (fwd_ws) *fwd_ws = fdc::scan_fwd_ws_floats(B, L, D, N, G) * sizeof(float);
  if (bwd_ws) *bwd_ws = fdc::scan_bwd_ws_floats(B, L, D, N, G) * sizeof(float);
  return FDC_OK;
}

fdc_status fdc_scan_forward(const fdc_scan_args *a, float *saved, void *ws, size_t ws_bytes, hipStream_t s) {
  FDC_TRY(check_scan(a, true));
  if (a->h_last && a->h_last == a->h0) return fail(FDC_EINVAL, "h_last must not be h0");
  if (reinterpret_cast<uintptr_t>(saved) & 15) return fail(FDC_EINVAL, "saved must be 16-byte aligned");
  FDC_TRY(check_ws(ws, ws_bytes, fdc::scan_fwd_ws_floats(a->B, a->L, a->D, a->N, a->G) * sizeof(float), "scan forward"));
  FDC_TRY(check_scan_apart(a));
  return check_hip(fdc::launch_scan_fwd(*a, saved, static_cast<float *>(ws), s), "scan");
}

fdc_status fdc_scan_backward(const fdc_scan_args *a, const float *saved, const fdc_scan_grads *g, void *ws,
                             size_t ws_bytes, hipStream_t s) {
  FDC_TRY(check_scan(a, false));
  if (!g) return fail(FDC_EINVAL, "gradients are NULL");
  if (!saved || (reinterpret_cast<uintptr_t>(saved) & 15))
    return fail(FDC_EINVAL, "saved must be given and 16-byte aligned");
  const int64_t GN = (int64_t)a->G * a->N;
  FDC_TRY(check_tokens(g->gy, "gy", a->B, a->L, a->D, false));
  FDC_TRY(check_tokens(g->gx, "gx", a->B, a->L, a->D, true));
  FDC_TRY(check_tokens(g->gdt, "gdt", a->B, a->L, a->D, true));
  FDC_TRY(check_tokens(g->ggate, "ggate", a->B, a->L, a->D, true, a->gate.p == nullptr));
  FDC_TRY(check_tokens(g->gBm, "gBm", a->B, a->L, GN, true));
  FDC_TRY(check_tokens(g->gCm, "gCm", a->B, a->L, GN, true));
  if (!g->gA) return fail(FDC_EINVAL, "gA is NULL");
  if ((a->skip != nullptr) != (g->gskip != nullptr) || (a->dt_bias != nullptr) != (g->gdt_bias != nullptr))
    return fail(FDC_EINVAL, "gskip and gdt_bias go with skip and dt_bias");
  FDC_TRY(check_ws(ws, ws_bytes, fdc::scan_bwd_ws_floats(a->B, a->L, a->D, a->N, a->G) * sizeof(float),
                   "scan backward"));
  return check_hip(fdc::launch_scan_bwd(*a, saved, *g, static_cast<float *>(ws), s), "scan backward");
}

fdc_status fdc_scan_step(const fdc_scan_args *a, hipStream_t s) {
  FDC_TRY(check_scan(a, true));
  if (a->L != 1 || a->lengths) return fail(FDC_EINVAL, "a step takes one token of every sequence (L = 1, no lengths)");
  if (!a->h0 || !a->h_last) return fail(FDC_EINVAL, "a step needs h0 and h_last");
  FDC_TRY(check_scan_apart(a));
  return check_hip(fdc::launch_scan_step(*a, s), "scan step");
}

// ---------------------------------------------------------------------------
// block norm
// ---------------------------------------------------------------------------
fdc_status fdc_block_norm_forward(const fdc_block_norm_args *a, void *out, int64_t out_stride, void *n,
                                  int64_t n_stride, float *stats, hipStream_t s) {
  FDC_TRY(check_norm(a));
  if ((a->w_pre != nullptr) != (n != nullptr)) return fail(FDC_EINVAL, "n goes with w_pre");
  if (!out && !n) return fail(FDC_EINVAL, "neither out nor n is wanted");
  if (out) FDC_TRY(check_row_stride(out_stride, a->R, a->D, "out", true));
  if (n) FDC_TRY(check_row_stride(n_stride, a->R, a->D, "n", true));
  return check_hip(fdc::launch_block_norm_fwd(*a, out, out_stride, n, n_stride, stats, s), "block norm");
}

fdc_status fdc_block_norm_workspace_size(int64_t R, int D, size_t *bytes) {
  FDC_TRY(check_norm_sizes(R, D));
  if (!bytes) return fail(FDC_EINVAL, "bytes is NULL");
  *bytes = fdc::block_norm_bwd_ws_floats(R, D) * sizeof(float);
  return FDC_OK;
}

fdc_status fdc_block_norm_backward(const fdc_block_norm_args *a, const float *stats, const fdc_block_norm_grads *g,
                                   void *ws, size_t ws_bytes, hipStream_t s) {
  FDC_TRY(check_norm(a));
  if (!g || !stats) return fail(FDC_EINVAL, "stats or gradients are NULL");
  if (!g->gout && !g->gn) return fail(FDC_EINVAL, "neither gout nor gn is given");
  if (g->gn && !a->w_pre) return fail(FDC_EINVAL, "gn without w_pre");
  if ((g->gf && !a->f) || (g->ggate && !a->gate) || (g->gscale && !a->scale) || (g->gw_post && !a->w_post) ||
      (g->gw_pre && !a->w_pre))
    return fail(FDC_EINVAL, "a gradient is asked for an input that is not given");
  if (g->gout) FDC_TRY(check_row_stride(g->gout_stride, a->R, a->D, "gout", false));
  if (g->gn) FDC_TRY(check_row_stride(g->gn_stride, a->R, a->D, "gn", false));
  if (g->gx) FDC_TRY(check_row_stride(g->gx_stride, a->R, a->D, "gx", true));
  if (g->gf) FDC_TRY(check_row_stride(g->gf_stride, a->R, a->D, "gf", true));
  if (g->ggate) FDC_TRY(check_row_stride(g->ggate_stride, a->R, a->D, "ggate", true));
  const size_t need = g->gscale || g->gw_post || g->gw_pre ? fdc::block_norm_bwd_ws_floats(a->R, a->D) * sizeof(float) : 0;
  FDC_TRY(check_ws(ws, ws_bytes, need, "block norm"));
  return check_hip(fdc::launch_block_norm_bwd(*a, stats, *g, static_cast<float *>(ws), s), "block norm backward");
}

// ---------------------------------------------------------------------------
// distillation
// ---------------------------------------------------------------------------
fdc_status fdc_distill_workspace_size(int dtype, int64_t R, int V, size_t *bytes) {
  FDC_TRY(check_distill_sizes(dtype, R, V));
  if (!bytes) return fail(FDC_EINVAL, "bytes is NULL");
  *bytes = fdc::distill_ws_floats(dtype, R, V) * sizeof(float);
  return FDC_OK;
}

fdc_status fdc_distill_forward(const fdc_distill_args *a, float *loss, float *stats, void *ws, size_t ws_bytes,
                               hipStream_t s) {
  FDC_TRY(check_distill(a));
  if (!loss || !stats) return fail(FDC_EINVAL, "loss or stats is NULL");
  FDC_TRY(check_ws(ws, ws_bytes, fdc::distill_ws_floats(a->dtype, a->R, a->V) * sizeof(float), "distillation"));
  return check_hip(fdc::launch_distill(*a, loss, stats, nullptr, nullptr, 0, static_cast<float *>(ws), s),
                   "distillation");
}

fdc_status fdc_distill_backward(const fdc_distill_args *a, const float *stats, const float *gloss, void *gz,
                                int64_t gz_stride, hipStream_t s) {
  FDC_TRY(check_distill(a));
  if (!stats || !gloss || !gz) return fail(FDC_EINVAL, "stats, gloss or gz is NULL");
  FDC_TRY(check_row_stride(gz_stride, a->R, a->V, "gz", true));
  FDC_TRY(check_apart({gz, gz_stride, 0}, "gz", a->V, {const_cast<void *>(a->z), a->z_stride, 0}, "z", a->V, a->R, 1,
                      a->dtype, true));
  return check_hip(fdc::launch_distill_bwd(*a, stats, gloss, gz, gz_stride, s), "distillation backward");
}

fdc_status fdc_distill_forward_backward(const fdc_distill_args *a, const float *gloss, float *loss, float *stats,
                                        void *gz, int64_t gz_stride, void *ws, size_t ws_bytes, hipStream_t s) {
  FDC_TRY(check_distill(a));
  if (!loss || !stats || !gloss || !gz) return fail(FDC_EINVAL, "loss, stats, gloss or gz is NULL");
  FDC_TRY(check_row_stride(gz_stride, a->R, a->V, "gz", true));
  FDC_TRY(check_apart({gz, gz_stride, 0}, "gz", a->V, {const_cast<void *>(a->z), a->z_stride, 0}, "z", a->V, a->R, 1,
                      a->dtype, true));
  FDC_TRY(check_ws(ws, ws_bytes, fdc::distill_ws_floats(a->dtype, a->R, a->V) * sizeof(float), "distillation"));
  return check_hip(fdc::launch_distill(*a, loss, stats, gloss, gz, gz_stride, static_cast<float *>(ws), s),
                   "distillation");
}

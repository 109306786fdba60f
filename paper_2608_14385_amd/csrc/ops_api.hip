// Host side of the operators beside the decode layer: validation, workspaces
// and launches.  Nothing here allocates, frees or waits.
#include <cmath>

#include "ops.h"

using namespace deamoe;

namespace {

int check(hipError_t e) { return e == hipSuccess ? DEAMOE_OK : DEAMOE_ERR_HIP; }

bool aligned(const void *p, size_t to) { return !((uintptr_t)p & (to - 1)); }
// required: given and aligned to its element
bool good(const void *p, size_t to) { return p && aligned(p, to); }
bool good_or_null(const void *p, size_t to) { return !p || aligned(p, to); }

size_t align16(size_t v) { return (v + 15) / 16 * 16; }

int check_rows(int32_t T, int32_t h, int32_t act_dtype) {
  if (T < 0 || h <= 0) return DEAMOE_ERR_INVALID;
  if (act_dtype != DEAMOE_F32 && act_dtype != DEAMOE_BF16) return DEAMOE_ERR_INVALID;
  if (T > DEAMOE_MAX_ROWS || h > DEAMOE_MAX_WIDTH) return DEAMOE_ERR_UNSUPPORTED;
  return DEAMOE_OK;
}
size_t bytes_of(int32_t act_dtype) { return act_dtype == DEAMOE_F32 ? 4 : 2; }

int check_pairs(int32_t T, int32_t k) {
  if (k <= 0) return DEAMOE_ERR_INVALID;
  if (k > DEAMOE_MAX_TOPK || (int64_t)T * k > DEAMOE_MAX_PAIRS) return DEAMOE_ERR_UNSUPPORTED;
  return DEAMOE_OK;
}

int check_groups(int32_t T, int32_t k, int32_t n) {
  if (T < 0 || n <= 0) return DEAMOE_ERR_INVALID;
  if (T > DEAMOE_MAX_ROWS || n > DEAMOE_MAX_EXPERTS) return DEAMOE_ERR_UNSUPPORTED;
  return check_pairs(T, k);
}

struct SortLayout {
  size_t hist, total, bytes;
};
SortLayout sort_layout(int32_t T, int32_t k, int32_t n) {
  SortLayout L{0, 0, 0};
  const int64_t P = (int64_t)T * k;
  if (P <= kSortSmallPairs) return L;
  L.total = align16((size_t)n * ((P + sort_chunk(P) - 1) / sort_chunk(P)) * 4);
  L.bytes = L.total + align16((size_t)n * 4);
  return L;
}

}  // namespace

extern "C" {

int deamoe_dispatch_workspace_bytes(int32_t T, int32_t k, int32_t n, size_t *bytes) {
  const int rc = check_groups(T, k, n);
  if (rc) return rc;
  if (!bytes) return DEAMOE_ERR_INVALID;
  *bytes = sort_layout(T, k, n).bytes;
  return DEAMOE_OK;
}

int deamoe_dispatch(int32_t T, int32_t k, int32_t n, int32_t h, int32_t act_dtype,
                    const int32_t *ids, const void *x, int32_t *offset, int32_t *pair,
                    int32_t *row, void *xs, void *ws, size_t ws_bytes, void *stream) {
  int rc = check_rows(T, h, act_dtype);
  if (rc || (rc = check_groups(T, k, n))) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (!good(offset, 4)) return DEAMOE_ERR_INVALID;
  if (T == 0) return check(launch_zero(offset, (size_t)(n + 1) * 4, s));
  if (!good(ids, 4) || !good(pair, 4) || !good(row, 4)) return DEAMOE_ERR_INVALID;
  if (xs && (!good(x, bytes_of(act_dtype)) || !good(xs, bytes_of(act_dtype))))
    return DEAMOE_ERR_INVALID;
  const SortLayout L = sort_layout(T, k, n);
  if (L.bytes && (!ws || ws_bytes < L.bytes || !aligned(ws, 16))) return DEAMOE_ERR_WORKSPACE;
  DispatchArgs a;
  a.T = T;
  a.k = k;
  a.n = n;
  a.h = h;
  a.act_f32 = act_dtype == DEAMOE_F32;
  a.ids = ids;
  a.x = x;
  a.offset = offset;
  a.pair = pair;
  a.row = row;
  a.xs = xs;
  a.hist = reinterpret_cast<int32_t *>(static_cast<char *>(ws) + L.hist);
  a.total = reinterpret_cast<int32_t *>(static_cast<char *>(ws) + L.total);
  return check(launch_dispatch(a, s));
}

static int collect(int32_t T, int32_t k, int32_t h, int32_t act_dtype, const int32_t *row,
                   const float *w, bool weighted, const void *ys, void *y, void *stream) {
  int rc = check_rows(T, h, act_dtype);
  if (rc || (rc = check_pairs(T, k))) return rc;
  if (T == 0) return DEAMOE_OK;
  const size_t b = bytes_of(act_dtype);
  if (!good(row, 4) || !good(ys, b) || !good(y, b) || (weighted && !good(w, 4)))
    return DEAMOE_ERR_INVALID;
  CollectArgs a{T, k, h, act_dtype == DEAMOE_F32, row, weighted ? w : nullptr, ys, y};
  return check(launch_collect(a, static_cast<hipStream_t>(stream)));
}

int deamoe_dispatch_backward(int32_t T, int32_t k, int32_t h, int32_t act_dtype,
                             const int32_t *row, const void *dxs, void *dx, void *stream) {
  return collect(T, k, h, act_dtype, row, nullptr, false, dxs, dx, stream);
}

int deamoe_combine(int32_t T, int32_t k, int32_t h, int32_t act_dtype, const int32_t *row,
                   const float *w, const void *ys, void *y, void *stream) {
  return collect(T, k, h, act_dtype, row, w, true, ys, y, stream);
}

int deamoe_combine_backward(int32_t T, int32_t k, int32_t h, int32_t act_dtype,
                            const int32_t *row, const float *w, const void *ys, const void *dy,
                            void *dys, float *dw, void *stream) {
  int rc = check_rows(T, h, act_dtype);
  if (rc || (rc = check_pairs(T, k))) return rc;
  if (T == 0) return DEAMOE_OK;
  const size_t b = bytes_of(act_dtype);
  if (!good(row, 4) || !good(dy, b) || !good_or_null(dys, b) || !good_or_null(dw, 4))
    return DEAMOE_ERR_INVALID;
  if ((dys && !good(w, 4)) || (dw && !good(ys, b))) return DEAMOE_ERR_INVALID;
  if (!dys && !dw) return DEAMOE_OK;
  CollectBackwardArgs a{T, k, h, act_dtype == DEAMOE_F32, row, w, ys, dy, dys, dw};
  return check(launch_collect_backward(a, static_cast<hipStream_t>(stream)));
}

static int w4(const deamoe_w4_config *c, int32_t M, const void *x, const int32_t *offset,
              int mats, const void *const *codes, const void *const *scale, void *y,
              void *stream) {
  if (!c || M < 0 || c->R <= 0 || c->K <= 0 || c->n <= 0) return DEAMOE_ERR_INVALID;
  if (c->group != 32 && c->group != 64 && c->group != 128) return DEAMOE_ERR_INVALID;
  if (c->K % c->group) return DEAMOE_ERR_INVALID;
  if (c->scale_dtype != DEAMOE_F32 && c->scale_dtype != DEAMOE_BF16) return DEAMOE_ERR_INVALID;
  if (c->n > 1 && M > 0 && !offset) return DEAMOE_ERR_INVALID;
  if (M > DEAMOE_MAX_PAIRS || c->n > DEAMOE_MAX_EXPERTS || c->K > DEAMOE_MAX_WIDTH ||
      c->R > DEAMOE_MAX_WIDTH)
    return DEAMOE_ERR_UNSUPPORTED;
  if (M == 0) return DEAMOE_OK;
  if (!good(x, 16) || !good(y, 2) || !good_or_null(offset, 4)) return DEAMOE_ERR_INVALID;
  W4Args a;
  a.M = M;
  a.R = c->R;
  a.K = c->K;
  a.n = c->n;
  a.group = c->group;
  a.scale_bf16 = c->scale_dtype == DEAMOE_BF16;
  a.x = x;
  a.offset = offset;
  a.y = y;
  for (int i = 0; i < 2; ++i) {
    const int from = i < mats ? i : 0;
    if (!good(codes[from], 16) || !good(scale[from], a.scale_bf16 ? 2 : 4))
      return DEAMOE_ERR_INVALID;
    a.w[i] = codes[from];
    a.scale[i] = scale[from];
  }
  return check(launch_w4(a, mats, static_cast<hipStream_t>(stream)));
}

int deamoe_w4_linear(const deamoe_w4_config *cfg, int32_t M, const void *x, const int32_t *offset,
                     const void *codes, const void *scale, void *y, void *stream) {
  return w4(cfg, M, x, offset, 1, &codes, &scale, y, stream);
}

int deamoe_w4_swiglu(const deamoe_w4_config *cfg, int32_t M, const void *x, const int32_t *offset,
                     const void *gate_codes, const void *gate_scale, const void *up_codes,
                     const void *up_scale, void *y, void *stream) {
  const void *codes[2] = {gate_codes, up_codes}, *scale[2] = {gate_scale, up_scale};
  return w4(cfg, M, x, offset, 2, codes, scale, y, stream);
}

static int check_norm(int32_t T, int32_t h, int32_t act_dtype, float eps) {
  const int rc = check_rows(T, h, act_dtype);
  if (rc) return rc;
  return eps > 0.f && std::isfinite(eps) ? DEAMOE_OK : DEAMOE_ERR_INVALID;
}

int deamoe_prenorm(int32_t T, int32_t h, int32_t act_dtype, float eps, const void *x,
                   const void *w, void *u, void *stream) {
  const int rc = check_norm(T, h, act_dtype, eps);
  if (rc || T == 0) return rc;
  const size_t b = bytes_of(act_dtype);
  if (!good(x, b) || !good(w, b) || !good(u, b)) return DEAMOE_ERR_INVALID;
  PrenormArgs a{T, h, act_dtype == DEAMOE_F32, eps, x, w, u};
  return check(launch_prenorm(a, static_cast<hipStream_t>(stream)));
}

static bool gate_given(int32_t mode, const void *gate, size_t b) {
  return mode == DEAMOE_GATE_NONE ? !gate : good(gate, b);
}

int deamoe_postnorm(int32_t T, int32_t h, int32_t act_dtype, float eps, float res_scale,
                    int32_t gate_mode, const void *x, const void *y, const void *w,
                    const void *gate, const void *w_next, void *z, void *u, void *stream) {
  const int rc = check_norm(T, h, act_dtype, eps);
  if (rc) return rc;
  if (!std::isfinite(res_scale) || gate_mode < DEAMOE_GATE_NONE || gate_mode > DEAMOE_GATE_FULL)
    return DEAMOE_ERR_INVALID;
  if (T == 0) return DEAMOE_OK;
  const size_t b = bytes_of(act_dtype);
  if (!good(x, b) || !good(y, b) || !good(w, b) || !good(z, b) || !gate_given(gate_mode, gate, b))
    return DEAMOE_ERR_INVALID;
  if (!u != !w_next || !good_or_null(u, b) || !good_or_null(w_next, b)) return DEAMOE_ERR_INVALID;
  PostnormArgs a{T,   h, act_dtype == DEAMOE_F32, gate_mode, eps, res_scale, x, y, w, gate,
                 w_next, z, u};
  return check(launch_postnorm(a, static_cast<hipStream_t>(stream)));
}

static size_t norm_bytes(int32_t T, int32_t h) {   // enough for either type
  const int bf16 = norm_backward_blocks(T, h, 0), f32 = norm_backward_blocks(T, h, 1);
  return align16((size_t)(bf16 > f32 ? bf16 : f32) * 3 * h * 4);
}

int deamoe_norm_workspace_bytes(int32_t T, int32_t h, size_t *bytes) {
  const int rc = check_rows(T, h, DEAMOE_F32);
  if (rc) return rc;
  if (!bytes) return DEAMOE_ERR_INVALID;
  *bytes = norm_bytes(T, h);
  return DEAMOE_OK;
}

static int norm_backward(NormBackwardArgs &a, void *ws, size_t ws_bytes, hipStream_t s) {
  if (!ws || ws_bytes < norm_bytes(a.T, a.h) || !aligned(ws, 16)) return DEAMOE_ERR_WORKSPACE;
  a.part = static_cast<float *>(ws);
  return check(launch_norm_backward(a, s));
}

int deamoe_prenorm_backward(int32_t T, int32_t h, int32_t act_dtype, float eps, const void *x,
                            const void *w, const void *du, const void *dres, void *dx, float *dw,
                            void *ws, size_t ws_bytes, void *stream) {
  const int rc = check_norm(T, h, act_dtype, eps);
  if (rc) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (!good(dw, 4)) return DEAMOE_ERR_INVALID;
  if (T == 0) return check(launch_zero(dw, (size_t)h * 4, s));
  const size_t b = bytes_of(act_dtype);
  if (!good(x, b) || !good(w, b) || !good(du, b) || !good_or_null(dres, b) || !good(dx, b))
    return DEAMOE_ERR_INVALID;
  NormBackwardArgs a{};
  a.T = T;
  a.h = h;
  a.act_f32 = act_dtype == DEAMOE_F32;
  a.gate_mode = DEAMOE_GATE_NONE;
  a.eps = eps;
  a.res_scale = 1.f;
  a.z = x;
  a.w_next = w;
  a.du = du;
  a.dz = dres;
  a.dx = dx;
  a.dw_next = dw;
  return norm_backward(a, ws, ws_bytes, s);
}

int deamoe_postnorm_backward(int32_t T, int32_t h, int32_t act_dtype, float eps, float res_scale,
                             int32_t gate_mode, const void *y, const void *w, const void *gate,
                             const void *z, const void *w_next, const void *dz, const void *du,
                             void *dx, void *dy, float *dw, void *dgate, float *dw_next, void *ws,
                             size_t ws_bytes, void *stream) {
  const int rc = check_norm(T, h, act_dtype, eps);
  if (rc) return rc;
  if (!std::isfinite(res_scale) || gate_mode < DEAMOE_GATE_NONE || gate_mode > DEAMOE_GATE_FULL)
    return DEAMOE_ERR_INVALID;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const size_t b = bytes_of(act_dtype);
  const bool shared = gate_mode == DEAMOE_GATE_SHARED;
  if (!good(dw, 4) || !good_or_null(dw_next, 4)) return DEAMOE_ERR_INVALID;
  if (shared && !good(dgate, 4)) return DEAMOE_ERR_INVALID;
  if (T == 0) {
    int e = check(launch_zero(dw, (size_t)h * 4, s));
    if (!e && shared) e = check(launch_zero(dgate, (size_t)h * 4, s));
    if (!e && dw_next) e = check(launch_zero(dw_next, (size_t)h * 4, s));
    return e;
  }
  if (!good(y, b) || !good(w, b) || !good(dz, b) || !good(dx, b) || !good(dy, b) ||
      !gate_given(gate_mode, gate, b) || !gate_given(gate_mode, dgate, shared ? 4 : b))
    return DEAMOE_ERR_INVALID;
  const bool next = du != nullptr;
  if (next ? !good(z, b) || !good(w_next, b) || !good(du, b) || !dw_next : z || w_next || dw_next)
    return DEAMOE_ERR_INVALID;
  NormBackwardArgs a{};
  a.T = T;
  a.h = h;
  a.act_f32 = act_dtype == DEAMOE_F32;
  a.gate_mode = gate_mode;
  a.eps = eps;
  a.res_scale = res_scale;
  a.y = y;
  a.w = w;
  a.gate = gate;
  a.z = z;
  a.w_next = w_next;
  a.dz = dz;
  a.du = du;
  a.dx = dx;
  a.dy = dy;
  a.dgate = dgate;
  a.dw = dw;
  a.dw_next = dw_next;
  return norm_backward(a, ws, ws_bytes, s);
}

}  // extern "C"

/* deamoe.h -- C ABI of the MI355X (gfx950) DeaMoE decode-layer library.
 *
 * What is computed (the paper's notation; no code of the paper is used):
 *   Router (Sec. 2.1, Eq. 2): logits l = W_r x (+ optional bias), the top-k
 *     experts S(x) by (logit desc, expert id asc), optionally limited to the
 *     top_k_dept departments by group score (Sec. 3.3, group-limited top-k);
 *     routing weights p after softmax or sigmoid normalisation and scaling
 *     (Sec. 2.1, the sentence after Eq. 3).
 *   Departments (Sec. 3.1): n experts in m departments of E_d = n / m
 *     consecutive experts; expert e belongs to department e / E_d.
 *   Expert output, SLICE form: department-shared SwiGLU slice (intermediate
 *     d_shared) plus a private SwiGLU slice (intermediate d_private), summed.
 *   Expert output, FACTORED form (Sec. 3.1, Eq. 4):
 *     d_i(g_i(x) * u_i(x)), g_i = SiLU(A_g sigma(W_g x)), u_i = A_u sigma(W_u x),
 *     d_i(v) = W_d^T sigma(A_d^T v), sigma = SiLU, identity, GeLU or RMSNorm.
 *   Layer output (Eq. 3): y = sum_{i in S(x)} p_i expert_i(x), plus an optional
 *     always-on shared SwiGLU expert with weight 1.
 *   Two-stage evaluation (Sec. 3.2): each touched department's shared
 *     matrices are streamed once per step for all of its tokens (X^j), each
 *     touched expert's private matrices once for its tokens, then the weighted
 *     combine.  The result equals the per-expert definition up to rounding.
 *
 * Conventions for every entry point:
 *   - Tensor pointers are DEVICE pointers owned by the caller, except where a
 *     parameter says "host".  `stream` is a hipStream_t (NULL = null stream).
 *   - All device work is enqueued on `stream`; no call allocates device or
 *     host memory, frees, or synchronises; every call is hipGraph-capturable.
 *   - Arguments are validated on the host before anything is enqueued; an
 *     invalid call returns a negative DEAMOE_ERR_* code and enqueues nothing.
 *     A launch failure returns DEAMOE_ERR_HIP.
 *   - T == 0 returns DEAMOE_OK and enqueues nothing once the configuration
 *     is valid (tensor pointers may then be NULL).
 *   - Identical inputs give bit-identical outputs (no atomics in any sum).
 *   - The library holds no state: calls on different streams are independent
 *     as long as each uses its own workspace and outputs.
 *
 * Layouts: every matrix is row-major [out, in] and stacked over departments
 * or experts.  Activations x and y are row-major [T, hidden].
 */
#ifndef DEAMOE_H
#define DEAMOE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* status codes */
#define DEAMOE_OK 0
#define DEAMOE_ERR_INVALID (-1)      /* bad argument or inconsistent config        */
#define DEAMOE_ERR_UNSUPPORTED (-2)  /* valid but outside this build's limits      */
#define DEAMOE_ERR_WORKSPACE (-3)    /* workspace missing or too small             */
#define DEAMOE_ERR_HIP (-4)          /* a HIP launch failed                        */

/* element types */
#define DEAMOE_F32 0
#define DEAMOE_BF16 1
#define DEAMOE_FP8_E4M3_B128 2  /* OCP e4m3fn codes + one fp32 scale per 128x128 block */

/* expert form */
#define DEAMOE_FORM_SLICE 0
#define DEAMOE_FORM_FACTORED 1

/* routing score */
#define DEAMOE_SCORE_SOFTMAX 0
#define DEAMOE_SCORE_SIGMOID 1

/* interface nonlinearity sigma of the FACTORED form (Sec. 3.1; the
 * alternatives are the ones compared in Sec. 3.4) */
#define DEAMOE_SIGMA_SILU 0
#define DEAMOE_SIGMA_NONE 1      /* identity                                            */
#define DEAMOE_SIGMA_GELU 2      /* v * Phi(v), the exact (erf) form                     */
#define DEAMOE_SIGMA_RMSNORM 3   /* v / sqrt(mean(v^2) + 1e-6) over the d-vector, unit gain */

/* Limits of this build (DEAMOE_ERR_UNSUPPORTED beyond them). */
#define DEAMOE_MAX_TOKENS 128
#define DEAMOE_MAX_EXPERTS 2048
#define DEAMOE_MAX_TOPK 32
/* every width (hidden, d_shared, d_private, d_shared_expert) is at most this
 * many columns, so that the token rows one stage reads lie within 4 GiB of
 * their buffer (32-bit row offsets in the expert stages) */
#define DEAMOE_MAX_WIDTH 65536
/* fp8 weights: every contraction length (hidden, d_shared, d_private,
 * d_shared_expert) is at most this many columns (64 scale blocks) */
#define DEAMOE_MAX_FP8_K 8192

typedef struct {
  int32_t hidden;           /* h                                                        */
  int32_t n_experts;        /* n                                                        */
  int32_t n_depts;          /* m, divides n                                             */
  int32_t top_k;            /* k experts per token (Eq. 2)                              */
  int32_t top_k_dept;       /* at most this many departments per token; 0 = no limit    */
  int32_t d_shared;         /* SLICE: department slice intermediate; FACTORED: d        */
  int32_t d_private;        /* SLICE: private slice intermediate (0 = none);
                               FACTORED: ignored (private matrices are d x d)           */
  int32_t d_shared_expert;  /* always-on shared expert intermediate; 0 = none           */
  int32_t form;             /* DEAMOE_FORM_*                                            */
  int32_t score;            /* DEAMOE_SCORE_*                                           */
  int32_t renorm;           /* 1: weights renormalised over the selected k experts      */
  int32_t sigma;            /* DEAMOE_SIGMA_* (FACTORED only)                           */
  float route_scale;        /* routing weights are multiplied by this                   */
  int32_t w_dtype;          /* expert weight type: DEAMOE_F32 | BF16 | FP8_E4M3_B128    */
  int32_t act_dtype;        /* x, y and router weight type: DEAMOE_F32 | DEAMOE_BF16    */
  int32_t max_tokens;       /* largest T the workspace is sized for (<= 128)            */
  int32_t dept_cover;       /* 0: top_k_dept is an upper bound (group-limited top-k).
                               1: strict coverage (Sec. 3.4): while a token's k experts
                               span fewer than top_k_dept departments, its lowest-ranked
                               expert whose department holds another selected expert is
                               replaced by the best expert of a kept department not yet
                               covered.  Needs top_k_dept > 0 and top_k >= top_k_dept. */
} deamoe_config;

/* Expert weights.  Shapes ([out, in], stacked):
 *   router      [n, h]           act_dtype
 *   dept_gate   [m, d_s, h]      W_g^j
 *   dept_up     [m, d_s, h]      W_u^j
 *   dept_down   [m, h, d_s]      (W_d^j)^T
 *   SLICE:    priv_gate [n, d_p, h], priv_up [n, d_p, h], priv_down [n, h, d_p]
 *             (NULL when d_private == 0)
 *   FACTORED: priv_gate = A_g [n, d, d], priv_up = A_u [n, d, d],
 *             priv_down = (A_d)^T [n, d, d]
 *   se_gate [d_se, h], se_up [d_se, h], se_down [h, d_se] (NULL when d_se == 0)
 *   scale[0..8]: fp8 only, one fp32 per 128 x 128 block of each matrix, in the
 *     order dept_gate, dept_up, dept_down, priv_gate, priv_up, priv_down,
 *     se_gate, se_up, se_down; each [stack, ceil(out/128), in/128].
 * All pointers 16-byte aligned. */
typedef struct {
  const void *router;
  const void *dept_gate, *dept_up, *dept_down;
  const void *priv_gate, *priv_up, *priv_down;
  const void *se_gate, *se_up, *se_down;
  const float *scale[9];
} deamoe_weights;

/* Routing results (device arrays, caller-allocated).
 *   topk_ids   [T, k]  selected experts in rank order
 *   topk_w     [T, k]  routing weights p (fp32)
 *   tok_depts  [T, k]  distinct departments of the token, ascending, -1 padded
 *   tok_dept_w [T, k]  P_{t,j}: summed weight of the token's experts in each
 *   tok_ndept  [T]     number of distinct departments
 *   dept_count [m], dept_offset [m+1], dept_tokens [T*k]: the token list X^j of
 *     every department (ascending token index), CSR
 *   exp_count [n], exp_offset [n+1], exp_tokens [T*k]: the same per expert
 *   logits     [T, n]  fp32 logits after the bias (may be NULL) */
typedef struct {
  int32_t *topk_ids;
  float *topk_w;
  int32_t *tok_depts;
  float *tok_dept_w;
  int32_t *tok_ndept;
  int32_t *dept_count, *dept_offset, *dept_tokens;
  int32_t *exp_count, *exp_offset, *exp_tokens;
  float *logits;
} deamoe_routing;

/* Human-readable text of a status code (static storage). */
const char *deamoe_status_string(int status);

/* Host.  Bytes of device workspace that deamoe_route / deamoe_layer_forward /
 * deamoe_baseline_forward need for up to cfg->max_tokens tokens. */
int deamoe_workspace_bytes(const deamoe_config *cfg, size_t *bytes);

/* Router only (Eq. 2 and the department bookkeeping of Sec. 3.2).
 * x [T, h] act_dtype; router_w [n, h] act_dtype.  logits_in: optional fp32
 * [T, n] logits used instead of W_r x.  router_bias: optional fp32 [n] added
 * to the logits (one fp32 add after the complete dot product) before both
 * selection and weighting.  `out` receives every array of deamoe_routing
 * (out->logits may be NULL). */
int deamoe_route(const deamoe_config *cfg, int32_t T, const void *x, const void *router_w,
                 const float *logits_in, const float *router_bias, deamoe_routing *out,
                 void *ws, size_t ws_bytes, void *stream);

/* The DeaMoE layer (Eq. 3 over SLICE or FACTORED experts, two-stage order).
 * y [T, h] act_dtype.  routing_out: optional, receives the routing (NULL: the
 * routing lives in the workspace). */
int deamoe_layer_forward(const deamoe_config *cfg, int32_t T, const void *x,
                         const deamoe_weights *w, const float *logits_in,
                         const float *router_bias, deamoe_routing *routing_out, void *y,
                         void *ws, size_t ws_bytes, void *stream);

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the same
 * call as deamoe_layer_forward, same kernels and results, with the workspace
 * taken from a library-owned device array of DEAMOE_SCRATCH_BYTES per GPU
 * (the current device's), held until the process ends.  Nothing is allocated
 * or freed.  A configuration whose workspace (deamoe_workspace_bytes, sized
 * for cfg->max_tokens) exceeds DEAMOE_SCRATCH_BYTES returns
 * DEAMOE_ERR_WORKSPACE before any HIP call.  The first call on a device
 * resolves that device's array address (DEAMOE_ERR_HIP if that fails).
 * Every call on one GPU shares its array: calls that overlap in time on one
 * GPU (other streams, other host threads) race and must be serialised by the
 * caller.  No part of the array needs clearing between calls; each call
 * writes everything it reads.  `stream` must belong to the current device. */
#define DEAMOE_SCRATCH_BYTES (64u << 20)
int deamoe_layer_forward_noalloc(const deamoe_config *cfg, int32_t T, const void *x,
                                 const deamoe_weights *w, const float *logits_in,
                                 const float *router_bias, deamoe_routing *routing_out, void *y,
                                 void *stream);

/* The same with caller-created hipEvent_t handles recorded on `stream` at the
 * stage boundaries, for timing: events[0] before the router, then one after
 * each launched kernel in order (SLICE: router GEMV, route, gate/up, down,
 * combine; FACTORED: router GEMV, route, department gate/up, private gate/up,
 * private down, Z collect, department down, combine).  Small batches may
 * run the last down stage and the combine as one kernel
 * (deamoe_trace_points gives the count).  n_events may be
 * smaller than that count; NULL / 0 records nothing.  With injected logits
 * the router GEMV is not launched and has no boundary. */
int deamoe_layer_forward_traced(const deamoe_config *cfg, int32_t T, const void *x,
                                const deamoe_weights *w, const float *logits_in,
                                const float *router_bias, deamoe_routing *routing_out, void *y,
                                void *ws, size_t ws_bytes, void *stream, void *const *events,
                                int32_t n_events);

/* Host: the number of events deamoe_layer_forward_traced records for a batch
 * of T tokens with computed logits (1 + one per stage listed above).  Returns
 * DEAMOE_ERR_INVALID for a NULL pointer, T < 1 or T > max_tokens. */
int deamoe_trace_points(const deamoe_config *cfg, int32_t T, int32_t *n_events);

/* Vanilla MoE of Eq. 1-3 at the same shape, the comparator for speedups:
 * cfg must describe one expert per department (n_depts == n_experts), no
 * private part (d_private == 0), SLICE form; d_shared is the expert
 * intermediate size f and dept_* hold the n experts' matrices. */
int deamoe_baseline_forward(const deamoe_config *cfg, int32_t T, const void *x,
                            const deamoe_weights *w, const float *logits_in,
                            const float *router_bias, deamoe_routing *routing_out, void *y,
                            void *ws, size_t ws_bytes, void *stream);

/* Host.  Algorithmic HBM bytes of one step: the per-step weight loading that
 * Sec. 3.3 compares between DeaMoE and vanilla MoE (Fig. 2), with the router
 * counted as that comparison's budget accounting counts it.  Given the
 * realised routing counts (host arrays dept_count [m], exp_count [n]):
 * every touched department's and expert's matrices once (fp8: plus block
 * scales), the router, the shared expert -> *weight_bytes; *total_bytes adds
 * x read and y written (T x h activations each).  Either output may be NULL.
 * DEAMOE_ERR_INVALID for a NULL count array or T < 0. */
int deamoe_loaded_bytes(const deamoe_config *cfg, int32_t T, const int32_t *dept_count,
                        const int32_t *exp_count, int64_t *weight_bytes, int64_t *total_bytes);

/* ---------------------------------------------------------------------------
 * Operators beside the decode layer.  The conventions above hold, for batches
 * of any size: tensors are row-major and contiguous, aligned to their element
 * (stated where more is needed); outputs do not overlap inputs except where
 * this header says so; T is at most DEAMOE_MAX_ROWS, widths at most
 * DEAMOE_MAX_WIDTH.  Sums over no tokens are written as zeros. */
#define DEAMOE_MAX_ROWS (1 << 23)
#define DEAMOE_MAX_PAIRS (1 << 26)   /* T * k of the sorted tokens */

/* --- Tokens sorted by expert and back (X^j and X^{j,i} of Sec. 3.2 as rows).
 * A pair p = t * k + s is slot s of token t.  ids [T, k]: its group (expert or
 * department), in any order, repeats allowed; an id outside [0, n) drops the
 * pair (deamoe_route's topk_ids and its -1 padded tok_depts both fit).
 *   offset [n + 1]   first row of every group; offset[n] = rows used
 *   pair   [T * k]   pair of every row, by (group, pair) ascending; -1 from
 *                    offset[n] on
 *   row    [T, k]    row of every pair, -1 if dropped
 * xs [T * k, h]: row r is x of token pair[r] / k; rows from offset[n] on are
 * left as they were.  xs may be NULL (lists only; then x may be NULL too).
 * n <= DEAMOE_MAX_EXPERTS, k <= DEAMOE_MAX_TOPK.  ws 16-byte aligned. */
int deamoe_dispatch_workspace_bytes(int32_t T, int32_t k, int32_t n, size_t *bytes);
int deamoe_dispatch(int32_t T, int32_t k, int32_t n, int32_t h, int32_t act_dtype,
                    const int32_t *ids, const void *x, int32_t *offset, int32_t *pair,
                    int32_t *row, void *xs, void *ws, size_t ws_bytes, void *stream);

/* The gradient of x: dx[t] = sum over the token's pairs of dxs[row], in slot
 * order, summed in fp32 and rounded once (zeros for a token without pairs). */
int deamoe_dispatch_backward(int32_t T, int32_t k, int32_t h, int32_t act_dtype,
                             const int32_t *row, const void *dxs, void *dx, void *stream);

/* y[t] = sum over the token's pairs of w[t, s] * ys[row[t, s]], in slot order,
 * summed in fp32 and rounded once (zeros for a token without pairs).  Weights
 * of dropped pairs and rows that no pair has are not read. */
int deamoe_combine(int32_t T, int32_t k, int32_t h, int32_t act_dtype, const int32_t *row,
                   const float *w, const void *ys, void *y, void *stream);

/* Its gradients: dys[row[t, s]] = w[t, s] * dy[t] (rows that no pair has are
 * left as they were), dw[t, s] = <dy[t], ys[row[t, s]]> in fp32 (0 for a dropped
 * pair).  dys or dw may be NULL; without dw, ys may be NULL, without dys, w. */
int deamoe_combine_backward(int32_t T, int32_t k, int32_t h, int32_t act_dtype,
                            const int32_t *row, const float *w, const void *ys, const void *dy,
                            void *dys, float *dw, void *stream);

/* --- Products with 4-bit weights and group scales.
 * A weight is (q - 8) * scale: codes [n, R, K / 2], column 2j in the low and
 * column 2j + 1 in the high four bits of byte j; scale [n, R, K / group], one
 * for `group` consecutive columns of a row, fp32 or bf16.  x [M, K] and the
 * outputs [M, R] are bf16; sums are fp32, a group's scale multiplies its whole
 * sum, results are rounded once.
 * offset (device, [n + 1], non-decreasing): rows offset[e] to offset[e + 1] of
 * x meet matrix e (the lists of deamoe_dispatch); rows outside [offset[0],
 * offset[n]) are left as they were; values outside [0, M] are taken as the
 * nearer end.  NULL: one matrix (n == 1) for all rows.
 * An infinity or NaN in a row of x makes that row of the output NaN; finite
 * values may where 31 times the sum of a group's |x| passes the fp32 range.
 * K a multiple of group; group 32, 64 or 128; any R; n <= DEAMOE_MAX_EXPERTS;
 * codes and x 16-byte aligned. */
typedef struct {
  int32_t R;            /* rows of a matrix = columns of the output */
  int32_t K;            /* columns of a matrix                      */
  int32_t n;            /* matrices                                 */
  int32_t group;        /* columns that share a scale               */
  int32_t scale_dtype;  /* DEAMOE_F32 | DEAMOE_BF16                 */
} deamoe_w4_config;

/* y = x W^T */
int deamoe_w4_linear(const deamoe_w4_config *cfg, int32_t M, const void *x, const int32_t *offset,
                     const void *codes, const void *scale, void *y, void *stream);

/* y = SiLU(x Wg^T) * (x Wu^T), both sums kept in fp32 */
int deamoe_w4_swiglu(const deamoe_w4_config *cfg, int32_t M, const void *x, const int32_t *offset,
                     const void *gate_codes, const void *gate_scale, const void *up_codes,
                     const void *up_scale, void *y, void *stream);

/* --- Norms around a block, with its gate and residual scale.
 * RMSNorm: v^ = v * r, r = 1 / sqrt(mean(v^2) + eps), eps > 0.  All tensors
 * are act_dtype, gradients of [h] parameters fp32.  Statistics, sums and
 * everything between input and output are fp32; outputs are rounded once. */

/* u = x^ * w, the input of a block.  u may be x. */
int deamoe_prenorm(int32_t T, int32_t h, int32_t act_dtype, float eps, const void *x,
                   const void *w, void *u, void *stream);

/* dx = dres + the gradient of x from du (dres: the residual path's gradient,
 * may be NULL, may be dx); dw [h] = sum over tokens of du * x^. */
int deamoe_prenorm_backward(int32_t T, int32_t h, int32_t act_dtype, float eps, const void *x,
                            const void *w, const void *du, const void *dres, void *dx, float *dw,
                            void *ws, size_t ws_bytes, void *stream);

/* z = res_scale * x + gate * (y^ * w): the block's output y joins the residual
 * stream x.  gate: NULL (1), [h] for all tokens, or [T, h].
 * u = z^ * w_next, the next block's input, of the rounded z (bit for bit what
 * deamoe_prenorm makes of z); u and w_next are both NULL or both given.  z may
 * be x. */
#define DEAMOE_GATE_NONE 0
#define DEAMOE_GATE_SHARED 1   /* [h]    */
#define DEAMOE_GATE_FULL 2     /* [T, h] */
int deamoe_postnorm(int32_t T, int32_t h, int32_t act_dtype, float eps, float res_scale,
                    int32_t gate_mode, const void *x, const void *y, const void *w,
                    const void *gate, const void *w_next, void *z, void *u, void *stream);

/* Its gradients from dz and, with a next norm, du: with d = dz + the gradient
 * of z from du, dx = res_scale * d (may be dz), dy through the norm, dw [h],
 * dgate ([h] fp32 for a shared gate, [T, h] act_dtype for a full one),
 * dw_next [h].  z, w_next, du, dw_next: all NULL or all given. */
int deamoe_postnorm_backward(int32_t T, int32_t h, int32_t act_dtype, float eps, float res_scale,
                             int32_t gate_mode, const void *y, const void *w, const void *gate,
                             const void *z, const void *w_next, const void *dz, const void *du,
                             void *dx, void *dy, float *dw, void *dgate, float *dw_next, void *ws,
                             size_t ws_bytes, void *stream);

/* Workspace of either gradient (16-byte aligned). */
int deamoe_norm_workspace_bytes(int32_t T, int32_t h, size_t *bytes);

#ifdef __cplusplus
}
#endif
#endif /* DEAMOE_H */

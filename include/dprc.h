/*
 * dprc.h -- randomized per-sample gradient-norm estimation for DP-SGD with
 * randomized clipping (DP-SGD-RC), for AMD Instinct MI355X (gfx950).
 *
 * The calls follow the problem statement of the paper "Efficient DP-SGD for
 * LLMs with Randomized Clipping":
 *   - Algorithm 2 (Norm-Estimation-Routine): per-sample squared-norm estimates
 *     of a bias-free linear layer S = A W from its activations A[B,T,d] and
 *     output gradients E = dL/dS [B,T,p], by the Hutchinson estimator
 *     (dprc_norm_hutch) or by Hutch++ (dprc_norm_hutchpp);
 *   - Algorithm 1 (DP-SGD-RC step): the squared norms summed over layers, the
 *     clip factors min(1, C/sqrt(n_i)) (dprc_clip_scale), the clipped gradient
 *     sum_i c_i A_i^T E_i that the second backward pass produces for a linear
 *     layer (dprc_clip_accumulate), and the Gaussian noise sigma*C*N(0,I)
 *     (dprc_add_noise).
 *
 * Conventions for every call:
 *   - Pointers named A, E, n2, c, grad, ws, out are DEVICE pointers; the
 *     dprc_layer array itself is HOST memory and is read during the call only.
 *   - Every call is asynchronous on `stream` (0 = the null stream) and returns
 *     after enqueueing; results are valid once the stream reaches that point.
 *   - The library never allocates or frees memory and creates no streams or
 *     events; its only host state is the opt-in, per-thread launch-trace hook
 *     (dprc_trace_launches).  Scratch space is the caller's `ws` buffer of at least the size returned
 *     by the matching *_workspace() query, 256-byte aligned.  Calls that share
 *     a workspace must be ordered (same stream, or synchronised).
 *   - Arguments are validated on the host before anything is enqueued; a
 *     failed check returns a non-zero dprc_status and enqueues nothing.  A
 *     failed launch returns DPRC_ERROR_HIP.  No C++ exception crosses the ABI.
 *   - Tensors are row-major with token rows: element (i, t, j) of A is at
 *     A + (i*T + t)*lda + j.  Pointers must be aligned to their element size
 *     (else DPRC_ERROR_NOT_SUPPORTED).  bf16 rows that start on 16-byte
 *     boundaries (16-byte aligned base, stride a multiple of 8) with a width
 *     that is a multiple of 8 take 16-byte buffer loads; other layouts take
 *     16-byte loads at the element's own address, somewhat slower (element
 *     loads for operands of fewer than 8 elements).
 *
 * Probes: +-1 (Rademacher) entries from Philox4x32-10 (Salmon et al., SC'11)
 * keyed by (seed, layer_id, stream), shared by all samples of a layer and
 * fresh per layer; the caller folds the training step into `seed`.  Column j,
 * rows 32w..32w+31 of a layer's probe matrix in stream s is word (w mod 4) of
 * Philox(counter = (w div 4, j, layer_id, s), key = (seed lo, seed hi)); bit b
 * gives row 32w+b, 0 -> +1, 1 -> -1.  Streams: 0 = Hutchinson probes (also
 * the Hutch++ residual probes), 1 = Hutch++ sketch, 2 = Gaussian noise, 3 =
 * Gaussian probes, 4 = dropout.
 */
#ifndef DPRC_H
#define DPRC_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  DPRC_SUCCESS = 0,
  DPRC_ERROR_INVALID_VALUE = 1,      /* null pointer, non-positive size, bad enum, ...   */
  DPRC_ERROR_NOT_SUPPORTED = 2,      /* alignment / stride / size outside supported range */
  DPRC_ERROR_WORKSPACE_TOO_SMALL = 3,
  DPRC_ERROR_HIP = 4,                /* a HIP runtime call or launch failed              */
  DPRC_ERROR_SCRATCH_LIMIT = 5       /* dprc_norm_hutch_clip_static: needs more scratch
                                        than DPRC_STATIC_SCRATCH_BYTES                   */
} dprc_status;

typedef enum { DPRC_F32 = 0, DPRC_BF16 = 1 } dprc_dtype;

/* Which dimension the probes sketch.  OUT sketches the p side (Z is p x k,
 * Algorithm 2 as printed), IN sketches the d side (Z is d x k; the text notes
 * the two are equivalent since ||A^T E||_F = ||E^T A||_F), AUTO sketches the
 * larger dimension (the paper's proof sketch projects the larger one), ties
 * going to OUT. */
typedef enum { DPRC_SIDE_OUT = 0, DPRC_SIDE_IN = 1, DPRC_SIDE_AUTO = 2 } dprc_side;

/* Probe family.  RADEMACHER: the counter-generated +-1 probes above.
 * HADAMARD: the deterministic Sylvester-Hadamard signs z(u,j) =
 * (-1)^popcount(u & j) (verification: with k = 2^q >= the sketched dimension
 * the estimate equals the exact squared norm).  GAUSSIAN (Hutchinson only,
 * k <= 32): the normal-law probes of Algorithm 2 (standard normal entries, the
 * estimate divided by k as for the other families), entry (u, j) from Philox
 * stream 3 block (u div 4, j, layer_id, 3) through the Box-Muller transform of
 * dprc_add_noise: words (x0, x1) give rows 4q, 4q+1 and (x2, x3) rows 4q+2,
 * 4q+3.  They are generated into the workspace as bf16 hi + lo pairs (fp32 for
 * fp32 layers) and applied as dense probe columns. */
typedef enum { DPRC_PROBE_RADEMACHER = 0, DPRC_PROBE_HADAMARD = 1, DPRC_PROBE_GAUSSIAN = 2 } dprc_probe;

/* One bias-free linear layer S = A W (section "Proposed Method"). */
typedef struct {
  const void* A;      /* activations [B,T,d], device                       */
  const void* E;      /* output gradients dL/dS [B,T,p], device            */
  int64_t B, T, d, p; /* all >= 1                                          */
  int64_t lda, lde;   /* token-row strides in elements, lda >= d, lde >= p */
  dprc_dtype dtype;   /* both tensors share it                             */
  uint32_t layer_id;  /* probe-key component; unique per layer in a step   */
} dprc_layer;

/* ---- Hutchinson (Algorithm 2, Hutch branch) --------------------------------
 * For each layer and sample i: Y_i = X_i Z (X the sketched operand, T x m,
 * Z the m x k probes), W_i = X'_i^T Y_i (X' the other operand), estimate
 * ||W_i||_F^2 / k, an unbiased estimate of ||A_i^T E_i||_F^2.
 *   n2[B]                 : = (accumulate == 0) or += (accumulate != 0) the
 *                           sum over the layers of the estimates (Algorithm 1,
 *                           layer-wise summation).  fp32, device.
 *   n2_layers[num_layers*B]: optional (may be NULL) per-layer estimates.
 *   k in [1, 256] (GAUSSIAN probes: k <= 32, else DPRC_ERROR_NOT_SUPPORTED).
 *   All layers must have the same B.
 * Workspace: dprc_norm_hutch_workspace() bytes for the same arguments (0 when
 * they are invalid).  When every layer is bf16, up to 32 groups of layers
 * keep their own token-split partials in it at once (their split sums take one
 * launch) and their own projected Y (B x T rounded up to 64, x 2 x the group's
 * columns rounded up to 16, bf16; with GAUSSIAN probes also every layer's probe
 * columns), so their projections and token reductions are batched too; it grows
 * with the number of layers up to that many groups.  GAUSSIAN calls also run, with
 * the same results, in a workspace that holds these only once (a probe buffer and a
 * Y shared by the groups), with launches per group.  Every group's tile sums (B x
 * ceil(reduced width / 128) doubles per layer) stay in it until the per-sample
 * sums of all layers at the end of the call. */
size_t dprc_norm_hutch_workspace(const dprc_layer* layers, int32_t num_layers, int32_t k,
                                 dprc_probe probe, dprc_side side);
dprc_status dprc_norm_hutch(const dprc_layer* layers, int32_t num_layers, int32_t k,
                            dprc_probe probe, uint64_t seed, dprc_side side, float* n2,
                            float* n2_layers, int32_t accumulate, void* ws, size_t ws_bytes,
                            hipStream_t stream);

/* Hutchinson estimates followed by the clip factors of Algorithm 1 in the same
 * launches: as dprc_norm_hutch, then c[i] = the dprc_clip_scale factor of the
 * final n2[i] (bitwise the same as calling dprc_clip_scale on n2).  C > 0 and
 * finite; c [B] device.  Workspace: dprc_norm_hutch_workspace(). */
dprc_status dprc_norm_hutch_clip(const dprc_layer* layers, int32_t num_layers, int32_t k,
                                 dprc_probe probe, uint64_t seed, dprc_side side, float C, float* n2,
                                 float* c, float* n2_layers, int32_t accumulate, void* ws,
                                 size_t ws_bytes, hipStream_t stream);

/* The same call for callers that cannot allocate (code under HIP graph capture,
 * tight serving loops, harnesses that forbid allocation): identical arguments and
 * results (bit for bit) to dprc_norm_hutch_clip, without the workspace.  Its scratch
 * is a static device array of DPRC_STATIC_SCRATCH_BYTES that the library's code
 * object holds on every device it runs on until the process ends; the call allocates
 * nothing and frees nothing.  A call whose dprc_norm_hutch_workspace() exceeds that
 * size returns DPRC_ERROR_SCRATCH_LIMIT and enqueues nothing (the 113-layer
 * Llama-3.2-1B stack at B = 8, T = 4096, k = 32 needs 224 MiB; GAUSSIAN calls that
 * exceed it run with launches per group as long as those fit).  `stream` must belong
 * to the current device (else DPRC_ERROR_INVALID_VALUE); the first call on a device
 * looks up that device's copy of the array (hipGetSymbolAddress) and keeps its
 * address for the process, so make that first call outside graph capture.  Every
 * call on one device shares the array: calls that overlap on one device (different
 * streams, or host threads without ordering between their streams) race on it and
 * must be serialised by the caller.  Nothing in it needs to start cleared; it keeps
 * the last call's contents. */
#define DPRC_STATIC_SCRATCH_BYTES (256u << 20)
dprc_status dprc_norm_hutch_clip_static(const dprc_layer* layers, int32_t num_layers, int32_t k,
                                        dprc_probe probe, uint64_t seed, dprc_side side, float C,
                                        float* n2, float* c, float* n2_layers, int32_t accumulate,
                                        hipStream_t stream);

/* ---- Hutch++ (Algorithm 2, Hutch++ branch; estimator section) --------------
 * With M_i = X'_i^T X_i (m probed columns): sketch O S = M_i^T (M_i S) with s
 * sketch probes (stream 1), Q = orthonormal basis of its columns (Householder
 * QR), U = M_i Q, V = M_i P - U (Q^T P) with r residual probes P (stream 0),
 * estimate ||U||_F^2 + ||V||_F^2 / r.  s in [0, 32], r in [1, 256],
 * s + r <= 256, s <= the sketched dimension.  s = 0 gives Hutchinson with r
 * probes.  A sketched dimension above 2^21 rows returns DPRC_ERROR_NOT_SUPPORTED
 * (the QR tree of 128-row blocks is at most eight levels deep).  Outputs as for
 * dprc_norm_hutch.  With several bf16 layers and s > 0, up to eight layers keep
 * their sketches, QR trees and partials in the workspace at once (each level of
 * their QR trees is one launch for all of them), so dprc_norm_hutchpp_workspace()
 * grows with the number of layers up to eight.  Everything is enqueued on
 * `stream` alone. */
size_t dprc_norm_hutchpp_workspace(const dprc_layer* layers, int32_t num_layers, int32_t s,
                                   int32_t r, dprc_side side);
dprc_status dprc_norm_hutchpp(const dprc_layer* layers, int32_t num_layers, int32_t s, int32_t r,
                              uint64_t seed, dprc_side side, float* n2, float* n2_layers,
                              int32_t accumulate, void* ws, size_t ws_bytes, hipStream_t stream);

/* ---- clip factors (Algorithm 1, scaled loss) ---------------------------------
 * c[i] = min(1, C / sqrt(n2[i])); n2 = 0 gives 1; a NaN, infinite or negative
 * n2 gives 0 (the sample is dropped).  C > 0 and finite.  Device n2[B], c[B]. */
dprc_status dprc_clip_scale(const float* n2, int64_t B, float C, float* c, hipStream_t stream);

/* ---- clipped accumulation (Algorithm 1, second backward pass) ----------------
 * grad[j*ldg + u] (=|+=) sum_i c[i] * sum_t A[i,t,j] * E[i,t,u]   (d x p, fp32)
 * i.e. the weight gradient of S = A W for the loss sum_i c_i L_i with the c_i
 * held constant.  Samples with c[i] == 0 are skipped entirely.  bf16 inputs
 * run on bf16 matrix cores with fp32 accumulation; the per-sample factor is
 * applied to the fp32 accumulator, never to the bf16 inputs.  ldg >= p. */
size_t dprc_clip_accumulate_workspace(const dprc_layer* layer);
dprc_status dprc_clip_accumulate(const dprc_layer* layer, const float* c, float* grad,
                                 int64_t ldg, int32_t accumulate, void* ws, size_t ws_bytes,
                                 hipStream_t stream);

/* The same for num_layers bf16 layers of one batch (same B; T, d and p free):
 * grads[l][j*ldg[l] + u] (=|+=) the sum above for layer l.  No layer is split over its
 * tokens, so no workspace is needed: a layer with at least 256 output tiles of
 * 256 x 256 takes a launch of its own (two when its last round of 256 tiles is at most
 * half full), and the smaller ones share launches (up to 64 layers each) where
 * dprc_clip_accumulate would split them.  grads and ldg
 * are host arrays of num_layers entries (device pointers, row strides >= p); the
 * gradients must not overlap.  Each layer's result is the one dprc_clip_accumulate
 * gives with one token split, up to the order of the fp32 sums.  Any fp32 layer gives
 * DPRC_ERROR_NOT_SUPPORTED. */
dprc_status dprc_clip_accumulate_layers(const dprc_layer* layers, int32_t num_layers, const float* c,
                                        float* const* grads, const int64_t* ldg, int32_t accumulate,
                                        hipStream_t stream);

/* ---- Gaussian noise (Algorithm 1) ---------------------------------------------
 * grad[e] += sigma * C * xi_e for e in [0, numel), xi_e standard normal from
 * Philox (stream 2) keyed by (seed, tensor_id): element e uses words of
 * block e div 4 through the Box-Muller transform with uniforms
 * (floor(x / 2^9) + 1/2) * 2^-23.  sigma >= 0, C > 0, both finite. */
dprc_status dprc_add_noise(float* grad, int64_t numel, float sigma, float C, uint64_t seed,
                           uint32_t tensor_id, hipStream_t stream);

/* ---- Private AdamW step (Algorithm 1: noise addition and optimizer step) --------
 * One AdamW step (Adam with decoupled weight decay, the optimizer of the
 * paper's private runs) on one layer's fp32 master weights, fed the private
 * gradient
 *   g[r][c] = (G[r][c] + sigma * C * xi_e) * inv_batch,   e = r * p + c,
 * where G [d, p] (row stride ldg) is the clipped gradient sum from
 * dprc_clip_accumulate and xi_e is the value dprc_add_noise(seed, tensor_id)
 * would add to element e of a contiguous [d, p] buffer (sigma = 0: none).
 * With t = hp->step (1-based), for every element:
 *   theta *= 1 - lr * weight_decay;
 *   m = beta1 m + (1 - beta1) g;   v = beta2 v + (1 - beta2) g^2;
 *   theta -= lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps).
 * theta, m, v: fp32 [d, p] with row stride ldt >= p, updated in place; G is
 * read only.  w (may be NULL) receives bf16(theta) transposed, w[c][r] with
 * row stride ldw >= d (the [p, d] weight of a linear layer), rounded to
 * nearest even.  Device pointers, fp32 ones 4-byte aligned, w 2-byte aligned;
 * 16-byte aligned rows with p a multiple of 4 take vector accesses.
 * hp: host pointer; lr >= 0, 0 <= beta1, beta2 < 1, eps > 0, step >= 1. */
typedef struct {
  float lr, beta1, beta2, eps, weight_decay;
  int32_t step;
} dprc_adamw_params;
dprc_status dprc_private_adamw(float* theta, float* m, float* v, int64_t ldt, const float* G, int64_t ldg,
                               int64_t d, int64_t p, float sigma, float C, uint64_t seed,
                               uint32_t tensor_id, float inv_batch, const dprc_adamw_params* hp,
                               uint16_t* w, int64_t ldw, hipStream_t stream);

/* ---- Dropout, residual sum and norm -------------------------------------------------
 * What lies between two linear layers of a decoder block, and the private
 * gradient of the norm's own weight and bias.
 *
 * Dropout's mask is never stored: it is a function of (seed, site_id, row, column),
 * so the backward pass makes it again.  Row r of a call is token row i*T + t.  The
 * 16 bits of element (r, c) are half (c mod 2) (0 = the low one) of word
 * (c mod 8) div 2 of Philox(counter = (c div 8, r, site_id, 4), key = (seed lo,
 * seed hi)); with q = floor(65536 p + 1/2) it is dropped iff these bits are below q
 * (p acts in steps of 2^-16).  A dropped element counts as exactly 0, also where the
 * input is infinite or NaN; a kept one is multiplied by 65536 / (65536 - q).
 * q = 0 leaves the input as it is, q = 65536 drops everything.  The caller folds
 * the training step into `seed` and gives each place in the model its site_id.  Rows
 * are counted from 0 in every call: calls on parts of a batch (micro-batches, ranks)
 * need a seed each, or they share their masks.
 *
 * All arithmetic is in fp32 on inputs of either type, each output rounded once.  Rows
 * may lie at any alignment of their element (16-byte boundaries are fastest).
 * B, T, n >= 1; B * T <= 2^31 and n <= 2^30, else DPRC_ERROR_NOT_SUPPORTED, as is a
 * pointer that is not aligned to its element.  An output may be the very tensor (same
 * pointer and row stride) that an input of the call is, where it says so; no other
 * overlap is allowed.
 *
 * dprc_dropout: out = res + dropout(x) (res may be NULL: none).  The backward pass is
 * the same call on the gradient, without res.  out may be x or res. */
dprc_status dprc_dropout(const void* x, int64_t ldx, const void* res, int64_t ldr, void* out, int64_t ldo,
                         int64_t rows, int64_t n, dprc_dtype dtype, float p, uint64_t seed, uint32_t site_id,
                         hipStream_t stream);

typedef enum { DPRC_LAYERNORM = 0, DPRC_RMSNORM = 1 } dprc_ln_kind;

/* One norm over the last axis of [B, T, n] rows, and the dropout before it. */
typedef struct {
  int64_t B, T, n;
  dprc_dtype dtype;     /* x, res, sum, y and their gradients                   */
  dprc_dtype wdtype;    /* weight, bias                                         */
  dprc_ln_kind kind;
  float eps;            /* > 0, finite (forward)                                */
  const void* weight;   /* [n], NULL = ones                                     */
  const void* bias;     /* [n], NULL = zeros (forward only)                     */
  float p;              /* dropout rate in [0, 1]                               */
  uint32_t site_id;
  uint64_t seed;
} dprc_ln;

/* Forward, per row:  s = res + dropout(x);  y = (s - mu) * rstd * weight + bias
 *   LAYERNORM: mu = mean(s), rstd = 1 / sqrt(mean((s - mu)^2) + eps)
 *   RMSNORM:   mu = 0,       rstd = 1 / sqrt(mean(s^2) + eps)
 * The norm is taken of s in fp32, before s is rounded for `sum`.  res may be NULL
 * (none); sum may be NULL (s is not wanted, or is x itself); mean (LAYERNORM only) and
 * rstd, [B*T] fp32, may be NULL (no backward pass follows).  y may be x or res,
 * sum may be x or res (y and sum must differ). */
dprc_status dprc_layernorm(const dprc_ln* L, const void* x, int64_t ldx, const void* res, int64_t ldr, void* sum,
                           int64_t lds, void* y, int64_t ldy, float* mean, float* rstd, hipStream_t stream);

/* Backward, from dy = dL/dy, s (the forward's `sum`, or x where there was none) and its
 * statistics.  With xh = (s - mu) * rstd and g = dy * weight, per row:
 *   dx = ds + rstd * (g - mean(g) - xh * mean(g * xh))       (RMSNORM: no mean(g))
 *   dh = dropout(dx)                                         (from dx before rounding)
 *   dw[i] = sum_t dy * xh,   db[i] = sum_t dy                of each sample i, [B, n] fp32
 * ds (may be NULL: zero) is the gradient that reaches s past the norm, dx is the
 * gradient with respect to s (and so res), dh that with respect to x.  Each of dx, dh,
 * dw, db may be NULL; one at least is not.  dw and db have row stride ldg >= n.  dx or dh
 * may be dy, s or ds (dx and dh must differ).  mean is read for LAYERNORM only; L->bias
 * and L->eps are not read.  With a rounded `sum` beside statistics of the unrounded row,
 * xh is off by up to 2^-8 |s| rstd in bf16, and dx and dw with it: about their own
 * rounding where a row's mean is within a few of its spreads, but up to a quarter of a
 * spread where it is 64 of them.  Such rows are better kept in fp32.  Workspace (needed
 * with dw or db): dprc_layernorm_backward_workspace() bytes (0 when the arguments are
 * invalid). */
size_t dprc_layernorm_backward_workspace(const dprc_ln* L);
dprc_status dprc_layernorm_backward(const dprc_ln* L, const void* dy, int64_t lddy, const void* s, int64_t lds,
                                    const float* mean, const float* rstd, const void* ds, int64_t ldds, void* dx,
                                    int64_t lddx, void* dh, int64_t lddh, float* dw, float* db, int64_t ldg,
                                    void* ws, size_t ws_bytes, hipStream_t stream);

/* ---- per-sample vector gradients (norm weights, biases) ------------------------------
 * G [B, n] fp32 (row stride ldg >= n) holds every sample's gradient of a vector parameter,
 * or of all of a model's side by side.  dprc_norm_vectors adds their exact squared
 * norms to the estimates of the linear layers:  n2[i] (=|+=) sum_j G[i,j]^2  (the sum
 * in fp64).  dprc_clip_accumulate_vectors is the clipped sum:
 * grad[j] (=|+=) sum_i c[i] G[i,j], samples with c[i] == 0 skipped entirely.
 * 1 <= B, n; B <= 2^24 and n <= 2^40, else DPRC_ERROR_NOT_SUPPORTED.  Workspaces: the
 * matching queries (0 bytes: none needed, ws may be NULL; also 0 for invalid sizes). */
size_t dprc_norm_vectors_workspace(int64_t B, int64_t n);
dprc_status dprc_norm_vectors(const float* G, int64_t ldg, int64_t B, int64_t n, float* n2, int32_t accumulate,
                              void* ws, size_t ws_bytes, hipStream_t stream);
size_t dprc_clip_accumulate_vectors_workspace(int64_t B, int64_t n);
dprc_status dprc_clip_accumulate_vectors(const float* G, int64_t ldg, const float* c, int64_t B, int64_t n,
                                         float* grad, int32_t accumulate, void* ws, size_t ws_bytes,
                                         hipStream_t stream);

/* ---- output head: cross entropy over a vocabulary, without its logits ---------------
 * The loss of a bias-free head S = h W^T with V outputs (the last layer of Algorithm 1's model) and the
 * gradients that it starts, with the logits l_tv = <h_t, W_v> formed in matrix-core tiles only:
 *   lse_t = log sum_v exp l_tv,  loss_t = lse_t - l_t,y(t)                        (dprc_head_loss)
 *   E_tv = g_t (exp(l_tv - lse_t) - [v = y(t)]),  g_t = dL/dloss_t               (dprc_head_errors)
 *   dh = E W,  dW = E^T h,  every sample's squared norm of h_i^T E_i             (dprc_head_backward)
 *   grad = sum_i c_i h_i^T E_i                                                   (dprc_head_clip_accumulate)
 * for the same lse and g.  A token with a negative target has no loss: loss_t = 0 and E_t = 0, and neither
 * h_t nor g_t (NaN, say) reaches any output but lse_t.  A target of V or more makes loss_t and lse_t NaN, and
 * with that lse every gradient of the token.  Products are summed in fp32, exponentials taken in fp32 (logits of
 * 1e38 or more give infinities or NaN); E is rounded to the head's dtype once (as the gradient of stored logits is),
 * then enters the products.  In dh and dW of bf16 heads the target's entry of E, by far the largest of its row, enters
 * as two bf16 numbers: the rounded one and what its rounding lost.  The norms and the clipped sum take E rounded once, as
 * dprc_head_errors gives it: they are those of one and the same per-sample gradient.
 *
 * The last four go through the vocabulary in pieces of `piece` columns, of which E is held in the workspace:
 * a positive multiple of DPRC_HEAD_BLOCK, or 0 for as many as E of 1 GiB holds (at least one block).  dh, dW
 * and grad do not depend on it beyond the rounding of their fp32 sums.
 *
 * Estimates: for the norms the head counts as ceil(V / DPRC_HEAD_BLOCK) layers of DPRC_HEAD_BLOCK outputs each,
 * with probes of their own (layer ids layer_id, layer_id + 1, ...): their gradients are disjoint columns of
 * the head's, so that the squared norms add up, and the estimate is that of dprc_norm_hutch for these
 * layers.
 *
 *   h       [B,T,d] token rows (stride ldh), W [V,d] rows (stride ldw), both of `dtype`; any alignment of
 *           the element.  bf16 rows of W on 16-byte boundaries with d a multiple of 8 are faster.
 *   target  [B*T] int64.  loss, lse, g: [B*T] fp32.
 *   dh      [B,T,d] token rows of `dtype`, may be NULL; dW [V,d] rows of `dtype`, may be NULL.  Neither may
 *           overlap an input.
 *   norms   may be NULL: k, probe, seed, side, n2 and accumulate as in dprc_norm_hutch.
 *   c       [B] fp32.  grad [d,V] fp32, row stride ldg, (=|+=) by accumulate: the layout of
 *           dprc_clip_accumulate.
 *   E       (dprc_head_errors) [B,T,nv] token rows of `dtype`, stride lde: the columns v0 .. v0 + nv of E.
 * B <= 65535, B*T <= 2^31, d <= 2^20, V <= 2^30, d*V and d*B*T <= 2^40, B*T*V <= 2^44. */
#define DPRC_HEAD_BLOCK 8192
typedef struct {
  const void* h;
  const void* W;
  const int64_t* target;
  int64_t B, T, d, V;     /* all >= 1 */
  int64_t ldh, ldw;
  dprc_dtype dtype;
  int64_t piece;
} dprc_head;
typedef struct {
  int32_t k;
  dprc_probe probe;
  uint64_t seed;
  dprc_side side;
  uint32_t layer_id;
  float* n2;              /* [B] */
  int32_t accumulate;
} dprc_head_norms;
size_t dprc_head_loss_workspace(const dprc_head* H);
dprc_status dprc_head_loss(const dprc_head* H, float* loss, float* lse, void* ws, size_t ws_bytes,
                           hipStream_t stream);
size_t dprc_head_errors_workspace(const dprc_head* H);
dprc_status dprc_head_errors(const dprc_head* H, const float* lse, const float* g, int64_t v0, int64_t nv,
                             void* E, int64_t lde, void* ws, size_t ws_bytes, hipStream_t stream);
/* dh, dW: whether they are wanted; norms: its k, probe and side. */
size_t dprc_head_backward_workspace(const dprc_head* H, int32_t dh, int32_t dW, const dprc_head_norms* norms);
dprc_status dprc_head_backward(const dprc_head* H, const float* lse, const float* g, void* dh, int64_t lddh,
                               void* dW, int64_t lddw, const dprc_head_norms* norms, void* ws, size_t ws_bytes,
                               hipStream_t stream);
size_t dprc_head_clip_accumulate_workspace(const dprc_head* H);
dprc_status dprc_head_clip_accumulate(const dprc_head* H, const float* lse, const float* g, const float* c,
                                      float* grad, int64_t ldg, int32_t accumulate, void* ws, size_t ws_bytes,
                                      hipStream_t stream);

/* ---- rotary positions -----------------------------------------------------------------
 * The pairs (a, b) of the first 2 r features of every head, turned by the angle position * freqs[j], j < r:
 *   a' = scale (a cos - b sin),  b' = scale (b cos + a sin);   inverse != 0: -sin for sin.
 * Pair j is the features (j, r + j), or (2 j, 2 j + 1) with interleaved != 0; features from 2 r on are copied.
 * The inverse call is the transpose: applied to a gradient it is the backward pass.
 *   freqs   [r] fp64, radians a position (scaled for long contexts or not, as the caller likes), device.
 *   pos     [B*T] int64 positions, device; NULL: start + t.  The angle is formed and reduced in fp64.
 *   x       `count` (1 to 4) tensors [B,T,H,D], elements of x dtype at x + b*xb + t*xt + h*xh + feature, to y
 *           likewise (ydtype).  y may be x (with its dtype and strides); otherwise outputs overlap neither
 *           inputs nor each other.
 * B*T <= 2^31, 1 <= 2 r <= D <= 2^20, r <= 4096, at most 2^16 heads and 2^30 features of a token in all. */
typedef struct {
  int64_t B, T;
  int32_t D, r;
  const double* freqs;
  const int64_t* pos;
  int64_t start;
  float scale;
  int32_t interleaved, inverse;
  dprc_dtype xdtype, ydtype;
} dprc_rope;
typedef struct {
  const void* x;
  void* y;
  int64_t H, xb, xt, xh, yb, yt, yh;
} dprc_heads;
dprc_status dprc_rotary(const dprc_rope* R, const dprc_heads* heads, int32_t count, hipStream_t stream);

/* ---- the joint norm of many tensors, and clipping ---------------------------------------
 * dprc_grad_norm: norm[0] = sqrt(sum over the tensors of x^2).  dprc_grad_clip: out = c x for every tensor, c =
 * min(1, max_norm / norm), and norm[0] (norm may be NULL).  Of a private gradient with its noise this is
 * post-processing, which costs no privacy.  Squares are summed in fp64 in a fixed order; a norm that is not
 * finite gives c = 0: zeros, as dprc_clip_scale does for such a sample.  Each tensor is rows x cols
 * elements of its own dtype, rows ldx apart, to out (row stride ldo, may be x with ldo = ldx; NULL in
 * dprc_grad_norm); outputs overlap nothing else.  A tensor may be empty (rows or cols 0).  The array is HOST
 * memory, read during the call.  max_norm > 0 and finite; rows, cols and rows * cols <= 2^40.  Workspace:
 * dprc_grad_norm_workspace() bytes. */
typedef struct {
  const void* x;
  void* out;
  int64_t rows, cols, ldx, ldo;
  dprc_dtype dtype;
} dprc_tensor;
size_t dprc_grad_norm_workspace(const dprc_tensor* tensors, int32_t count);
dprc_status dprc_grad_norm(const dprc_tensor* tensors, int32_t count, float* norm, void* ws, size_t ws_bytes,
                           hipStream_t stream);
dprc_status dprc_grad_clip(const dprc_tensor* tensors, int32_t count, float max_norm, float* norm, void* ws,
                           size_t ws_bytes, hipStream_t stream);

/* ---- Envelope CDF of the Hutchinson estimate (privacy accounting) ------------------
 * Proposition on the extremal envelope and the appendix algorithms cdf-grid and
 * binary-search-xplus.  dprc_envelope_middle evaluates MiddleRegionCDF at nx
 * points: best[e] = the largest P(S <= x[e]) over the two-level forms
 *   S(i, j, lam) = lam/(ik) chi^2(ik) + (1-lam)/(jk) chi^2(jk),
 *   i, j >= 1, i + j <= d, lam = l / (2 (n_lambda - 1)), l = 0 .. n_lambda - 1
 * (lam = 0 only when n_lambda = 1), in fp64.  arg (may be NULL) receives
 * (i, j, l) of the maximiser, the first in (i, j, l) order among equal values.
 * Each form's CDF is a convolution integral evaluated by composite
 * Gauss-Legendre quadrature (at least 16 panels of 16 nodes) over a chi density and the
 * integral of a gamma density; about 1e-12 absolute.  x, best, arg: device.  Limits:
 * 1 <= nx <= 65535, k >= 1, 2 <= d, k * d < 2^31, 1 <= n_lambda <= 4096.
 * Workspace: dprc_envelope_middle_workspace() bytes. */
size_t dprc_envelope_middle_workspace(int32_t nx, int32_t d, int32_t n_lambda);
dprc_status dprc_envelope_middle(const double* x, int32_t nx, int32_t k, int32_t d, int32_t n_lambda,
                                 double* best, int32_t* arg, void* ws, size_t ws_bytes,
                                 hipStream_t stream);

/* out[e] = P(chi^2(dof) <= x[e] * scale) for e < n (the extremal parts of the
 * envelope: dof = k, scale = k for the single coordinate; dof = scale = k d for
 * uniform weights).  dof > 0, scale > 0; x, out: device, fp64. */
dprc_status dprc_chi2_cdf(const double* x, int64_t n, double dof, double scale, double* out,
                          hipStream_t stream);

/* ---- privacy accountant (appendix: Algorithm accounting) ---------------------------
 * The accountant for DP-SGD-RC runs Poisson-subsampled Gaussian steps whose
 * effective scale a = 1/sqrt(Y) is averaged over the envelope law of Y, and
 * composes their privacy-loss distributions (PLD).  All arrays are fp64, device.
 *
 * dprc_envelope_bins: the envelope law as bins.  F[0..n_bins] holds the envelope
 * CDF at y_j = y_min + j (y_max - y_min) / n_bins; the CDF is made monotone by a
 * running maximum and clipped to [0, 1], w[j] = its increment over bin j (clamped
 * at zero) divided by the sum of the increments, ybar[j] = the bin's midpoint.  A
 * CDF with no increase on the range gives NaN weights.  n_bins >= 1, y_max > y_min.
 *
 * dprc_pld_step: one step's PLD on the cell-centred grid t_j = (j - n_half + 1) h,
 * j < 2 n_half - 1 (q, normalised with q_inf to total one), from the survival
 * function S(t) = P(L > t) at the cuts (c - n_half + 1/2) h, c < 2 n_half:
 *   S(t) = p betabar(t + s(t)) + (1 - p) alpha(t + s(t)),
 *   s(t) = log(1/p - (1 - p)/p e^-t), for t > log(1 - p); S = 1 at and below it,
 *   alpha(u) = sum_i w_i Phi(-u/mu_i - mu_i/2), betabar(u) = sum_i w_i Phi(-u/mu_i + mu_i/2),
 *   mu_i = 1 / (sigma sqrt(ybar_i))   (n_bins = 0: one term, w = 1, mu = 1/sigma).
 * q_j = S(cut j) - S(cut j + 1) clamped at zero; the mass below the first cut
 * joins q_0 and S at the last cut is the atom q_inf[0] at +infinity.  sigma > 0,
 * 0 < p <= 1, h > 0.  Workspace: dprc_pld_step_workspace(n_half) bytes (S).
 *
 * dprc_pld_fold: the composition of two PLDs on the same grid of L cells (L odd)
 * with atoms *ainf and *binf, given r[0 .. 2L - 2], their linear convolution
 * (r[j] sits at cell j - (L - 1)/2 of the result grid): negatives clipped; the
 * L centred cells kept, the mass below them added to the lowest one; the atom
 * becomes 1 - (1 - ainf)(1 - binf) plus the mass above them, rescaled with the
 * cells so that the total stays one.  q [L] and q_inf [1] must not overlap r, nor q
 * the atoms; q_inf may be ainf or binf.
 *
 * dprc_pld_delta: delta[e] = sum over t_j >= eps[e] of q_j (1 - e^(eps[e] - t_j))
 * + q_inf[0], clipped to [0, 1], t_j = (j - (L - 1)/2) h, for 1 <= n_eps <= 65535.
 */
dprc_status dprc_envelope_bins(const double* F, int32_t n_bins, double y_min, double y_max, double* ybar,
                               double* w, hipStream_t stream);
size_t dprc_pld_step_workspace(int64_t n_half);
dprc_status dprc_pld_step(double sigma, double p, double h, int64_t n_half, const double* ybar,
                          const double* w, int32_t n_bins, double* q, double* q_inf, void* ws,
                          size_t ws_bytes, hipStream_t stream);
dprc_status dprc_pld_fold(const double* r, int64_t L, const double* ainf, const double* binf, double* q,
                          double* q_inf, hipStream_t stream);
dprc_status dprc_pld_delta(const double* q, int64_t L, double h, const double* q_inf, const double* eps,
                           int32_t n_eps, double* delta, hipStream_t stream);

/* ---- probe bits (verification) -------------------------------------------------
 * out[j*ceil(m/32) + w] = packed probe word w of column j (k columns), bits of
 * rows >= m cleared.  probe selects the family; for HADAMARD, seed, layer_id
 * and stream_id are ignored.  Device out. */
dprc_status dprc_probe_bits(dprc_probe probe, uint64_t seed, uint32_t layer_id,
                            uint32_t stream_id, int64_t m, int32_t k, uint32_t* out,
                            hipStream_t stream);

/* ---- Gaussian probe values (verification) ----------------------------------------
 * out[j*m + u] = the GAUSSIAN probe entry (u, j) in fp32, u < m, j < k (k in
 * [1, 256]).  Device out. */
dprc_status dprc_probe_gaussian(uint64_t seed, uint32_t layer_id, int64_t m, int32_t k, float* out,
                                hipStream_t stream);

/* ---- per-launch timing (diagnostics, for profilers and benchmarks) ------------
 * While `events` is non-NULL, every kernel that a dprc call enqueues from THIS
 * host thread is launched with hipExtLaunchKernelGGL and start/stop events that
 * the dispatch itself stamps (no extra packets): launch j (counted from this
 * call) uses events[2j] (start) and events[2j+1] (stop),
 * kinds[j] (if kinds is non-NULL) receives its dprc_kernel_kind, and the host
 * integer *count is advanced; recording stops once *count reaches `capacity`
 * (the events array must hold 2*capacity created events).  *count is reset
 * to 0 here.  events == NULL switches the hook off.  The state is per host
 * thread and holds the caller's pointers until switched off. */
typedef enum {
  DPRC_KERNEL_PROJECT = 1,            /* Y = X Z (bf16 matrix cores)          */
  DPRC_KERNEL_TOKEN_REDUCE = 2,       /* X'^T Y, estimate or store            */
  DPRC_KERNEL_QR = 3,                 /* Hutch++ QR of 128-row blocks of O S  */
  DPRC_KERNEL_HUTCHPP_FINAL = 4,      /* Hutch++ V = W_P - U Q^T P, estimate  */
  DPRC_KERNEL_CLIP_SCALE = 5,
  DPRC_KERNEL_ACCUMULATE = 6,         /* clipped accumulation GEMM            */
  DPRC_KERNEL_SPLITK_REDUCE = 7,
  DPRC_KERNEL_NOISE = 8,
  DPRC_KERNEL_PROBE_BITS = 9,
  DPRC_KERNEL_PROJECT_F32 = 10,
  DPRC_KERNEL_TOKEN_REDUCE_F32 = 11,
  DPRC_KERNEL_SAMPLE_SQ = 12,
  DPRC_KERNEL_ACCUMULATE_F32 = 13,
  DPRC_KERNEL_TOKEN_SPLITS = 14,      /* sum of token splits per tile          */
  DPRC_KERNEL_SAMPLE_SUM = 15,        /* per-sample sum of tile squares         */
  DPRC_KERNEL_QR_COMBINE = 16,        /* QR of stacked block R factors (upper tree levels) */
  DPRC_KERNEL_QR_EXPAND = 17,         /* rows of Q per tree level; Q^T P at the first */
  DPRC_KERNEL_HUTCHPP_SUM = 18,       /* per-sample Hutch++ estimate            */
  DPRC_KERNEL_PROBE_GAUSS = 19,       /* Gaussian probe columns                  */
  DPRC_KERNEL_ADAMW = 20,             /* private AdamW step                      */
  DPRC_KERNEL_ENVELOPE = 21,          /* MiddleRegionCDF candidates and reduction */
  DPRC_KERNEL_CHI2_CDF = 22,          /* chi-squared CDF values                  */
  DPRC_KERNEL_PLD = 23,               /* accountant: bins, step PLD, fold, delta */
  DPRC_KERNEL_DROPOUT = 24,           /* dropout and residual sum                */
  DPRC_KERNEL_LAYERNORM = 25,         /* dropout, residual sum and norm          */
  DPRC_KERNEL_LAYERNORM_BACKWARD = 26,
  DPRC_KERNEL_VECTOR_NORMS = 27,      /* squared norms of per-sample vectors     */
  DPRC_KERNEL_VECTOR_SUMS = 28,       /* clipped sums of per-sample vectors      */
  DPRC_KERNEL_HEAD_SUMS = 29,         /* head: logit tiles' maxima and sums      */
  DPRC_KERNEL_HEAD_JOIN = 30,         /* head: losses and log-sum-exps           */
  DPRC_KERNEL_HEAD_ERRORS = 31,       /* head: E of a piece of the vocabulary    */
  DPRC_KERNEL_HEAD_BACK = 32,         /* head: E W (for few tokens with E^T h)    */
  DPRC_KERNEL_HEAD_ROWS = 33,         /* head: rows laid out, sums rounded       */
  DPRC_KERNEL_ROTARY = 34,
  DPRC_KERNEL_GRAD_SQUARES = 35,      /* joint norm of many tensors              */
  DPRC_KERNEL_GRAD_SCALE = 36,        /* their clipping                          */
  DPRC_KERNEL_HEAD_WEIGHT = 37        /* head: E^T h                             */
} dprc_kernel_kind;
dprc_status dprc_trace_launches(hipEvent_t* events, int32_t* kinds, int32_t capacity,
                                int32_t* count);

const char* dprc_status_string(dprc_status status);
const char* dprc_version(void);

#ifdef __cplusplus
}
#endif
#endif /* DPRC_H */

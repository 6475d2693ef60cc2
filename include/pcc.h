/*
 * pcc.h -- C ABI of libpcc: per-pixel causal-context lossless image coding on
 * one MI355X (gfx950).
 *
 * The method is the learned pixel-by-pixel coder of arXiv 2212.01185: a small
 * network maps every pixel's causal neighbourhood of already coded pixels to
 * the parameters of a discretised Gaussian mixture per colour channel
 * (Sec. III-A, Eq. (1)-(4); network Sec. III-B), an entropy coder codes the
 * sub-pixels with those distributions, the encoder evaluates all pixels in
 * parallel and the decoder proceeds as a wavefront (Sec. III-C, Eq. (6)).
 *
 * Conventions
 *   - Images are uint8, layout [n][H][W][3] (rows, columns, RGB), contiguous,
 *     in DEVICE memory.  "d_" arguments are device pointers, "h_" host pointers.
 *   - `hip_stream` is a hipStream_t passed as void* (NULL = the null stream).
 *     Kernels are launched on it; nothing else is synchronised.
 *   - Every buffer named in a call is owned by the caller; the library neither
 *     frees nor keeps it beyond the call.  A pcc_ctx owns its packed copy of
 *     the weights and a private device workspace that grows on demand
 *     (hipMalloc inside the first call that needs it, reused afterwards).
 *   - A pcc_ctx must not be used by two calls at the same time.
 *   - All functions returning int return PCC_OK (0) or a negative PCC_E_* code;
 *     no exceptions or aborts cross this boundary and damaged input cannot
 *     make a call hang (device waits are bounded).
 *
 * Weight blob (host memory): 16 little-endian uint32 header words {magic
 * "PCCW", version 1, n_layers, dims[8], K, neighbourhood size, wavefront delay
 * per row, activation id, distribution id}, then per layer W[out][in] and
 * b[out] as fp32.  Weights must be exactly representable in bf16 (biases are
 * fp32); components are Gaussian (distribution id 0, Eq. (1)) or logistic
 * (id 1, Eq. (8)).  This library accepts these models:
 *   - 30 -> 160 -> 160 -> 128 -> 60, ReLU (activation id 0), K = 5, the
 *     10-pixel neighbourhood {rows r-2, r-1 at columns c-2..c+1; row r at
 *     c-2, c-1}, delay 2 (the measured workloads);
 *   - 36 -> 128 -> 128 -> 128 -> 128 -> 36, LeakyReLU with slope 0.01 (id 1),
 *     K = 3, the 12-pixel neighbourhood {rows r-2, r-1 at columns c-2..c+2;
 *     row r at c-2, c-1}, delay 3 (the network of Sec. III-B with the
 *     hyper-parameters of Sec. IV-E);
 *   - the same shape with delay 1: the diagonal decoding order of Sec. III-C,
 *     Eq. (7).  A pass decodes the anti-diagonal r + c = t; the inputs of the
 *     three neighbours not yet decoded then, (r-2,c+2), (r-1,c+1), (r-1,c+2),
 *     carry copies of pixel (r-1,c) (zero in the first row), at the encoder too;
 *   - the six shapes of the ablations of Sec. IV-E, each the second model with
 *     one hyper-parameter changed: K = 5 (36 -> 128 x 4 -> 60), K = 7
 *     (36 -> 128 x 4 -> 84), 64 filters (36 -> 64 x 4 -> 36), 192 filters
 *     (36 -> 192 x 4 -> 36), four layers (36 -> 128 x 3 -> 36), six layers
 *     (36 -> 128 x 5 -> 36).
 * Head layout o[12 K]: for each of R,G,B: K mixture logits, K means, K
 * log-sigmas (units of 1/256 of the grey range); then K alphas, K betas,
 * K gammas of Eq. (3)-(4).
 *
 * Stream (device memory): 8 little-endian uint32 words {magic "PCC1", version
 * 2, n, H, W, K | nbhd<<8 | delay<<16 | 16<<24, distribution id, 0}, uint64 offsets[n*H+1]
 * (relative to the end of that table), then one rANS payload per image row:
 * the two initial decoder states (8 bytes each; sub-pixel i = 3 c + channel of
 * the row is coded on state i mod 2), then the 32-bit words, shared by both
 * states, in the order the decoder reads them.  Streams written by this library are read by this library; the
 * bytes depend on its floating-point evaluation order and are not portable to
 * another implementation of the same model.
 */
#ifndef PCC_H
#define PCC_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define PCC_OK 0
#define PCC_E_ARG (-1)      /* null pointer, non-positive or too large dimension */
#define PCC_E_BLOB (-2)     /* weight blob: bad magic, unsupported shape, size mismatch, non-bf16 weight */
#define PCC_E_CAP (-3)      /* output capacity too small */
#define PCC_E_STREAM (-4)   /* stream: bad header, dimensions differ, offsets out of range, payload over/under-read */
#define PCC_E_HIP (-5)      /* a HIP runtime call failed */
#define PCC_E_INTERNAL (-6) /* zero frequency or bounded device wait expired */
#define PCC_E_UNIMPL (-7)
#define PCC_E_SCRATCH (-8)  /* pcc_decode_static: the job needs more than PCC_STATIC_SCRATCH_BYTES of scratch memory */

#define PCC_HEAD_OUTPUTS 60 /* of the 30-160-160-128-60 network; in general pcc_model_info()[0] */

typedef struct pcc_ctx pcc_ctx;

/* Parse and pack the weight blob (host pointer) for device `hip_device`.
 * On success *out owns device memory until pcc_destroy.
 * Reads these environment variables, which exist for tests and measurements and
 * never change a result: PCC_ENCODE_OVERLAP (0: the row coder
 * always runs after the pixel kernel), PCC_RANS_PATIENCE (polls for a symbol
 * before a row coder running beside the pixel kernel stands down),
 * PCC_RANS_SUMS_PATIENCE (polls of a row coder's workgroup for the sizes of
 * those before it, four times as many unless set), PCC_DECODE_VARIANT (1, 2:
 * decoder workgroups per compute unit; 3: one, with bands of eight rows;
 * 0: chosen per job), PCC_DECODE_SPIN_LIMIT
 * (polls of a band for the band above before pcc_decode fails with
 * PCC_E_INTERNAL). */
int pcc_create(pcc_ctx **out, const void *h_blob, size_t blob_bytes, int hip_device);
void pcc_destroy(pcc_ctx *ctx);

/* Upper bound in bytes of the stream pcc_encode writes for n images of H x W. */
size_t pcc_stream_bound(int n, int H, int W);

/* Number of wavefront passes for an H x W image when each row trails the row
 * above by `delay` columns (right reach of the neighbourhood + 1): Eq. (6)
 * generalised, T = W + delay (H - 1).  0 for non-positive arguments. */
long pcc_wavefront_steps(int H, int W, int delay);

/* Shape of the network the ctx was created with, h_info[6] (host): head
 * outputs per pixel (12 K), K, neighbourhood size, delay, distribution id,
 * number of layers. */
int pcc_model_info(const pcc_ctx *ctx, int *h_info);

/* Network evaluation for every pixel (Sec. III-C first paragraph: at the
 * encoder all pixels are known and are processed in parallel).
 *   d_params [n][H][W][12 K] fp32: raw head outputs in the head layout above.
 *   d_bits   [n][H][W] fp32 or NULL: -log2 of the quantised joint probability
 *            of the pixel's true (r,g,b), i.e. its term of the loss Eq. (5).
 * Asynchronous: returns after the launch. */
int pcc_encode_probs(pcc_ctx *ctx, const uint8_t *d_img, int n, int H, int W,
                     float *d_params, float *d_bits, void *hip_stream);

/* Encoder (Sec. IV-C first paragraph): parameters for all pixels in parallel,
 * integer CDF values of the true sub-pixels, row-wise rANS, stream assembly.
 * Writes at most cap_bytes to d_stream and the byte count to *h_nbytes_out.
 * Synchronises hip_stream before returning (the size is read back).  The
 * stream may be written over the images: d_stream may point into them or they
 * may lie inside the buffer.  When
 * hip_stream is idle at the call, the job has at most 3072 rows and the images
 * and the stream buffer share no bytes, the row
 * coder and the stream assembly run on a stream the ctx owns, beside the
 * pixel kernel; both streams have been waited for when the call returns, so
 * the caller's view is the same.  The pixel kernel is queued first: where the
 * two streams share one of the process's hardware queues, the row coder finds all
 * symbols when it starts.  Where the pixel kernel is held up while the row coder
 * already runs (by other work in front of it, on a chip another job fills, by a
 * profiler that collects counters and runs the kernels one at a time in an order
 * of its own), the row coder gives up after PCC_RANS_PATIENCE polls (a few
 * milliseconds with the default) and is launched again behind the pixel kernel:
 * the result is the same, but such a call pays that wait.  With images of up to
 * 1024 columns the row coder's workgroups, which place their rows in the stream
 * themselves, also wait for the sizes of those before them: where the chip, full
 * of other work, starts one late, the others hold their compute units until it
 * ends or PCC_RANS_SUMS_PATIENCE polls (some 10 ms) are over, and then all rows
 * are coded again in the same way.  PCC_ENCODE_OVERLAP=0 avoids the mode
 * altogether.
 * One call at a time per ctx.  On an error return no kernel of the call is
 * still running on either stream. */
int pcc_encode(pcc_ctx *ctx, const uint8_t *d_img, int n, int H, int W,
               uint8_t *d_stream, size_t cap_bytes, size_t *h_nbytes_out, void *hip_stream);

/* Wavefront decoder (Sec. III-C): pass t decodes every pixel (r, c) with
 * delay * r + c = t.  d_img_out [n][H][W][3] is fully overwritten.  Synchronises
 * hip_stream before returning (the device status word is read back).  On
 * PCC_E_STREAM the image content is unspecified. */
int pcc_decode(pcc_ctx *ctx, const uint8_t *d_stream, size_t nbytes, int n, int H, int W,
               uint8_t *d_img_out, void *hip_stream);

/* pcc_decode for callers that cannot allocate device memory: code under HIP
 * graph capture restrictions, tight serving loops, harnesses that forbid
 * hipMalloc.  Same arguments, same result and same errors as pcc_decode, but the
 * decoder's only scratch buffer -- the mailbox through which a band of 16 rows
 * hands its last two rows to the band below, 8 bytes per pixel column and band:
 * pcc_decode_static_scratch_bytes(n, H, W), or twice that for bands of eight
 * rows, which are only used where they fit -- lives in an array of
 * PCC_STATIC_SCRATCH_BYTES that is part of the library's device code (every GPU
 * the library runs on holds it until the process ends) instead of the ctx's
 * workspace.  The call allocates and frees nothing, and clears what it uses of
 * the array with a kernel (no memset node).  A job that needs more returns
 * PCC_E_SCRATCH before anything is launched (8 MiB covers one 4096 x 2160 image
 * and 24 images of 768 x 512).  All ctxs on a GPU share that GPU's array: two
 * pcc_decode_static calls that overlap in time on one GPU race, whatever their
 * ctxs and streams.  Synchronises hip_stream before returning. */
#define PCC_STATIC_SCRATCH_BYTES (8u << 20)
size_t pcc_decode_static_scratch_bytes(int n, int H, int W);   /* 0 for invalid dimensions */
int pcc_decode_static(pcc_ctx *ctx, const uint8_t *d_stream, size_t nbytes, int n, int H, int W,
                      uint8_t *d_img_out, void *hip_stream);

/* Test hooks (not on the hot path). */

/* Eq. (1)-(4) + integer CDF rule alone: from given head outputs d_params
 * [count][12 K] and the conditioning sub-pixels d_rg [count][2] (r, g) write the
 * full tables d_cq [count][3][257] (uint32).  Asynchronous. */
int pcc_cdf_tables(pcc_ctx *ctx, const float *d_params, const uint8_t *d_rg, size_t count,
                   uint32_t *d_cq, void *hip_stream);

/* Copy the (start, freq) pairs the last pcc_encode on this ctx fed to the
 * coder: d_out [n][H][W][3] uint32, start | (freq - 1) << 16.  Asynchronous. */
int pcc_copy_intervals(pcc_ctx *ctx, uint32_t *d_out, size_t count, void *hip_stream);

/* Per-kernel timing.  With profiling enabled, pcc_encode and pcc_decode bracket
 * each kernel they launch with HIP events on the caller's stream; after the
 * call, pcc_last_timings copies the durations in milliseconds of the last such
 * call into h_ms[PCC_N_TIMINGS] (kernels that did not run: 0). */
#define PCC_T_ENCODE_PIXELS 0 /* gather + network + mixture -> (start,freq), all pixels */
#define PCC_T_ENCODE_RANS 1   /* row-wise rANS */
#define PCC_T_ENCODE_SCAN 2   /* offsets */
#define PCC_T_ENCODE_COMPACT 3 /* rows to the stream (0 where the row coder does it) */
#define PCC_T_DECODE 4        /* wavefront decode kernel */
#define PCC_N_TIMINGS 5
int pcc_set_profiling(pcc_ctx *ctx, int enabled);
int pcc_last_timings(pcc_ctx *ctx, float *h_ms);

/* ---- Training ----------------------------------------------------------
 * The operators of a training step of the codec's networks: a pixel's causal
 * context as a row of inputs, the layers' products and their backward pass,
 * the code length with its gradient (the loss Eq. (5)), the optimizer.  They
 * work on rows of several networks of one shape at once: rows
 * [offsets[g], offsets[g+1]) belong to network ("group") g, whose weights are
 * the g-th of a stacked tensor.
 *
 * These functions belong to no pcc_ctx.  They launch on hip_stream, on the
 * device that is current at the call, which all pointers belong to; they are
 * asynchronous, allocate nothing, keep nothing, use no memory but their
 * arguments and may be captured into a HIP graph.  Types are PCC_BF16,
 * PCC_FP16 and PCC_FP32.  ld... is the distance between rows in elements, at
 * least the row's length and at most 2^22.  Outputs must not overlap inputs or
 * each other (PCC_E_ARG; rows at one distance may lie beside each other, as columns
 * of one buffer).  Without any rows the pointers to rows may be NULL.  A call that
 * would take 2^32 threads or more (products of some 2^31 rows) is PCC_E_ARG. */

#define PCC_BF16 0
#define PCC_FP16 1
#define PCC_FP32 2
#define PCC_ACT_RELU 0  /* the blob's activation ids */
#define PCC_ACT_LEAKY 1 /* slope 0.01 */
#define PCC_ACT_NONE 2
#define PCC_MAX_GROUPS 65535
#define PCC_MAX_FEATURES 65536

/* Causal contexts of all pixels: row p of d_x (bf16) is the network input of
 * pixel p = (image * H + r) * W + c, value / 256 (exact), 0 outside the image,
 * in the order of the blob's first layer; `nbhd` and `delay` as in the blob
 * ((10, 2), (12, 3) or (12, 1)).  Columns 3 nbhd .. width - 1 are set to 0, so
 * that rows can be padded to a multiple of eight; columns from `width` on are
 * left as they are. */
int pcc_contexts(const uint8_t *d_img, int n, int H, int W, int nbhd, int delay,
                 void *d_x, int width, size_t ldx, void *hip_stream);

/* y_i = act(W_g x_i + b_g) for the rows i of each group g, sums in fp32.
 *   d_x [rows][in] and d_w [groups][out][in] (contiguous) of `type` bf16 or
 *   fp16; d_bias [groups][out] fp32 or NULL; d_offsets [groups + 1] int64 on
 *   the device, rising, within 0..rows.  d_y [rows][out] of `type` or fp32;
 *   rows of no group are neither read nor written. */
int pcc_grouped_linear(const void *d_x, size_t ldx, const void *d_w, const float *d_bias,
                       const int64_t *d_offsets, int groups, size_t rows, int in, int out,
                       int type, int act, void *d_y, int y_type, size_t ldy, void *hip_stream);

/* Its backward pass.  d_dz [rows][out] is the gradient before this layer's
 * activation; `x_act` is the activation that made x (PCC_ACT_NONE if none did):
 *   d_dx [rows][in]         (W_g^T dz_i) * x_act'(x_i): the gradient before the
 *                           activation of the layer in front, its dz; or NULL
 *   d_dw [groups][out][in]  sum of dz_i x_i^T over the group's rows, fp32, or NULL
 *   d_db [groups][out]      sum of dz_i, fp32, or NULL (wants d_dw too)
 * Groups without rows get zeros in d_dw and d_db.  Sums are taken in an order
 * that depends on the arguments alone: the same call gives the same bits.
 * d_workspace: pcc_grouped_linear_grad_workspace_bytes(...) bytes, aligned to
 * 16, that no other call running at the same time uses (two captured graphs
 * that may run at once need one each); PCC_E_SCRATCH if it is smaller. */
size_t pcc_grouped_linear_grad_workspace_bytes(size_t rows, int groups, int in, int out);
int pcc_grouped_linear_grad(const void *d_dz, size_t lddz, const void *d_x, size_t ldx, const void *d_w,
                            const int64_t *d_offsets, int groups, size_t rows, int in, int out,
                            int type, int x_act, void *d_dx, size_t lddx, float *d_dw, float *d_db,
                            void *d_workspace, size_t workspace_bytes, void *hip_stream);

/* Code length of given pixels under given head outputs, and its gradient.
 * With p(x) the probability of Eq. (1)-(4) (open tails; `dist` 0 Gaussian, 1
 * logistic; log-sigma clamped to -8..4, NaN as -8), the coder's integer rule
 * gives level x the share (65280 p(x) + 1) / 65536 but for rounding down to
 * whole counts, so
 *   d_bits[i] = - sum over R, G, B of log2((65280 p + 1) / 65536)
 *   d_grad[i][12 K] = scale * weight[i] * d bits[i] / d params[i], of grad_type,
 *                     rounded to nearest; 0 for a log-sigma beyond the clamp
 * (Eq. (5) is the mean of d_bits: scale = 1 / count.)
 *   d_params [count][12 K] fp32 (K 3, 5 or 7), d_rgb [count][3], d_weight
 *   [count] fp32 or NULL (all 1).  A pixel of weight 0 (padding) is not looked
 *   at: its bits and gradients are 0 whatever its parameters hold.
 * Either of d_bits and d_grad may be NULL.  d_grad may be d_params where
 * grad_type is PCC_FP32 and the ld are equal.
 * Arithmetic is in fp32 but for a level's distance from a mean (fp64), with the
 * hardware's exponential and reciprocal: gradients are some 1.5e-7 of their size
 * off, a term some 3e-5 of its own far out in a tail. */
int pcc_mixture_loss(const float *d_params, size_t ldp, const uint8_t *d_rgb, const float *d_weight, size_t count,
                     int K, int dist, float scale, float *d_bits, void *d_grad, int grad_type, size_t ldg,
                     void *hip_stream);

/* AdamW over many tensors, all in one launch.  With t = *d_step + 1, written back:
 *   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g g,
 *   param = param (1 - lr weight_decay) - lr / (1 - beta1^t) m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
 * in fp32 (the last quotient as m times a reciprocal, 1.5 units in the last place
 * off at most), and the 16-bit copy of the new param where there is one (what the
 * products read and a blob holds).
 * States in 32 bits: m, v fp32 [n].  States in 8 bits: m and the root of v as
 * e4m3 codes [n] and an fp32 scale for each 256 elements [ceil(n / 256)]; the
 * scale is the block's largest magnitude / 448, codes are rounded up or down by
 * a fixed sequence of place in the block and t, in proportion to what is
 * cut off (to the nearest, a v that changes by 0.1 % a step would never
 * move); a v above 0 never gets the code of 0.  A moment that is not finite has
 * the code of NaN, and the scale is that of the others.  The update itself uses
 * the moments before they are rounded. */
typedef struct {
    float *d_param;
    const void *d_grad;
    void *d_copy;               /* or NULL */
    void *d_m, *d_v;
    float *d_m_scale, *d_v_scale; /* 8-bit states, else NULL */
    size_t n;                   /* elements; 0 is allowed */
} pcc_adamw_tensor;

typedef struct {
    double lr, beta1, beta2, eps, weight_decay; /* betas in [0, 1); eps 0 or at least 2^-126.  With 0 an element whose
                                                   gradients were all 0 becomes 0 / 0 */
    const float *d_lr; /* device; used in place of lr if not NULL: a captured step then follows a schedule */
} pcc_adamw_hyper;

typedef struct pcc_adamw pcc_adamw;

/* Lay out the list of tensors (host array, copied) on device `hip_device`.  The
 * tensors stay the caller's, where they are, and must outlive the plan; what a step
 * writes must not overlap, nor a gradient with it (PCC_E_ARG; an fp32 gradient may be
 * its own parameter).  So must the plan outlive graphs that have captured its steps.
 * Allocates device memory and waits for the copy.  grad_type PCC_FP32, PCC_BF16 or PCC_FP16; copy_type
 * PCC_BF16 or PCC_FP16; state_bits 32 or 8. */
int pcc_adamw_create(pcc_adamw **out, const pcc_adamw_tensor *h_tensors, int count, int grad_type, int copy_type,
                     int state_bits, int hip_device);
void pcc_adamw_destroy(pcc_adamw *plan);
/* One step.  Asynchronous, allocates nothing; may be captured.  d_step: int64 on
 * the device, the number of steps taken so far.  One step of a plan at a time. */
int pcc_adamw_step(pcc_adamw *plan, const pcc_adamw_hyper *h_hyper, int64_t *d_step, void *hip_stream);

/* ---- Layers round the grouped products ---------------------------------
 * What deeper networks and mixtures of networks need beside the products, with
 * the conventions of the training operators above: they belong to no pcc_ctx,
 * are asynchronous, allocate and keep nothing, may be captured into a HIP
 * graph, and refuse outputs that overlap inputs or each other (PCC_E_ARG)
 * unless said otherwise.  Sums are taken in an order that depends on the
 * arguments alone.  A mixture runs as
 *   pcc_layer_norm -> pcc_route -> pcc_expert_sort -> pcc_expert_rows ->
 *   pcc_grouped_linear ... -> pcc_expert_join -> pcc_dropout
 * where the sort's offsets are the groups of the products. */

#define PCC_MAX_EXPERTS 1024
#define PCC_MAX_CHOICES 16

/* Layer norm of the rows of each group g:
 *   y_i = gamma_g (x_i - mean) / sqrt(mean((x_i - mean)^2) + eps) + beta_g
 *   d_x [rows][features] of `type`, d_y of y_type: the same, or of 16 bits where
 *   x is fp32.  d_gamma, d_beta [groups][features] fp32, or NULL (1 and 0).
 *   d_offsets [groups + 1] as above, or NULL for one group of all rows.  d_stats
 *   [rows][2] fp32 or NULL: each row's mean and 1 / sqrt(...), which the backward
 *   pass takes.  Rows of no group are neither read nor written.  eps is at least
 *   2^-126.
 * The mean is right to its rounding to fp32, also far from 0: a row of one value
 * has y = beta.  Squares of distances from it are summed in fp32: a finite row for
 * which that sum is infinite (distances beyond 2^64 / sqrt(features)) has
 * 1 / sqrt(...) = 0. */
int pcc_layer_norm(const void *d_x, size_t ldx, const float *d_gamma, const float *d_beta,
                   const int64_t *d_offsets, int groups, size_t rows, int features, float eps,
                   int type, void *d_y, int y_type, size_t ldy, float *d_stats, void *hip_stream);

/* Its backward pass: d_dx [rows][features] of `type` (or NULL) from d_dy of
 * y_type; d_dgamma, d_dbeta [groups][features] fp32 (both or neither): sums over
 * the group's rows, 0 for a group without any.  d_workspace:
 * pcc_layer_norm_grad_workspace_bytes(...) bytes (none without d_dgamma), aligned
 * to 16, that no other call running at the same time uses; PCC_E_SCRATCH if it is
 * smaller. */
size_t pcc_layer_norm_grad_workspace_bytes(size_t rows, int groups, int features);
int pcc_layer_norm_grad(const void *d_dy, int y_type, size_t lddy, const void *d_x, size_t ldx,
                        const float *d_stats, const float *d_gamma, const int64_t *d_offsets, int groups,
                        size_t rows, int features, int type, void *d_dx, size_t lddx, float *d_dgamma,
                        float *d_dbeta, void *d_workspace, size_t workspace_bytes, void *hip_stream);

/* The k experts with the largest logits of each token, by falling logit (equal
 * ones: the lowest index first), and their weights: the softmax over the chosen, or
 * with over_all = 1 the chosen's part of the softmax over all.
 *   d_logits [tokens][experts] of `type`; d_expert [tokens][k], d_weight
 *   [tokens][k] fp32.  1 <= k <= experts.
 * A logit of -inf is never chosen: where fewer than k are left, the other
 * choices are -1 with weight 0.  A NaN is above all numbers, and a NaN or +inf
 * among those that are summed makes the token's weights NaN. */
int pcc_route(const void *d_logits, size_t ldl, size_t tokens, int experts, int k, int type, int over_all,
              int32_t *d_expert, float *d_weight, void *hip_stream);

/* Its gradient d_dlogits [tokens][experts] of `type`, all of it written: from
 * d_dweight [tokens][k] fp32 (not looked at where the choice is -1) and what the
 * call above was given and wrote.  d_logits may be NULL where over_all is 0.  A
 * logit of -inf has gradient 0, whatever the token's other values are. */
int pcc_route_grad(const float *d_dweight, const void *d_logits, size_t ldl, const int32_t *d_expert,
                   const float *d_weight, size_t tokens, int experts, int k, int type, int over_all,
                   void *d_dlogits, size_t lddl, void *hip_stream);

/* Rows by expert: d_place [tokens][k] is the row of each choice d_expert
 * [tokens][k], those of lower experts first, those of one expert in the order of
 * the tokens (and of a token's choices); d_offsets [experts + 1]: where each
 * expert's rows begin, the groups of a grouped product.  A choice outside
 * 0..experts - 1 has place -1 and no row.  d_workspace:
 * pcc_expert_sort_workspace_bytes(...) bytes, aligned to 16, that no other call
 * running at the same time uses; PCC_E_SCRATCH if it is smaller.  tokens k is
 * below 2^31. */
size_t pcc_expert_sort_workspace_bytes(size_t tokens, int k, int experts);
int pcc_expert_sort(const int32_t *d_expert, size_t tokens, int k, int experts, int64_t *d_offsets,
                    int32_t *d_place, void *d_workspace, size_t workspace_bytes, void *hip_stream);

/* d_rows[place[t][j]] = d_x[t] for all choices with a place in 0..rows - 1; other
 * rows are left as they are.  (Its gradient is pcc_expert_join without weights.)
 * No place may stand twice. */
int pcc_expert_rows(const void *d_x, size_t ldx, const int32_t *d_place, size_t tokens, int k, size_t rows,
                    int features, int type, void *d_rows, size_t ldr, void *hip_stream);

/* d_y[t] = sum over j of weight[t][j] d_z[place[t][j]], in fp32 and in the order of
 * j; choices without a place in 0..rows - 1 are left out.  d_z [rows][features] of
 * `type`, d_y [tokens][features] of `type` or fp32, d_weight [tokens][k] fp32 or
 * NULL (all 1). */
int pcc_expert_join(const void *d_z, size_t ldz, const int32_t *d_place, const float *d_weight, size_t tokens,
                    int k, size_t rows, int features, int type, void *d_y, int y_type, size_t ldy,
                    void *hip_stream);

/* Its gradient:  d_dz[place[t][j]] = weight[t][j] d_dy[t] (rows without a choice are left as
 * they are), d_dweight[t][j] = d_dy[t] . d_z[place[t][j]] in fp32, 0 without a place.
 * Either may be NULL; d_z may be without d_dweight.  No place may stand twice. */
int pcc_expert_join_grad(const void *d_dy, int y_type, size_t lddy, const void *d_z, size_t ldz,
                         const int32_t *d_place, const float *d_weight, size_t tokens, int k, size_t rows,
                         int features, int type, void *d_dz, size_t lddz, float *d_dweight,
                         void *hip_stream);

/* y = residual + x s where an element is kept, residual where it is dropped:
 * s = 65536 / (65536 - b), b = round(65536 p), and an element is dropped if its 16
 * bits are below b (all are with p = 1).  The bits are those of Philox4x32 with ten rounds whose key is the
 * seed (low word first) and whose counter is {column / 8 | (row >> 32) << 16, row,
 * step, step >> 32}: the (column % 8)-th half word of the result, low halves first.  So
 * the same seed and step give the same mask in the backward pass (this call on the
 * gradient, without a residual), whatever the types and strides.
 *   d_x [rows][features] of `type`; d_residual [rows][features] of y_type or NULL
 *   (0); d_y of y_type: the same type or one of them fp32.  d_step: int64 on the
 *   device, or NULL for 0: a captured step has another mask each time.  d_y may
 *   be d_x where type and ld are the same, and d_residual where ld is. */
int pcc_dropout(const void *d_x, size_t ldx, const void *d_residual, size_t ldr, size_t rows, int features,
                int type, double p, uint64_t seed, const int64_t *d_step, void *d_y, int y_type, size_t ldy,
                void *hip_stream);

const char *pcc_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* PCC_H */

/*
 * ea_lm.h -- C ABI of the operators at the two ends of a language-model worker's training step, beside
 * the round of ea.h: the lookup of tokens in an embedding table and the gradient of that table, the norm
 * by which gradients are clipped, and an AdamW step over many tensors with moments in 32 or in 8 bits.
 *
 * As in ea.h: every call is asynchronous on the stream given to the init call and never synchronizes,
 * except the *_sync_status and *_selftest_* calls and ea_adamw_step_index; the library allocates no device memory, the
 * caller passes one workspace (256-byte aligned, *_workspace_bytes() bytes, untouched by anyone else until
 * the destroy call) and owns it, the stream and every tensor.  A handle belongs to the device that was
 * current at its init call, and to one host thread at a time.  All calls but the init and synchronizing ones
 * may be captured into a CUDA graph; a replay does what the calls would do again.
 *
 * Return values: EA_OK or a negative EA_E_* code of ea.h; ea_last_error(NULL) describes the calling thread's
 * last failure.  A call that is refused has done nothing.
 */
#ifndef EA_LM_H
#define EA_LM_H

#include "ea.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
typedef enum { EA_T_F32 = 0, EA_T_BF16 = 1, EA_T_F16 = 2, EA_T_I32 = 3, EA_T_I64 = 4 } ea_type;

/* ------------------------------------------------------------------------------- embedding table */

typedef struct ea_embed_config {
    int64_t vocab;       /* rows of the table, 1 .. 2^31 - 2 */
    int64_t dim;         /* its columns, 1 .. 2^20 */
    int64_t max_tokens;  /* most tokens of one call, 0 .. 2^30 */
    int64_t padding;     /* a token that takes no gradient, or -1 */
    float scale;         /* finite; the output and the gradient are multiplied by it */
} ea_embed_config;

typedef struct ea_embed ea_embed;

/* One call's tokens and rows: outer x inner of them (a batch of sequences; each >= 0).  Token (i, j) lies at
 * tokens + i * token_outer + j * token_inner (in tokens) and its row, dim consecutive elements, at
 * rows + i * row_outer + j * row_inner (in elements).  Strides may be any that stay inside the caller's
 * memory; rows that are written may not overlap. */
typedef struct ea_embed_call {
    int64_t outer, inner;
    int64_t token_outer, token_inner;
    int64_t row_outer, row_inner;
    int64_t table_stride; /* elements between the table's rows, >= dim */
    int32_t token_type;   /* EA_T_I32 or EA_T_I64 */
    int32_t row_type;     /* of y or dy: EA_T_F32, EA_T_BF16 or EA_T_F16 */
    int32_t table_type;   /* of w or dw: the same */
} ea_embed_call;

int ea_embed_workspace_bytes(const ea_embed_config *cfg, size_t *bytes);
int ea_embed_init(const ea_embed_config *cfg, void *workspace, size_t workspace_bytes, void *stream, ea_embed **out);

/* y[t, :] = scale * w[token[t], :], the product in binary32, rounded once to y's type.  The row of a token
 * outside [0, vocab) is zero, and ea_embed_sync_status reports it.  w and y: device, aligned to their
 * element. */
int ea_embed_lookup(ea_embed *h, const ea_embed_call *c, const void *tokens, const void *w, void *y);

/* The table's gradient: dw[v, :] = scale * sum of dy[t, :] over the tokens t equal to v, zero for a token
 * that does not occur and for the padding token; with accumulate = 1 that is added to what dw holds (rows
 * whose token does not occur are not touched).  Sums are formed in binary32, in an order that depends on the
 * tokens and the sizes alone (the same bits on every run), and rounded once to dw's type.  A token outside
 * [0, vocab) contributes nothing, and ea_embed_sync_status reports it. */
int ea_embed_grad(ea_embed *h, const ea_embed_call *c, const void *tokens, const void *dy, void *dw,
                  int32_t accumulate);

/* Synchronize the stream; EA_E_CUDA for a CUDA error, EA_E_DEVICE_CHECK if a token since the last such call
 * lay outside [0, vocab). */
int ea_embed_sync_status(ea_embed *h);
int ea_embed_destroy(ea_embed *h);

/* ------------------------------------------------------------------------------- gradient norm */

typedef struct ea_grad_norm_config {
    int32_t n_tensors;     /* 1 .. 2^20 */
    int32_t grad_type;     /* EA_T_F32, EA_T_BF16 or EA_T_F16 */
    const int64_t *sizes;  /* host memory, n_tensors sizes >= 0; copied */
} ea_grad_norm_config;

typedef struct ea_norm ea_norm;

int ea_grad_norm_workspace_bytes(const ea_grad_norm_config *cfg, size_t *bytes);
int ea_grad_norm_init(const ea_grad_norm_config *cfg, void *workspace, size_t workspace_bytes, void *stream,
                      ea_norm **out);

/* out[0] = N = |grad_scale| * the 2-norm of all gradients together, out[1] = grad_scale * min(1, max_norm / N)
 * (grad_scale where N = 0), the factor that takes gradients held as multiples 1 / grad_scale of themselves to
 * clipped ones.  Where N is not finite (an infinite or NaN gradient), out[1] is NaN, which ea_adamw_step takes
 * as a step to be skipped; a gradient multiplied by it would make a round's moments and residuals NaN for good.
 * Values of any magnitude count: N overflows only where it exceeds binary32.
 * grads: n_tensors device addresses in host memory, read before this returns, each aligned to its element
 * (those of empty tensors are ignored).  grad_scale: finite, not 0.  max_norm: >= 0, may be infinite.  out:
 * device, two binary32.  The same bits on every run. */
int ea_grad_norm(ea_norm *h, const void *const *grads, float grad_scale, float max_norm, float *out);
int ea_grad_norm_destroy(ea_norm *h);

/* ------------------------------------------------------------------------------- AdamW */

/* Coordinates of a tensor that share a scale of the 8-bit states; a tensor's last block may be shorter. */
#define EA_ADAMW_BLOCK 256

/* One parameter tensor and its state, device memory of the caller; every address is aligned to its element.
 * 32-bit states: m and v are size binary32 values (zero before the first step).
 * 8-bit states: m and v are size bytes, e4m3 floating-point numbers (4 exponent bits, bias 7, 3 mantissa
 * bits, no infinity, largest 448) that stand for themselves times their block's power of two in m_scale /
 * v_scale (ceil(size / EA_ADAMW_BLOCK) binary32 values); m holds the first moment, v the square root of the
 * second (zero bytes and zero scales before the first step). */
typedef struct ea_adamw_tensor {
    int64_t size;        /* >= 0 */
    void *param;
    void *m, *v;
    float *m_scale, *v_scale; /* 8-bit states only */
    void *copy;          /* NULL, or size values of copy_type that receive the new parameters too */
    float weight_decay;  /* >= 0, decoupled */
    float lr_scale;      /* >= 0, multiplies the step's lr for this tensor */
} ea_adamw_tensor;

typedef struct ea_adamw_config {
    int32_t n_tensors;              /* 1 .. 2^20 */
    int32_t param_type;             /* EA_T_F32 or EA_T_BF16 */
    int32_t grad_type;              /* EA_T_F32, EA_T_BF16 or EA_T_F16 */
    int32_t copy_type;              /* EA_T_BF16 or EA_T_F16 (of the copies, where there are any) */
    int32_t state_bits;             /* 32 or 8 */
    float beta1, beta2;             /* in [0, 1) */
    float eps;                      /* >= 1e-30 */
    uint64_t seed;                  /* Philox key of the 8-bit states' rounding */
    int64_t step;                   /* steps taken before (0 for a new run; a checkpoint's otherwise), < 2^32 */
    const ea_adamw_tensor *tensors; /* host memory, n_tensors of them; copied */
} ea_adamw_config;

typedef struct ea_adamw ea_adamw;

int ea_adamw_workspace_bytes(const ea_adamw_config *cfg, size_t *bytes);
int ea_adamw_init(const ea_adamw_config *cfg, void *workspace, size_t workspace_bytes, void *stream, ea_adamw **out);

/* Step t (1-based, counted on the device) of every tensor, with g the gradient times clip[1]:
 *   m <- beta1 m + (1 - beta1) g;  v <- beta2 v + (1 - beta2) g^2
 *   p <- p - (l weight_decay p + a m / (sqrt(v) + e)),  l = lr lr_scale,
 *   a = l sqrt(1 - beta2^t) / (1 - beta1^t),  e = eps sqrt(1 - beta2^t)
 * which is lr_scale lr ((m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps) + weight_decay p), in binary32
 * with one rounding per operation, but that the quotient is m times a reciprocal within one unit in the last place
 * (three units together; the reciprocal of a denominator above 2^126 is 0) and a's product is fused with the sum
 * after it.  p is rounded to the parameters' type, and the unrounded binary32 p to the copy's.  With 8-bit states
 * the step uses m and v as just formed; then each is scaled by the smallest power of two (>= 2^-126) that brings
 * its block's largest finite magnitude to at most 448 and rounded to e4m3 stochastically (up with the probability of the remainder, in 2^-16): coordinate j of tensor i draws word
 * j mod 4 of Philox4x32-10 at the counter (j/4 low, j/4 high, i, t - 1) under the key seed, its low half for
 * m and its high half for v; a nonzero root is never rounded to zero, and a value that is not finite is held
 * as NaN.
 * grads: n_tensors device addresses in host memory, as in ea_grad_norm.  lr: finite; an argument of the launches, so a
 * captured step is replayed with the lr of its capture (and with the device's own t and clip).  clip: device, what
 * ea_grad_norm writes, or NULL for a factor of 1.  Where clip[1] is NaN the step is skipped: nothing is
 * written and t does not advance. */
int ea_adamw_step(ea_adamw *h, const void *const *grads, float lr, const float *clip);

/* Steps taken, skipped ones not counted (synchronizes the stream). */
int ea_adamw_step_index(ea_adamw *h, int64_t *t);
int ea_adamw_destroy(ea_adamw *h);

/* Self-test of the 8-bit step's square root against the correctly rounded one, for every binary32 value below 2^60:
 * the number of values for which they differ.  Synchronizes the stream. */
int ea_adamw_selftest_sqrt(void *stream, uint64_t *unequal);

#ifdef __cplusplus
}
#endif

#endif /* EA_LM_H */

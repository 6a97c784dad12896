/*
 * forge_ops.h -- C ABI of the operators around the fused linear-layer steps of forge.h:
 *
 *   forge_rmsnorm            residual add and RMS norm, the output in bf16 and / or in fp8
 *   forge_rmsnorm_backward   its gradient
 *   forge_grad_norm          the global norm of many gradients and the clip coefficient
 *   forge_adamw_multi        one AdamW step over many tensors at once
 *
 * forge_linear_step steps the weights of linear layers and forge_input_grad yields the
 * gradient dX that leaves them; the norms stand before those layers, and the last two step
 * what no linear layer's call covers (gains, biases, embeddings, tied heads) and every
 * tensor of a run that needs the global gradient norm before any of them changes.
 *
 * The conventions of forge.h hold: row-major contiguous device tensors owned by the caller,
 * 16-byte aligned; no device memory allocated and no state kept between calls; calls only
 * enqueue on `stream`; arguments are validated on the host before any HIP call (dtype codes,
 * shapes, empty problems, pointers, hyper-parameters, alignment, aliasing, the device), and
 * NaN / Inf inputs propagate.  Sums run in an order that the sizes alone decide: a call
 * repeated on the same inputs gives the same bits.  The current device must be the one that
 * the tensors are on.  Every call may be captured into a HIP graph (kernel launches only).
 */
#ifndef FORGE_OPS_H
#define FORGE_OPS_H

#include "forge.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of this header's tensors. */
typedef enum {
    FORGE_DTYPE_F32 = 0,
    FORGE_DTYPE_BF16 = 1,
    FORGE_DTYPE_FP8 = 2   /* OCP E4M3 codes with fp32 scales, see each use */
} forge_dtype;

/* Columns that share a scale in the fp8 output of forge_rmsnorm with q_group = FORGE_Q_GROUP. */
#define FORGE_Q_GROUP 128

/*
 * forge_rmsnorm -- h = round(residual + x);  y = h / sqrt(mean_j h_j^2 + eps) * w, row by row.
 *
 *   x         [T, d]: with a residual the sublayer's output, bf16; without one the stream
 *             itself, in h_dtype
 *   residual  [T, d] in h_dtype, or NULL
 *   w         [d] gain in w_dtype
 *   h         [T, d] in h_dtype, output: the sum as it is stored, and what the norm is taken
 *             of.  Given exactly when there is a residual; may be the residual itself
 *   y         bf16 [T, d], output, or NULL
 *   q         fp8 E4M3 codes [T, d], output, or NULL: y = q * scale, scale = amax / 448 over
 *             a row (q_group 0; q_scale [T]) or over 128 columns, a shorter last group
 *             (q_group FORGE_Q_GROUP; q_scale [T, ceil(d / 128)]).  The codes are the quotient
 *             of the fp32 y, not of its bf16 form, by the scale, rounded to fp32 and from there
 *             to nearest even; amax / 448 is the product with 1/448 rounded.  Where that is no
 *             normal number (rows of zeros among them) the scale and its codes are zero; a
 *             group that holds a NaN has a NaN scale, one that holds an Inf but no NaN an Inf
 *   q_scale   fp32, output with q
 *   h_dtype, w_dtype  FORGE_DTYPE_F32 or FORGE_DTYPE_BF16
 *
 * At least one of y and q is given.  T >= 0; d a multiple of 8; T * d below 2^31.  T == 0 or
 * d == 0 returns FORGE_OK without a launch.  eps > 0, no subnormal number.  The squares are
 * summed in fp32: a row whose sum passes its largest number (values of about 10^17 on) has a
 * norm of Inf and an output of zeros.  Outputs must not overlap each other or any input, but
 * for h == residual.
 */
FORGE_API forge_status forge_rmsnorm(const void *x, const void *residual, const void *w, void *h, void *y, void *q,
                                     float *q_scale, int64_t T, int64_t d, int32_t h_dtype, int32_t w_dtype,
                                     int32_t q_group, float eps, void *stream);

/*
 * forge_rmsnorm_backward -- the gradient of forge_rmsnorm's y with respect to h and w.  With
 * s = 1 / sqrt(mean_j h_j^2 + eps) of each row:
 *
 *   dh = dres + s (dy w - h s^2 mean_j(dy_j w_j h_j))
 *   dw_j = sum over rows of dy_j h_j s
 *
 *   dy     bf16 [T, d]
 *   h      [T, d] in h_dtype: what the norm was taken of (h, or x without a residual)
 *   dres   [T, d] in h_dtype: the gradient that reaches the stream past the norm, or NULL
 *   dh     [T, d] in h_dtype, output, or NULL; may be dres itself.  It is the gradient of the
 *          residual and of x
 *   dx     bf16 [T, d], output, or NULL: the same gradient as the dY of the layer before
 *   dw     fp32 [d], output, overwritten
 *   ws     workspace of forge_rmsnorm_backward_workspace(T, d) bytes, 16-byte aligned; its
 *          contents before and after mean nothing.  Calls that may overlap in time need one each
 *
 * At least one of dh and dx is given.  T == 0 fills dw with zeros (every other pointer may be
 * NULL); d == 0 returns FORGE_OK without a launch.  ws_bytes too small: FORGE_ERR_INVALID_SHAPE.
 * Other rules as for forge_rmsnorm.
 */
FORGE_API forge_status forge_rmsnorm_backward(const void *dy, const void *h, const void *w, const void *dres, void *dh,
                                              void *dx, float *dw, int64_t T, int64_t d, int32_t h_dtype,
                                              int32_t w_dtype, float eps, void *ws, int64_t ws_bytes, void *stream);

/* Bytes of the workspace of forge_rmsnorm_backward (0 for sizes that it refuses or skips).
   The same on every device. */
FORGE_API int64_t forge_rmsnorm_backward_workspace(int64_t T, int64_t d);

/* Consecutive elements that share a scale in the fp8 state of forge_adamw_multi. */
#define FORGE_STATE_BLOCK 64

/* One tensor of a list, of any shape (numel elements, contiguous). */
typedef struct forge_tensor {
    void *W;                  /* weight in w_dtype, in/out; NULL in a list for forge_grad_norm only */
    const void *G;            /* gradient in g_dtype */
    void *m, *v;              /* state in state_dtype, in/out; unused where W is NULL */
    float *m_scale, *v_scale; /* state FORGE_DTYPE_FP8 only: fp32 [ceil(numel / 64)], in/out */
    int64_t numel;            /* 0 <= numel < 2^31 */
    float lr_scale;           /* factor of the learning rate, >= 0 */
    float weight_decay;       /* decoupled decay, finite */
    int32_t w_dtype, g_dtype; /* FORGE_DTYPE_F32 or FORGE_DTYPE_BF16 */
    int32_t state_dtype;      /* FORGE_DTYPE_F32, _BF16, or _FP8: E4M3 codes of m and of sqrt(v),
                                 each with one scale per 64 consecutive elements (a shorter last
                                 block), scale = amax / 448 of the new values themselves; a
                                 sqrt(v) > 0 is never stored as zero.  All zero for a cold start.
                                 A block with a NaN has a NaN scale.  Codes and scales come from
                                 unfused, correctly rounded fp32 operations in the order of the
                                 formulas (amax / 448 as a product with 1/448 rounded; zero where
                                 that is no normal number) */
    int32_t reserved;         /* 0 */
} forge_tensor;

/* A list as forge_tensor_list_build laid it out; plain values, to be passed on unchanged. */
typedef struct forge_tensor_list {
    int64_t table_bytes;   /* of the table */
    int64_t chunks;        /* of all tensors together */
    int32_t n;             /* tensors */
    int32_t steppable;     /* every tensor has its weight and state */
} forge_tensor_list;

/* Bytes of the table of a list: what forge_tensor_list_build fills (0 for n == 0, or where
   `tensors` is NULL, n negative or a numel out of range). */
FORGE_API int64_t forge_tensor_list_bytes(const forge_tensor *tensors, int32_t n);

/*
 * forge_tensor_list_build -- checks n tensors of any types and sizes and lays out the table
 * that the kernels read them from.  Host only: `table` is host memory of
 * forge_tensor_list_bytes(...) bytes, which the caller copies to 16-byte aligned device
 * memory; `list` is passed to the calls beside that copy.  Both stay valid for as long as
 * the tensors stay where they are; a list is read only, so that calls may share it.
 *
 * Errors: an unknown dtype code FORGE_ERR_INVALID_DTYPE; n or numel negative, or `bytes` too
 * small FORGE_ERR_INVALID_SHAPE; numel beyond 2^31 - 1, or a list of more
 * than 2^24 - 1 chunks (2048 elements of one tensor) FORGE_ERR_UNSUPPORTED_SHAPE; of a tensor with numel > 0 a NULL G, or W without m, v (or
 * the fp8 scales) FORGE_ERR_NULL_POINTER, a pointer not 16-byte aligned
 * FORGE_ERR_MISALIGNED; lr_scale or weight_decay out of range FORGE_ERR_INVALID_HYPERPARAM;
 * a weight or state tensor that overlaps any other tensor of the list (the same tensor twice
 * among them) FORGE_ERR_ALIASING.  Gradients may overlap one another.
 */
FORGE_API forge_status forge_tensor_list_build(const forge_tensor *tensors, int32_t n, void *table, int64_t bytes,
                                               forge_tensor_list *list);

/*
 * forge_grad_norm -- out[0] = sqrt(sum of the squares of all gradients of the list),
 * out[1] = min(1, max_norm / (out[0] + 1e-6)), the coefficient that clips them.
 *
 *   table    device copy of the list's table (may be NULL for an empty list, whose norm is 0)
 *   out      fp32 [2], output, 4-byte aligned; neither it nor ws in a tensor of the list
 *   ws       workspace of forge_grad_norm_workspace(list) bytes, 16-byte aligned, as in
 *            forge_rmsnorm_backward
 *   max_norm > 0, finite
 *
 * Squares are summed in fp64, so that none over- or underflows; only a norm beyond fp32's
 * largest number is stored as Inf (its coefficient is still right).  A NaN gives NaN in both,
 * an Inf a norm of Inf and a coefficient of 0.
 */
FORGE_API forge_status forge_grad_norm(const forge_tensor_list *list, const void *table, float max_norm, float *out,
                                       void *ws, int64_t ws_bytes, void *stream);

/* Bytes of the workspace of forge_grad_norm (0 where `list` is NULL). */
FORGE_API int64_t forge_grad_norm_workspace(const forge_tensor_list *list);

/*
 * forge_adamw_multi -- one AdamW step (forge_adamw's arithmetic) on every tensor of the list
 * in one launch, whatever their types and sizes:
 *
 *   g = grad_scale * G;  m, v as in forge_adamw;
 *   W <- (1 - lr lr_scale weight_decay) W - lr lr_scale mhat / (sqrt(vhat) + eps)
 *
 *   grad_scale   device pointer to one fp32 (out + 1 of forge_grad_norm, read when the step
 *                runs), 4-byte aligned, or NULL for 1; must not lie in a weight or state tensor
 *   step, lr, beta1, beta2, eps   as in forge_adamw, but for a subnormal eps, which is
 *                FORGE_ERR_INVALID_HYPERPARAM here
 *
 * With fp32 or bf16 state, lr_scale 1 and no grad_scale the results are bit-identical to
 * forge_adamw's.  The weight update reads the fp32 m' and v', not their stored forms.  A
 * list that holds a tensor without W: FORGE_ERR_NULL_POINTER.  An empty list returns FORGE_OK
 * without a launch.
 */
FORGE_API forge_status forge_adamw_multi(const forge_tensor_list *list, const void *table, float lr, float beta1,
                                         float beta2, float eps, const float *grad_scale, int64_t step, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* FORGE_OPS_H */

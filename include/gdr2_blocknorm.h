/*
 * gdr2_blocknorm.h -- C ABI of the norms before and after a block, fused with the
 * block's output gate, residual scale and residual sum (gfx950).  For every row of
 * width D (y: the block's output, x: the residual stream):
 *
 *     u = y * (mean(y^2) + eps)^(-1/2) * w_post      (w_post NULL: u = y)
 *     a = u * z / (1 + exp(-z))                      (SiLU gate z; NULL: a = u)
 *     h = x + c * a                                  (c NULL: 1; x NULL: no sum)
 *     n = h * (mean(h^2) + eps)^(-1/2) * w_pre       (w_pre NULL: no n)
 *
 * All arithmetic is fp32; h and n are each rounded once, n from the unrounded h.
 *
 * Layout and dtypes (contiguous, row-major, device memory, 16-byte aligned):
 *     y, z, n, dn, dy, dz      (rows, D)   dtype (bf16 or fp32)
 *     x, h, dh, dx             (rows, D)   stream_dtype with x given (the residual
 *                                          stream may be fp32 beside bf16 blocks),
 *                                          dtype without
 *     w_post, c, w_pre, dw_*   (D)         fp32
 * Any D from 1 to 8192.  Errors, ownership, streams and GDR2_DEBUG_SYNC as in gdr2.h;
 * rows = 0 is GDR2_OK and does nothing in the forward (the backward then sets the
 * gradients of the weights to zero).
 */
#ifndef GDR2_BLOCKNORM_H_
#define GDR2_BLOCKNORM_H_

#include "gdr2.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct gdr2_blocknorm {
  int64_t rows;         /* >= 0 */
  int32_t D;            /* 1 .. 8192 */
  int32_t dtype;        /* gdr2_dtype of y, z, n */
  int32_t stream_dtype; /* gdr2_dtype of x, h; must be dtype or GDR2_FP32 */
  float eps;            /* finite, >= 0 */
} gdr2_blocknorm;

/* h may be NULL where n is wanted alone. */
gdr2_status gdr2_blocknorm_fwd(const gdr2_blocknorm* problem, const void* y, const float* w_post, const void* z,
                               const void* x, const float* c, const float* w_pre, void* h, void* n,
                               hipStream_t stream);

/* Bytes of workspace of the backward (partial sums of the weights' gradients). */
gdr2_status gdr2_blocknorm_workspace_bytes(const gdr2_blocknorm* problem, size_t* bytes);

/* Gradients of sum <h, dh> + <n, dn>, everything else formed again from the inputs.
 * dh may be NULL (zero) where w_pre is given; dn is given exactly where w_pre is.
 * dw_post, dz, dx, dc and dw_pre are given exactly where w_post, z, x, c and w_pre
 * are (dx may be NULL: not wanted). */
gdr2_status gdr2_blocknorm_bwd(const gdr2_blocknorm* problem, const void* y, const float* w_post, const void* z,
                               const void* x, const float* c, const float* w_pre, const void* dh, const void* dn,
                               void* dy, float* dw_post, void* dz, void* dx, float* dc, float* dw_pre, void* ws,
                               size_t ws_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* GDR2_BLOCKNORM_H_ */

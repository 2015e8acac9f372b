/*
 * gdr2_dropout.h -- C ABI of dropout with the block's residual sum (gfx950).  For every
 * element e of a tensor, counted from 0 in memory order:
 *
 *     y_e = r_e + k_e x_e / (1 - p)          (r NULL: no sum)
 *     dx_e = k_e dy_e / (1 - p)              (r's gradient is dy itself)
 *
 * k_e is 1 where word e of a counter-based generator is at least p 2^32 (rounded to a whole number,
 * halves to even, and 2^32 - 1 at most), else 0, and is formed again where it is needed: no mask is stored.  Words are
 * those of Philox 4x32 with ten rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as
 * easy as 1, 2, 3", SC 2011): word e is word e % 4 of the block with counter (e / 4, offset), each
 * 64 bits, low half first, and key `seed`.  Calls with the same seed and offset drop the same
 * elements, at any size: a program takes another offset for each dropout of each step.
 *
 * Layout and dtypes (contiguous, device memory, 16-byte aligned):
 *     x, dx          n elements    dtype (bf16 or fp32)
 *     r, y, dy       n elements    stream_dtype: dtype, or fp32 (a 32-bit residual stream)
 * The product and the sum are fp32, y and dx are rounded once.  A dropped element contributes
 * zero whatever its value.  y may be r or, of one dtype, x; dx may be dy of one dtype.
 *
 * Errors, ownership, streams and GDR2_DEBUG_SYNC as in gdr2.h; n = 0 is GDR2_OK and does nothing.
 */
#ifndef GDR2_DROPOUT_H_
#define GDR2_DROPOUT_H_

#include "gdr2.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct gdr2_dropout {
  int64_t n;            /* 0 .. 2^40 */
  double p;             /* 0 <= p < 1 */
  uint64_t seed;
  uint64_t offset;
  int32_t dtype;        /* gdr2_dtype of x, dx */
  int32_t stream_dtype; /* gdr2_dtype of r, y, dy; must be dtype or GDR2_FP32 */
} gdr2_dropout;

/* `more` (8-byte aligned, may be NULL) is a value in device memory that is added to
 * problem->offset, modulo 2^64, when the kernel runs: a captured call that is replayed drops
 * other elements each time if the program advances it. */
gdr2_status gdr2_dropout_fwd(const gdr2_dropout* problem, const uint64_t* more, const void* x, const void* r, void* y,
                             hipStream_t stream);

gdr2_status gdr2_dropout_bwd(const gdr2_dropout* problem, const uint64_t* more, const void* dy, void* dx,
                             hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* GDR2_DROPOUT_H_ */

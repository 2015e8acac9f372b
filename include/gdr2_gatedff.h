/*
 * gdr2_gatedff.h -- C ABI of the gated feed-forward block (gfx950), the part of a layer behind
 * its token mixer.  For every row x of width D, with F hidden channels:
 *
 *     g = x Wg^T,   u = x Wu^T,   h = act(g) * u,   y = h Wd^T
 *
 * act is SiLU, g / (1 + exp(-g)), or GELU, g (1 + erf(g / sqrt 2)) / 2.
 *
 * Layout and dtypes (contiguous, row-major, device memory, 16-byte aligned), all of
 * problem->dtype (bf16 or fp32):
 *     x, y, dy, dx      (rows, D)
 *     Wg, Wu, dWg, dWu  (F, D)
 *     Wd, dWd           (D, F)
 * D and F are multiples of 8 up to 65536, rows up to 2^24 and rows D and rows F below 2^36, else
 * GDR2_EUNSUPPORTED.  rows = 0 is GDR2_OK: the forward does nothing, the backward sets the gradients
 * of the weights to zero.
 * Products accumulate in fp32.  bf16 problems round h, and backward the gradients at g and u, to
 * bf16 once on their way into the products that read them; the backward reads g and u in 11 bits of
 * their own (a power of two for each row and 32 channels beside them), whether saved or formed again.
 *
 * Errors, ownership, streams and GDR2_DEBUG_SYNC as in gdr2.h.  The same call gives the same bits.
 */
#ifndef GDR2_GATEDFF_H_
#define GDR2_GATEDFF_H_

#include "gdr2.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum gdr2_act { GDR2_ACT_SILU = 0, GDR2_ACT_GELU = 1 } gdr2_act;

typedef struct gdr2_gatedff {
  int64_t rows;  /* 0 .. 2^24 */
  int32_t D, F;  /* multiples of 8 */
  int32_t dtype; /* gdr2_dtype */
  int32_t act;   /* gdr2_act */
} gdr2_gatedff;

/* Bytes of device workspace (for_backward = 0: forward; 1: backward, and a forward with
 * save = 1). */
gdr2_status gdr2_gatedff_workspace_bytes(const gdr2_gatedff* problem, int for_backward, size_t* bytes);

/* Forward.  save = 1 leaves g, u and h in ws (sized for the backward). */
gdr2_status gdr2_gatedff_fwd(const gdr2_gatedff* problem, const void* x, const void* Wg, const void* Wu, const void* Wd,
                             void* y, void* ws, size_t ws_bytes, int save, hipStream_t stream);

/* Gradients of sum <y, dy>.  dx may be NULL (not wanted), and so may dWg, dWu and dWd together
 * (frozen weights); not all four.  saved = 1 takes what a save = 1 forward with the same
 * problem, x, Wg and Wu left in ws, and leaves it there; saved = 0 forms it again. */
gdr2_status gdr2_gatedff_bwd(const gdr2_gatedff* problem, const void* x, const void* Wg, const void* Wu, const void* Wd,
                             const void* dy, void* dx, void* dWg, void* dWu, void* dWd, void* ws, size_t ws_bytes,
                             int saved, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* GDR2_GATEDFF_H_ */

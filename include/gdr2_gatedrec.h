/*
 * gdr2_gatedrec.h -- C ABI of the gated linear recurrence (gfx950): the recurrence of
 * gdr2_linattn.h with a state of one value a channel and a decay of each token and channel.
 * For every batch row and channel:
 *
 *     h_t = a_t h_{t-1} + m_t i_t x_t,     a_t = exp(g_t),     o_t = h_t
 *
 * g is the log-decay, g <= 0; i is the input gate (NULL: 1); m_t = 1, or with
 * problem->normalize m_t = sqrt(1 - a_t^2), which keeps the variance of h at that of i x.
 * (A normalized token with g = 0 has m = 0, whose slope in g is infinite: the gradient at its
 * g leaves that term out.)
 *
 * Layout and dtypes (contiguous, row-major, device memory, 16-byte aligned; cu_seqlens
 * 4-byte aligned):
 *     x, i, o, dout, dx, di   (B, T, D)   problem->dtype (bf16 or fp32)
 *     g, dg                   (B, T, D)   fp32
 *     h0, h_T, h, dh_T, dh0   (B, D), packed (n_seqs, D)   fp32
 * Any D from 1 to 65536, and fewer than 2^23 workgroups, which take 64 tokens of 128 channels each (64
 * where D is odd or at most 64): fewer than 2^29 tokens (B T) of up to 64 channels, 2^25 of 2048.  Up to 2^24 packed
 * sequences, and fewer than 2^32 states with D rounded up to 256.  Else GDR2_EUNSUPPORTED, token by
 * token too.  States are fp32 throughout; o and the gradients are rounded once.
 *
 * Packed batches (B = 1, n_seqs > 0): cu_seqlens (n_seqs + 1) holds the sequences' offsets,
 * 0 <= cu_seqlens[0] <= ... <= cu_seqlens[n_seqs] <= T; n_seqs = 0: fixed length, cu_seqlens
 * ignored.  Rows outside every sequence are neither read into a result nor written.  An empty
 * sequence passes h0 to h_T and dh_T to dh0.  A sequence's values never meet another's, NaN
 * and infinities neither.
 *
 * Errors, ownership, streams and GDR2_DEBUG_SYNC as in gdr2.h; calls that share a workspace have to follow
 * one another (one stream, or an event between).  Calls that overlap on one end, but their outputs are
 * unspecified: wrong, unwritten or NaN.  The same call gives the same bits.
 */
#ifndef GDR2_GATEDREC_H_
#define GDR2_GATEDREC_H_

#include "gdr2.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct gdr2_gatedrec {
  int32_t B, T, D;
  int32_t dtype;     /* gdr2_dtype of x, i, o and their gradients */
  int32_t normalize; /* 0: m = 1; 1: m = sqrt(1 - a^2) */
} gdr2_gatedrec;

/* Bytes of device workspace (for_backward = 0: forward; 1: backward, and a forward with
 * save = 1).  At least 256. */
gdr2_status gdr2_gatedrec_workspace_bytes(const gdr2_gatedrec* problem, int32_t n_seqs, int for_backward,
                                          size_t* bytes);

/* Forward.  i, h0 and h_T may be NULL (no gate, zero start, final state not wanted).  save = 1
 * leaves the states that the backward starts from in ws (sized for the backward). */
gdr2_status gdr2_gatedrec_fwd(const gdr2_gatedrec* problem, const int32_t* cu_seqlens, int32_t n_seqs, const void* x,
                              const float* g, const void* i, const float* h0, void* o, float* h_T, void* ws,
                              size_t ws_bytes, int save, hipStream_t stream);

/* Gradients of sum <o, dout> + <h_T, dh_T>.  h0, dh_T and dh0 may be NULL (zero, not wanted); di
 * is given exactly where i is.  saved = 1 takes the states that a save = 1 forward with the same
 * problem, cu_seqlens, x, g, i and h0 left in ws, and leaves them there; saved = 0 forms them again. */
gdr2_status gdr2_gatedrec_bwd(const gdr2_gatedrec* problem, const int32_t* cu_seqlens, int32_t n_seqs, const void* x,
                              const float* g, const void* i, const float* h0, const void* dout, const float* dh_T,
                              void* dx, float* dg, void* di, float* dh0, void* ws, size_t ws_bytes, int saved,
                              hipStream_t stream);

/* Token by token for decoding: h (fp32) is updated in place over the call's tokens.  No
 * workspace. */
gdr2_status gdr2_gatedrec_step(const gdr2_gatedrec* problem, const int32_t* cu_seqlens, int32_t n_seqs, const void* x,
                               const float* g, const void* i, float* h, void* o, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* GDR2_GATEDREC_H_ */

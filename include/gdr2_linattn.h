/*
 * gdr2_linattn.h -- C ABI of linear attention with a decay for each head (gfx950),
 * the recurrence of gdr2.h without the erase term and with one decay per value head
 * in place of one per key channel.  For every batch row and value head, with state
 * S in R^{Dk x Dv}:
 *
 *     S_t = exp(g_t) S_{t-1} + k_t v_t^T,      o_t = scale * S_t^T q_t
 *
 * g is the log-decay, g <= 0 (log_decay = -inf, or any value below -200, forgets the
 * state).  `decay` says where it comes from:
 *     GDR2_DECAY_TOKEN   g (B, T, Hv): one value for each token and value head;
 *     GDR2_DECAY_HEAD    g (Hv): one value for each value head, the same for every
 *                        token; its gradient is the sum over batch and tokens.
 *
 * The problem description, layouts, dtypes, grouped value heads, packed batches
 * (cu_seqlens and n_seqs > 0; n_seqs = 0: fixed length, cu_seqlens ignored), errors,
 * ownership, streams and GDR2_DEBUG_SYNC are those of gdr2.h:
 *     q, k                  (B, T, H, Dk)     problem->dtype
 *     v, o, dout            (B, T, Hv, Dv)    problem->dtype
 *     g, dg                 (B, T, Hv) or (Hv)            fp32
 *     S0, S_T, S, dS_T, dS0 (B, Hv, Dk, Dv), packed (n_seqs, Hv, Dk, Dv)   fp32
 * A token has at most 2^22 values over all heads in a chunk call (Hv * max(Dk, Dv),
 * else GDR2_EUNSUPPORTED).  Pointers are 16-byte aligned (cu_seqlens: 4-byte).  Outputs
 * are overwritten.  An empty sequence of a packed batch passes S0 to S_T and dS_T to dS0.
 *
 * A non-finite value in a token's q, k, v or dout reaches the outputs of its own
 * 64-token chunk on both sides of the token, and what follows from the state: the tokens
 * behind the chunk and S_T from k and v, those before it and dS0 from q and dout.  In bf16
 * problems one in k or v also reaches dg of up to 1023 tokens before it, for the decays'
 * gradient is summed backwards over stretches of 1024 tokens from the state behind them.
 * With GDR2_DECAY_HEAD, dg of a head is a sum over all of these.
 */
#ifndef GDR2_LINATTN_H_
#define GDR2_LINATTN_H_

#include "gdr2.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum gdr2_decay { GDR2_DECAY_TOKEN = 0, GDR2_DECAY_HEAD = 1 } gdr2_decay;

/* Bytes of device workspace of a chunk call (for_backward = 0: forward; 1: backward,
 * and a forward with save = 1). */
gdr2_status gdr2_linattn_workspace_bytes(const gdr2_problem* problem, int32_t n_seqs, int for_backward,
                                         size_t* bytes);

/* Chunk forward.  S0 and S_T may be NULL (zero start, final state not wanted).
 * save = 1 leaves the states that the backward starts from in ws (sized for the
 * backward). */
gdr2_status gdr2_linattn_fwd(const gdr2_problem* problem, int32_t decay, const int32_t* cu_seqlens, int32_t n_seqs,
                             const void* q, const void* k, const void* v, const float* g, const float* S0, void* o,
                             float* S_T, void* ws, size_t ws_bytes, int save, hipStream_t stream);

/* Gradients of sum <o, dout> + <S_T, dS_T>.  S0, dS_T and dS0 may be NULL (zero, not
 * wanted).  dq, dk (B,T,H,Dk), dv (B,T,Hv,Dv) in problem->dtype; dg fp32, shaped as g.
 * saved = 1 takes the states that a save = 1 forward with the same problem, decay,
 * cu_seqlens, k, v, g and S0 left in ws; saved = 0 forms them again. */
gdr2_status gdr2_linattn_bwd(const gdr2_problem* problem, int32_t decay, const int32_t* cu_seqlens, int32_t n_seqs,
                             const void* q, const void* k, const void* v, const float* g, const float* S0,
                             const void* dout, const float* dS_T, void* dq, void* dk, void* dv, float* dg,
                             float* dS0, void* ws, size_t ws_bytes, int saved, hipStream_t stream);

/* Token by token for decoding: S (fp32) is updated in place over the call's tokens
 * (problem->T >= 1 a sequence; `chunk` is ignored).  No workspace. */
gdr2_status gdr2_linattn_step(const gdr2_problem* problem, int32_t decay, const int32_t* cu_seqlens, int32_t n_seqs,
                              const void* q, const void* k, const void* v, const float* g, float* S, void* o,
                              hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* GDR2_LINATTN_H_ */

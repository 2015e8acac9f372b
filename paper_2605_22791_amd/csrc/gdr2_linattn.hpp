// Linear attention with a decay for each head: what its kernels share and the launch
// interface between them and gdr2_linattn_api.hip.  Per value head, with
// G_r = sum_{j<=r} g_j inside a chunk of C = 64 tokens and D_rs = exp(G_r - G_s), r >= s:
//
//     o_r  = scale (exp(G_r) S0^T q_r + sum_{s<=r} D_rs (q_r . k_s) v_s)
//     S_C  = exp(G_C) S0 + sum_s exp(G_C - G_s) k_s v_s^T
//
// and backward, dS the gradient of the chunk's end state:
//
//     dq_r = scale (exp(G_r) S0 do_r + sum_{s<=r} D_rs (do_r . v_s) k_s)
//     dk_s = exp(G_C - G_s) dS v_s   + scale sum_{r>=s} D_rs (do_r . v_s) q_r
//     dv_s = exp(G_C - G_s) dS^T k_s + scale sum_{r>=s} D_rs (q_r . k_s) do_r
//     dS0  = exp(G_C) dS + scale sum_r exp(G_r) q_r do_r^T
//     dg_t = E + sum_{r>=t} a_r + sum_{s<t} b_s + sum_{r>=t>s} W_rs
//
// with W_rs = scale D_rs (q_r . k_s)(do_r . v_s), a_r = scale exp(G_r) q_r^T S0 do_r,
// b_s = exp(G_C - G_s) k_s^T dS v_s and E = exp(G_C) <S0, dS>: every pair of a write at
// or before t and a read at or after t passes the decay of t once.
#pragma once

#include "gdr2_kernels.hpp"

namespace gdr2 {

// Log-decays below this forget the state (exp(-200) = 1.4e-87 is zero in fp32, also
// times the largest state), -inf among them; cut off there, sums of a chunk's decays
// and their differences stay finite.
constexpr float kLaForget = -200.f;

// Where a call's tokens, chunks and decays are.
struct LaGeo {
  Varlen vl{};
  int B, T, H, G, NT;  // H value heads, G of them per key head; NT chunks a sequence, or chunk slots (packed)
  float scale;
  const float* g;  // (B, T, H), or (H) with per_head
  int per_head;
};

__device__ __forceinline__ float la_decay_at(const LaGeo& a, size_t row, int h) {
  const float g = a.per_head ? a.g[h] : a.g[row * a.H + h];
  return g < kLaForget ? kLaForget : g;
}

// ---- fp32 problems: chunk-parallel passes ----------------------------------
struct LaFwdArgs {
  LaGeo geo;
  const float *q, *k, *v;
  float* o;
  const float* N;  // states that enter the chunks
};

struct LaBwdArgs {
  LaGeo geo;
  const float *q, *k, *v, *dout;
  float *dq, *dk, *dv;
  float *Pq, *Pk;  // grouped heads: dq, dk of each value head (rows, H, Dk), else null
  float* dg;       // (rows, H)
  const float *N, *M;  // as above, and the gradients of the states behind them
};

// N_n = sum_s w_s x_s z_s^T of every chunk, w_s = exp(G_C - G_s), or scale exp(G_s) (rev)
struct LaStateArgs {
  LaGeo geo;
  const float *x, *z;
  float *N, *eGC;
};

// N (per chunk: the sum above) becomes the state that enters the chunk, from the
// first chunk on (rev: from the last one back); fin: the state behind the last.
struct LaCombineArgs {
  LaGeo geo;
  float* N;
  const float *eGC, *init;  // init nullable
  float* fin;               // nullable
  int nseq, size, rev;      // sequences, Dk * Dv
};

// ---- bf16 problems: scans over segments ------------------------------------
// A sequence is cut into segments of seg_tokens tokens (a multiple of 64; an empty
// sequence has one without tokens); slot = sequence * nseg + segment, or, packed, an
// entry of a table: first token, tokens and sequence of every slot, and the first
// slot of every sequence.  Up to 64 sequences need no table: a wave looks a slot up in
// the offsets, a sequence a lane (nine prompts of 8192 tokens in all: 84 us a
// forward call, 87 with the launch that writes the table and the reads of it).
struct LaSegs {
  const int *t0 = nullptr, *len = nullptr, *seq = nullptr, *off = nullptr;  // packed only
  const int* cu = nullptr;  // packed, up to 64 sequences: in place of the table
  int nseq, nseg, nslot, seg_tokens;
};

// Chunks between two of the points where the decay gradient's running sum starts anew
// from <S, dS> (LaScanArgs).
constexpr int kLaAnchor = 16;

struct LaScanArgs {
  LaGeo geo;
  LaSegs segs;
  const bf16_t *q, *k, *v, *dout;
  const float *S0, *dST;  // nullable
  float *S, *dS, *dec;    // states behind the segments (gradients before them), exp(sum g): (slot, H)
  bf16_t* o;
  float *ST, *dS0;  // nullable
  bf16_t *dq, *dk, *dv;
  float *Pq, *Pk;        // grouped heads: dq, dk of each value head
  float *pa, *pb;        // q . dq and v . dv without the diagonal (rows, H)
  float *ca, *cb;        // sixteen parts of their chunk's sum of what comes from the state (slot, H, chunks a segment)
  float *aS, *aD;        // S and dS at the anchors inside segments, S at the last one's end (slot, H, anchors a segment)
  float* dg;             // (rows, H)
  int anchors;
};

template <int DK, int DV>
hipError_t launch_la_segstate(const LaScanArgs& a, bool rev, hipStream_t st);
hipError_t launch_la_segcombine(const LaScanArgs& a, int size, bool rev, hipStream_t st);
template <int DK, int DV>
hipError_t launch_la_scan_fwd(const LaScanArgs& a, hipStream_t st);
template <int DK, int DV>
hipError_t launch_la_scan_bwd(const LaScanArgs& a, hipStream_t st);
hipError_t launch_la_segtable(const int* cu, const LaSegs& s, int T, int* t0, int* len, int* seq, int* off, hipStream_t st);

template <typename TIn>
struct LaStepArgs {
  const TIn *q, *k, *v;
  const float* g;
  float* S;
  TIn* o;
  const int* cu;  // null: B sequences of T tokens
  int nseq, T, H, G, per_head;
  float scale;
};

template <int DK, int DV>
hipError_t launch_la_state(const LaStateArgs& fwd, const LaStateArgs& rev, hipStream_t st);  // of N null: none
hipError_t launch_la_combine(const LaCombineArgs& fwd, const LaCombineArgs& rev, hipStream_t st);  // of N null: none
template <int DK, int DV>
hipError_t launch_la_fwd(const LaFwdArgs& a, hipStream_t st);
template <int DK, int DV>
hipError_t launch_la_bwd(const LaBwdArgs& a, hipStream_t st);
template <int DK, int DV, typename TIn>
hipError_t launch_la_step(const LaStepArgs<TIn>& a, hipStream_t st);
// out[r][h][c] = sum over the group's value heads of P[r][h G + j][c]
template <typename TOut>
hipError_t launch_la_group(const float* Pq, const float* Pk, TOut* dq, TOut* dk, size_t rows, int Hk, int G, int D, hipStream_t st);
// dg[h] = sum over the rows of P[r][h]
hipError_t launch_la_headsum(const float* P, float* dg, size_t rows, int H, hipStream_t st);

}  // namespace gdr2

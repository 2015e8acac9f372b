// Gated linear recurrence (include/gdr2_gatedrec.h): the launch interface between the C ABI and
// the kernels.
#pragma once

#include "gdr2_kernels.hpp"

namespace gdr2 {

constexpr int kRecTile = 128;  // tokens of a workgroup's tile, forward and backward

// What tiles hand to the tiles behind them, in the order in which they are taken: pref (tiles, D) the
// state behind a tile, agg (tiles, D, 2) the factor and the addend that a tile takes it there by.
// All ones: not there yet.
struct RecChain {
  float* pref;
  float* agg;
  uint32_t* ticket;  // the next tile to take; zero before the launch
};

template <typename T>
struct RecArgs {
  const T *x, *i;       // i nullable
  const float *g, *h0;  // h0 nullable
  const int32_t* cu;    // packed: nseq + 1 offsets; else NULL
  T* o;                 // nullable: the chain's states alone
  float* hT;            // nullable
  RecChain chain;
  int nseq, len;        // sequences; tokens of one (fixed length) or of the batch
  int rows, D, normalize;
};

template <typename T>
struct RecBwdArgs {
  const T *x, *i, *dout;
  const float *g, *h0, *dhT;
  const float* states;  // behind every tile, (tiles, D)
  const int32_t* cu;
  T *dx, *di;
  float *dg, *dh0;
  RecChain chain;
  int nseq, len;
  int rows, D, normalize;
};

template <typename T>
struct RecStepArgs {
  const T *x, *i;
  const float* g;
  const int32_t* cu;
  T* o;
  float* h;
  int nseq, len;
  int D, normalize;
};

template <typename T>
hipError_t launch_rec_fwd(const RecArgs<T>& a, hipStream_t st);
template <typename T>
hipError_t launch_rec_bwd(const RecBwdArgs<T>& a, hipStream_t st);
template <typename T>
hipError_t launch_rec_step(const RecStepArgs<T>& a, hipStream_t st);
// `chains` chains of `words` 16-byte words each: all ones, the first 256 bytes zero
hipError_t launch_rec_clear(void* p, size_t words, int chains, hipStream_t st);

}  // namespace gdr2

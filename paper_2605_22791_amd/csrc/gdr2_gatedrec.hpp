// Gated linear recurrence (include/gdr2_gatedrec.h): the launch interface between the C ABI and
// the kernels.
#pragma once

#include "gdr2_kernels.hpp"

namespace gdr2 {

template <typename T>
struct RecArgs {
  const T *x, *i;        // i nullable
  const float *g, *h0;   // h0 nullable
  const int32_t* cu;     // packed: nseq + 1 offsets; else NULL
  T* o;
  float* hT;             // nullable; step: the states in place (h0 too)
  float* hs;             // nullable: h of every token, (B T, D)
  int nseq, len;         // sequences; tokens of one (fixed length) or of the batch
  int D, normalize;
};

template <typename T>
struct RecBwdArgs {
  const T *x, *i, *dout;
  const float *g, *h0, *dhT, *hs;
  const int32_t* cu;
  T *dx, *di;
  float *dg, *dh0;
  int nseq, len;
  int D, normalize;
};

template <typename T>
hipError_t launch_rec_fwd(const RecArgs<T>& a, hipStream_t st);
template <typename T>
hipError_t launch_rec_bwd(const RecBwdArgs<T>& a, hipStream_t st);

}  // namespace gdr2

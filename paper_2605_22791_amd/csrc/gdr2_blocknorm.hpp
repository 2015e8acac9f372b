// Norms before and after a block with its gate and residual scale (include/gdr2_blocknorm.h):
// the launch interface between the C ABI and the kernels.
#pragma once

#include "gdr2_kernels.hpp"

namespace gdr2 {

// T: y, z, n; TS: x, h (TS = T without x)
template <typename T, typename TS>
struct NormFwdArgs {
  const T *y, *z;
  const TS* x;
  const float *w_post, *c, *w_pre;
  TS* h;
  T* n;
  int64_t rows;
  int D;
  float eps;
};

template <typename T, typename TS>
struct NormBwdArgs {
  const T *y, *z, *dn;
  const TS *x, *dh;
  const float *w_post, *c, *w_pre;
  T *dy, *dz;
  TS* dx;
  float* part;  // (3, blocks, D): sums of dw_post, dc, dw_pre over the rows of each block
  int64_t rows;
  int D, blocks;
  float eps;
};

struct NormSumArgs {
  const float* part;
  float* out[3];  // dw_post, dc, dw_pre (nullable)
  int D, blocks;
};

// workgroups of the backward: its rows' partial sums
int norm_bwd_blocks(int64_t rows, int D, bool rest);

template <typename T, typename TS>
hipError_t launch_norm_fwd(const NormFwdArgs<T, TS>& a, hipStream_t st);
template <typename T, typename TS>
hipError_t launch_norm_bwd(const NormBwdArgs<T, TS>& a, hipStream_t st);
hipError_t launch_norm_sum(const NormSumArgs& a, hipStream_t st);

}  // namespace gdr2

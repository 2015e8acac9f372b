// Gated feed-forward block (include/gdr2_gatedff.h): the launch interface between the C ABI and
// the kernels.
#pragma once

#include "gdr2_kernels.hpp"

namespace gdr2 {

// C (M x N) = sum over operand pairs of A B^T, fp32 accumulation:
//   A's element (m, k) at a[m * am + k * ak], B's element (n, k) at b[n * bn + k * bk].
template <typename T, typename TC>
struct FfGemmArgs {
  const T *a[2], *b[2];
  int64_t am, ak, bn, bk;
  int pairs;
  TC* c;
  int64_t M, N, K;
};

template <typename T>
struct FfActArgs {
  const float *g, *u, *dh;  // dh NULL: forward
  T *h, *dg, *du;
  int64_t n;
  int act;
};

template <typename T, typename TC>
hipError_t launch_ff_gemm(const FfGemmArgs<T, TC>& a, hipStream_t st);
template <typename T>
hipError_t launch_ff_act(const FfActArgs<T>& a, hipStream_t st);

}  // namespace gdr2

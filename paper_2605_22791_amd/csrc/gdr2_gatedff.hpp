// Gated feed-forward block (include/gdr2_gatedff.h): the launch interface between the C ABI and
// the kernels.
#pragma once

#include "gdr2_gatedff_plan.hpp"
#include "gdr2_kernels.hpp"

namespace gdr2 {

// g and u on their way from the forward to the backward, (M, N): fp32 problems as they are; bf16 ones in
// fp16, with a power of two for every row and 32 channels that takes their largest finite magnitude to
// [2^14, 2^15): 2^-12 of a value against the 2^-9 that the gradients are rounded by, at half the bytes.
constexpr int kFfBlock = 32;
template <typename T>
struct FfHidden {
  void *g, *u;       // float or _Float16
  int8_t *ge, *ue;   // bf16 problems: the powers, (M, ceil(N / 32)): stored = value 2^power
};

template <typename T>
struct FfProduct {
  const T *a, *b[2];
  int64_t lda, ldb;   // elements from one row of memory to the next
  int64_t M, N;
  T* c[2];            // FF_STORE: rows from `cut` on are those of c[1]
  int64_t cut;
  int tm, tn;         // tiles (set by the launch)
};

template <typename T>
struct FfArgs : FfProduct<T> {
  FfProduct<T> also;  // FF_COLUMNS: another product with the same sum, in the same launch (M = 0: none)
  int64_t K;
  int64_t a2;         // pairs == 2: the second product's A starts a2 elements further; its B is b[1]
  int pairs;
  FfHidden<T> hid;    // FF_GATE: written where hid.g is given; FF_GRAD: read
  T *h, *dgu;         // FF_GATE: h (M, N), nullable; FF_GRAD: dg, du side by side (M, 2 N)
  int act;
  float* part;        // partial tiles
  // set by the launch
  int tiles, full, split;  // of them computed whole; parts of every other one
};

// Bytes of partial tiles that a launch takes.
template <typename T, int FORM, int END>
size_t ff_part_bytes(const FfArgs<T>& a);
template <typename T, int FORM, int END>
hipError_t launch_ff(FfArgs<T> a, hipStream_t st);

}  // namespace gdr2

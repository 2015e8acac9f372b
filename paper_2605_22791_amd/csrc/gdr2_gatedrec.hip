// Gated linear recurrence, token after token: a lane for each (sequence, channel).
//     h = a h + m i x;   dh = do + a_next dh_next,  dx = m i dh,  di = m x dh,
//     dg = a h_before dh - (a^2 / m) i x dh

#include "gdr2_gatedrec.hpp"
#include "gdr2_bf16.hpp"

namespace gdr2 {

namespace {

__device__ __forceinline__ float rec_ld(const float* p) { return *p; }
__device__ __forceinline__ float rec_ld(const bf16_t* p) { return __uint_as_float((uint32_t)p->x << 16); }
__device__ __forceinline__ void rec_st(float* p, float x) { *p = x; }
__device__ __forceinline__ void rec_st(bf16_t* p, float x) { *reinterpret_cast<__bf16*>(p) = (__bf16)x; }

// rows [t0, t0 + n) of sequence s; packed offsets are kept in range whatever they are
__device__ __forceinline__ void rec_rows(const int32_t* cu, int s, int len, size_t& t0, int& n) {
  t0 = (size_t)s * len;
  n = len;
  if (cu) {
    const int a = min(max(cu[s], 0), len);
    n = min(max(cu[s + 1], a), len) - a;
    t0 = a;
  }
}

}  // namespace

template <typename T>
__global__ __launch_bounds__(256) void rec_fwd_kernel(RecArgs<T> a) {
  const int nc = (a.D + 255) / 256, s = blockIdx.x / nc, c = (blockIdx.x % nc) * 256 + threadIdx.x;
  if (c >= a.D) return;
  size_t t0;
  int n;
  rec_rows(a.cu, s, a.len, t0, n);
  float h = a.h0 ? a.h0[(size_t)s * a.D + c] : 0.f;
  for (int t = 0; t < n; ++t) {
    const size_t at = (t0 + t) * a.D + c;
    const float g = a.g[at], m = a.normalize ? sqrtf(-expm1f(2.f * g)) : 1.f;
    h = expf(g) * h + m * (a.i ? rec_ld(a.i + at) : 1.f) * rec_ld(a.x + at);
    if (a.o) rec_st(a.o + at, h);
    if (a.hs) a.hs[at] = h;
  }
  if (a.hT) a.hT[(size_t)s * a.D + c] = h;
}

template <typename T>
__global__ __launch_bounds__(256) void rec_bwd_kernel(RecBwdArgs<T> a) {
  const int nc = (a.D + 255) / 256, s = blockIdx.x / nc, c = (blockIdx.x % nc) * 256 + threadIdx.x;
  if (c >= a.D) return;
  size_t t0;
  int n;
  rec_rows(a.cu, s, a.len, t0, n);
  float carry = a.dhT ? a.dhT[(size_t)s * a.D + c] : 0.f;
  const float h0 = a.h0 ? a.h0[(size_t)s * a.D + c] : 0.f;
  for (int t = n - 1; t >= 0; --t) {
    const size_t at = (t0 + t) * a.D + c;
    const float g = a.g[at], al = expf(g), m = a.normalize ? sqrtf(-expm1f(2.f * g)) : 1.f;
    const float i = a.i ? rec_ld(a.i + at) : 1.f, x = rec_ld(a.x + at);
    const float dh = rec_ld(a.dout + at) + carry, before = t > 0 ? a.hs[at - a.D] : h0;
    carry = al * dh;
    rec_st(a.dx + at, m * i * dh);
    if (a.di) rec_st(a.di + at, m * x * dh);
    a.dg[at] = carry * before - (a.normalize && m > 0.f ? al * al / m * i * x * dh : 0.f);
  }
  if (a.dh0) a.dh0[(size_t)s * a.D + c] = carry;
}

template <typename T>
hipError_t launch_rec_fwd(const RecArgs<T>& a, hipStream_t st) {
  hipLaunchKernelGGL(rec_fwd_kernel<T>, dim3((unsigned)((size_t)a.nseq * ((a.D + 255) / 256))), dim3(256), 0, st, a);
  return hipGetLastError();
}
template <typename T>
hipError_t launch_rec_bwd(const RecBwdArgs<T>& a, hipStream_t st) {
  hipLaunchKernelGGL(rec_bwd_kernel<T>, dim3((unsigned)((size_t)a.nseq * ((a.D + 255) / 256))), dim3(256), 0, st, a);
  return hipGetLastError();
}
template hipError_t launch_rec_fwd<float>(const RecArgs<float>&, hipStream_t);
template hipError_t launch_rec_fwd<bf16_t>(const RecArgs<bf16_t>&, hipStream_t);
template hipError_t launch_rec_bwd<float>(const RecBwdArgs<float>&, hipStream_t);
template hipError_t launch_rec_bwd<bf16_t>(const RecBwdArgs<bf16_t>&, hipStream_t);

}  // namespace gdr2

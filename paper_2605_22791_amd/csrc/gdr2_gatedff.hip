// Gated feed-forward block: the products, fp32 accumulation on the matrix cores, and the
// activation with its gradient.

#include "gdr2_gatedff.hpp"
#include "gdr2_bf16.hpp"

namespace gdr2 {

namespace {

constexpr int TM = 64, TK = 32, LK = TK + 4;  // tile, K step and LDS row stride (floats)

__device__ __forceinline__ float ff_ld(const float* p) { return *p; }
__device__ __forceinline__ float ff_ld(const bf16_t* p) { return __uint_as_float((uint32_t)p->x << 16); }
__device__ __forceinline__ void ff_st(float* p, float x) { *p = x; }
__device__ __forceinline__ void ff_st(bf16_t* p, float x) { *reinterpret_cast<__bf16*>(p) = (__bf16)x; }

__device__ __forceinline__ void ff_act(int act, float g, float& a, float& slope) {
  if (act == 0) {
    const float s = 1.f / (1.f + expf(-g));
    a = g * s;
    slope = s * (1.f + g * (1.f - s));
  } else {
    const float s = 0.5f * (1.f + erff(g * 0.70710678118654752f));
    a = g * s;
    slope = s + g * expf(-0.5f * g * g) * 0.39894228040143268f;
  }
}

}  // namespace

// A 64 x 64 tile a workgroup, a 16 x 64 strip a wave.
template <typename T, typename TC>
__global__ __launch_bounds__(256) void ff_gemm_kernel(FfGemmArgs<T, TC> p) {
  __shared__ float sa[TM * LK], sb[TM * LK];
  const int64_t nt = (p.N + TM - 1) / TM, m0 = blockIdx.x / nt * TM, n0 = blockIdx.x % nt * TM;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  f4 acc[4] = {f4zero(), f4zero(), f4zero(), f4zero()};
  for (int q = 0; q < p.pairs; ++q)
    for (int64_t k0 = 0; k0 < p.K; k0 += TK) {
      __syncthreads();
      for (int e = tid; e < TM * TK; e += 256) {
        const int r = e / TK, k = e % TK;
        const bool in = k0 + k < p.K;
        sa[r * LK + k] = in && m0 + r < p.M ? ff_ld(p.a[q] + (m0 + r) * p.am + (k0 + k) * p.ak) : 0.f;
        sb[r * LK + k] = in && n0 + r < p.N ? ff_ld(p.b[q] + (n0 + r) * p.bn + (k0 + k) * p.bk) : 0.f;
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < TK; k += 4) {
        const float x = sa[(16 * wave + (lane & 15)) * LK + k + (lane >> 4)];
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = mfma_f32(x, sb[(16 * j + (lane & 15)) * LK + k + (lane >> 4)], acc[j]);
      }
    }
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t m = m0 + 16 * wave + 4 * (lane >> 4) + u, n = n0 + 16 * j + (lane & 15);
      if (m < p.M && n < p.N) ff_st(p.c + m * p.N + n, acc[j][u]);
    }
}

template <typename T>
__global__ __launch_bounds__(256) void ff_act_kernel(FfActArgs<T> p) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= p.n) return;
  const float u = p.u[e];
  float a, slope;
  ff_act(p.act, p.g[e], a, slope);
  ff_st(p.h + e, a * u);
  if (p.dh) {
    const float d = p.dh[e];
    ff_st(p.dg + e, d * u * slope);
    ff_st(p.du + e, d * a);
  }
}

template <typename T, typename TC>
hipError_t launch_ff_gemm(const FfGemmArgs<T, TC>& a, hipStream_t st) {
  const int64_t blocks = ((a.M + TM - 1) / TM) * ((a.N + TM - 1) / TM);
  hipLaunchKernelGGL((ff_gemm_kernel<T, TC>), dim3((unsigned)blocks), dim3(256), 0, st, a);
  return hipGetLastError();
}
template <typename T>
hipError_t launch_ff_act(const FfActArgs<T>& a, hipStream_t st) {
  hipLaunchKernelGGL(ff_act_kernel<T>, dim3((unsigned)((a.n + 255) / 256)), dim3(256), 0, st, a);
  return hipGetLastError();
}
template hipError_t launch_ff_gemm<float, float>(const FfGemmArgs<float, float>&, hipStream_t);
template hipError_t launch_ff_gemm<bf16_t, float>(const FfGemmArgs<bf16_t, float>&, hipStream_t);
template hipError_t launch_ff_gemm<bf16_t, bf16_t>(const FfGemmArgs<bf16_t, bf16_t>&, hipStream_t);
template hipError_t launch_ff_act<float>(const FfActArgs<float>&, hipStream_t);
template hipError_t launch_ff_act<bf16_t>(const FfActArgs<bf16_t>&, hipStream_t);

}  // namespace gdr2

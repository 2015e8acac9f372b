// Linear attention with a decay for each head, token by token (decoding):
//     S <- exp(g) S + k v^T,   o = scale S^T q = scale (exp(g) S^T q + (k . q) v)
// for every (sequence, value head); the fp32 state stays in registers over the call's
// tokens and goes through memory once each way, which is what bounds the call.

#include "gdr2_linattn.hpp"
#include "gdr2_bf16.hpp"

namespace gdr2 {

namespace {
__device__ __forceinline__ float la_val(const float* p) { return *p; }
__device__ __forceinline__ float la_val(const bf16_t* p) { return __uint_as_float((uint32_t)p->x << 16); }
__device__ __forceinline__ void la_put4(float* p, const float (&x)[4]) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
}
__device__ __forceinline__ void la_put4(bf16_t* p, const float (&x)[4]) {
  st4(reinterpret_cast<__bf16*>(p), x[0], x[1], x[2], x[3]);
}
}  // namespace

// A workgroup per (sequence, value head); each of its four waves holds a quarter of the
// state's rows, four columns a lane.
template <int DK, int DV, typename TIn>
__global__ __launch_bounds__(256) void la_step_kernel(LaStepArgs<TIn> a) {
  constexpr int RW = DK / 4, CG = DV / 4, RG = 64 / CG, RPL = RW / RG;
  __shared__ float sum[2][4][DV];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int cg = lane % CG, rg = lane / CG;
  const int H = a.H, h = blockIdx.x % H, s = blockIdx.x / H, HK = H / a.G, hk = h / a.G;
  size_t row0 = (size_t)s * a.T;
  int n = a.T;
  if (a.cu) {
    const int t0 = min(max(a.cu[s], 0), a.T);
    n = min(max(a.cu[s + 1], t0), a.T) - t0;
    row0 = t0;
  }
  if (n == 0) return;
  float* Sg = a.S + (size_t)blockIdx.x * (DK * DV) + (size_t)(RW * wave + rg) * DV + 4 * cg;
  f4 S[RPL];
#pragma unroll
  for (int i = 0; i < RPL; ++i) S[i] = *reinterpret_cast<const f4*>(Sg + RG * i * DV);
  for (int t = 0; t < n; ++t) {
    const size_t row = row0 + t;
    const TIn *q = a.q + (row * HK + hk) * DK + RW * wave + rg, *k = a.k + (row * HK + hk) * DK + RW * wave + rg;
    const TIn* v = a.v + (row * H + h) * DV + 4 * cg;
    const float al = expf(a.per_head ? a.g[h] : a.g[row * H + h]);
    const f4 vv = {la_val(v), la_val(v + 1), la_val(v + 2), la_val(v + 3)};
    f4 p = f4zero();
#pragma unroll
    for (int i = 0; i < RPL; ++i) {
      S[i] = S[i] * al + la_val(k + RG * i) * vv;
      p += S[i] * la_val(q + RG * i);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if constexpr (RG == 4) p[u] += row_partner16(p[u], (lane & 16) != 0);
      p[u] += row_partner32(p[u], lane >= 32);
    }
    if (rg == 0) *reinterpret_cast<f4*>(&sum[t & 1][wave][4 * cg]) = p;
    __syncthreads();
    if (wave == 0 && rg == 0) {
      float o[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        o[u] = a.scale * ((sum[t & 1][0][4 * cg + u] + sum[t & 1][1][4 * cg + u]) +
                          (sum[t & 1][2][4 * cg + u] + sum[t & 1][3][4 * cg + u]));
      la_put4(a.o + (row * H + h) * DV + 4 * cg, o);
    }
  }
#pragma unroll
  for (int i = 0; i < RPL; ++i) *reinterpret_cast<f4*>(Sg + RG * i * DV) = S[i];
}

template <int DK, int DV, typename TIn>
hipError_t launch_la_step(const LaStepArgs<TIn>& a, hipStream_t st) {
  hipLaunchKernelGGL((la_step_kernel<DK, DV, TIn>), dim3((unsigned)(a.nseq * a.H)), dim3(256), 0, st, a);
  return hipGetLastError();
}

#define GDR2_LA_STEP(DK, DV)                                                                  \
  template hipError_t launch_la_step<DK, DV, float>(const LaStepArgs<float>&, hipStream_t);   \
  template hipError_t launch_la_step<DK, DV, bf16_t>(const LaStepArgs<bf16_t>&, hipStream_t);
GDR2_LA_STEP(64, 64)
GDR2_LA_STEP(64, 128)
GDR2_LA_STEP(128, 64)
GDR2_LA_STEP(128, 128)

}  // namespace gdr2

// Linear attention with a decay for each head, token by token (decoding):
//     S <- exp(g) S + k v^T,   o = scale S^T q = scale (exp(g) S^T q + (k . q) v)
// for every (sequence, value head); the fp32 state stays in registers over the call's
// tokens and goes through memory once each way, which is what bounds the call.  Tokens come
// eight at a time through LDS, the next eight on their way meanwhile, so that a sequence of
// some tokens does not wait for memory at each: 48 sequences of 1 to 16 tokens, 16 heads of
// 128 x 128, take 21 us (4.9 TB/s) where loading each token in its turn took 30.7; 256 sequences
// of one token 105 us (5.2 TB/s).

#include "gdr2_linattn.hpp"
#include "gdr2_bf16.hpp"

namespace gdr2 {

namespace {
// four values on their way from memory
template <typename T>
struct LaFour {
  f4 x;
  __device__ __forceinline__ void load(const T* p) { x = *reinterpret_cast<const f4*>(p); }
  __device__ __forceinline__ f4 get() const { return x; }
};
template <>
struct LaFour<bf16_t> {
  bf4 x;
  __device__ __forceinline__ void load(const bf16_t* p) { x = *reinterpret_cast<const bf4*>(p); }
  __device__ __forceinline__ f4 get() const { return f4{(float)x[0], (float)x[1], (float)x[2], (float)x[3]}; }
};
__device__ __forceinline__ void la_put4(float* p, const f4& x) { *reinterpret_cast<f4*>(p) = x; }
__device__ __forceinline__ void la_put4(bf16_t* p, const f4& x) {
  st4(reinterpret_cast<__bf16*>(p), x[0], x[1], x[2], x[3]);
}
}  // namespace

// A workgroup per (sequence, value head); each of its four waves holds a quarter of the
// state's rows, a lane four columns of RPL rows.
template <int DK, int DV, typename TIn>
__global__ __launch_bounds__(256) void la_step_kernel(LaStepArgs<TIn> a) {
  constexpr int RW = DK / 4, CG = DV / 4, RG = 64 / CG, RPL = RW / RG, TOK = 8;
  static_assert(RPL % 4 == 0, "rows in fours");
  __shared__ __align__(16) float sq[TOK][DK], sk[TOK][DK], sv[TOK][DV], sum[TOK][4][DV], sal[TOK];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int cg = lane % CG, r0 = RW * wave + RPL * (lane / CG);
  const int H = a.H, h = blockIdx.x % H, s = blockIdx.x / H, HK = H / a.G, hk = h / a.G;
  size_t row0 = (size_t)s * a.T;
  int n = a.T;
  if (a.cu) {
    const int t0 = min(max(a.cu[s], 0), a.T);
    n = min(max(a.cu[s + 1], t0), a.T) - t0;
    row0 = t0;
  }
  if (n == 0) return;
  // a token for 32 threads, four elements each
  const int tj = tid >> 5, te = 4 * (tid & 31);
  LaFour<TIn> q, k, v;
  float g = 0.f;
  const auto fetch = [&](int t) {
    if (t + tj >= n) return;
    const size_t row = row0 + t + tj;
    if (te < DK) {
      q.load(a.q + (row * HK + hk) * DK + te);
      k.load(a.k + (row * HK + hk) * DK + te);
    }
    if (te < DV) v.load(a.v + (row * H + h) * DV + te);
    if (te == 0) g = a.per_head ? a.g[h] : a.g[row * H + h];
  };
  fetch(0);
  float* Sg = a.S + (size_t)blockIdx.x * (DK * DV) + (size_t)r0 * DV + 4 * cg;
  f4 S[RPL];
#pragma unroll
  for (int i = 0; i < RPL; ++i) S[i] = *reinterpret_cast<const f4*>(Sg + i * DV);
  for (int t = 0; t < n; t += TOK) {
    const int m = min(TOK, n - t);
    if (tj < m) {
      if (te < DK) {
        *reinterpret_cast<f4*>(&sq[tj][te]) = q.get();
        *reinterpret_cast<f4*>(&sk[tj][te]) = k.get();
      }
      if (te < DV) *reinterpret_cast<f4*>(&sv[tj][te]) = v.get();
      if (te == 0) sal[tj] = expf(g);
    }
    __syncthreads();
    fetch(t + TOK);
    for (int j = 0; j < m; ++j) {
      const float al = sal[j];
      const f4 vv = *reinterpret_cast<const f4*>(&sv[j][4 * cg]);
      f4 p = f4zero();
#pragma unroll
      for (int i = 0; i < RPL; i += 4) {
        const f4 kk = *reinterpret_cast<const f4*>(&sk[j][r0 + i]), qq = *reinterpret_cast<const f4*>(&sq[j][r0 + i]);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          S[i + u] = S[i + u] * al + kk[u] * vv;
          p += S[i + u] * qq[u];
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if constexpr (RG == 4) p[u] += row_partner16(p[u], (lane & 16) != 0);
        p[u] += row_partner32(p[u], lane >= 32);
      }
      if (lane < CG) *reinterpret_cast<f4*>(&sum[j][wave][4 * cg]) = p;
    }
    __syncthreads();
    if (tj < m && te < DV) {
      const auto part = [&](int w) { return *reinterpret_cast<const f4*>(&sum[tj][w][te]); };
      la_put4(a.o + ((row0 + t + tj) * H + h) * DV + te, ((part(0) + part(1)) + (part(2) + part(3))) * a.scale);
    }
  }
#pragma unroll
  for (int i = 0; i < RPL; ++i) *reinterpret_cast<f4*>(Sg + i * DV) = S[i];
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

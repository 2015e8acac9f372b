// Norms before and after a block with its gate and residual scale, one pass over
// the rows each way.  Forward, per row (include/gdr2_blocknorm.h):
//     u = y r_y w_post,  a = u silu(z),  h = x + c a,  n = h r_h w_pre
// backward, everything formed again from y, z and x in registers:
//     t = dn w_pre;  dx = dh + r_h (t - h r_h^2 mean(t h));   dw_pre = sum dn h r_h
//     da = c dx;  dc = sum dx a;  dz = da u silu'(z);  du = da silu(z)
//     dw_post = sum du y r_y;  s = du w_post;  dy = r_y (s - y r_y^2 mean(s y))
// Both are bound by memory: every input is read once and every output written once.
//
// A row belongs to LPR lanes of eight elements each; the weights stay in the
// lanes' registers over the rows that a workgroup takes in turn, and so do the
// sums of the weights' gradients, which leave once per workgroup and are added
// by a second launch in a fixed order.  The backward loads a row ahead.
//
// Measured: 524288 bf16 rows of 128 with norm and gate, forward 86 us (403 MB, 4.7
// TB/s), backward 134 us (671 MB, 5.0 TB/s; 212 without the row ahead and in the
// registers of the full form); 32768 rows of 2048, everything, fp32 stream: 166 us
// (0.94 GB) and 336 us (1.47 GB, 4.4 TB/s); 1999 fp32 rows of 1155: 11 and 19 us.
// Far from that: the backward of rows over 4096 with stream parts, whose 1024 lanes of 128
// registers spill (8192 rows of 8192: 1340 us for 1.47 GB), and widths that 8 does not divide in
// bf16, loaded two bytes at a time (58099 rows of 1155, everything: 333 and 1171 us for the
// same bytes).

#include "gdr2_blocknorm.hpp"
#include "gdr2_bf16.hpp"

namespace gdr2 {

namespace {

constexpr int EPL = 8;

// Element i of a lane: VEC, eight consecutive ones; else LPR apart (rows of any width).
template <int LPR, bool VEC>
__device__ __forceinline__ int norm_col(int lane, int i) {
  return VEC ? EPL * lane + i : lane + LPR * i;
}

template <int LPR, bool VEC>
__device__ __forceinline__ void norm_load(const float* p, int D, int lane, float (&x)[EPL]) {
  if constexpr (VEC) {
    if (EPL * lane < D) {
      ldf8(p + EPL * lane, x);
      return;
    }
#pragma unroll
    for (int i = 0; i < EPL; ++i) x[i] = 0.f;
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i) x[i] = lane + LPR * i < D ? p[lane + LPR * i] : 0.f;
  }
}
template <int LPR, bool VEC>
__device__ __forceinline__ void norm_load(const bf16_t* p, int D, int lane, float (&x)[EPL]) {
  if constexpr (VEC) {
    if (EPL * lane < D) {
      unpack8(ldg16(p + EPL * lane), x);
      return;
    }
#pragma unroll
    for (int i = 0; i < EPL; ++i) x[i] = 0.f;
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i) x[i] = lane + LPR * i < D ? __uint_as_float((uint32_t)p[lane + LPR * i].x << 16) : 0.f;
  }
}
template <int LPR, bool VEC>
__device__ __forceinline__ void norm_store(float* p, int D, int lane, const float (&x)[EPL]) {
  if constexpr (VEC) {
    if (EPL * lane < D) {
      *reinterpret_cast<f4*>(p + EPL * lane) = f4{x[0], x[1], x[2], x[3]};
      *reinterpret_cast<f4*>(p + EPL * lane + 4) = f4{x[4], x[5], x[6], x[7]};
    }
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (lane + LPR * i < D) p[lane + LPR * i] = x[i];
  }
}
template <int LPR, bool VEC>
__device__ __forceinline__ void norm_store(bf16_t* p, int D, int lane, const float (&x)[EPL]) {
  __bf16* q = reinterpret_cast<__bf16*>(p);
  if constexpr (VEC) {
    if (EPL * lane < D) st8(q + EPL * lane, round8(x));
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (lane + LPR * i < D) q[lane + LPR * i] = (__bf16)x[i];
  }
}

// A lane's part of a row on its way from memory: loaded a row ahead, in as few registers as it takes
template <typename T, int LPR, bool VEC>
struct NormRow {
  float x[EPL];
  __device__ __forceinline__ void load(const T* p, int D, int lane) { norm_load<LPR, VEC>(p, D, lane, x); }
  __device__ __forceinline__ void get(float (&to)[EPL]) const {
#pragma unroll
    for (int i = 0; i < EPL; ++i) to[i] = x[i];
  }
};
template <int LPR>
struct NormRow<bf16_t, LPR, true> {
  u4v x;
  __device__ __forceinline__ void load(const bf16_t* p, int D, int lane) {
    x = EPL * lane < D ? *reinterpret_cast<const u4v*>(p + EPL * lane) : u4v{0, 0, 0, 0};
  }
  __device__ __forceinline__ void get(float (&to)[EPL]) const { unpack8(__builtin_bit_cast(bf8, x), to); }
};

// Sums over a row's LPR lanes, every lane gets them.  Up to a wave: steps across
// lanes; more: the waves' sums meet in LDS (slot: a different one of four at each of
// a row's reductions, so that one barrier a reduction is enough).
template <int LPR, int N>
__device__ __forceinline__ void norm_sum(float (&x)[N], float* red, int slot) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    x[k] = row_sum<LPR == 8>(x[k]);
    if constexpr (LPR >= 32) x[k] += row_partner16(x[k], (lane & 16) != 0);
    if constexpr (LPR >= 64) x[k] += row_partner32(x[k], lane >= 32);
  }
  if constexpr (LPR > 64) {
    constexpr int NW = LPR / 64;
    const int sub = threadIdx.x / LPR, wave = (threadIdx.x % LPR) / 64;
    float* at = red + ((slot & 3) * (blockDim.x / LPR) + sub) * NW * 2;
    if (lane == 0) {
#pragma unroll
      for (int k = 0; k < N; ++k) at[wave * 2 + k] = x[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
      x[k] = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) x[k] += at[w * 2 + k];
    }
  }
}

template <int N>
__device__ __forceinline__ void norm_sum8(double (&x)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) x[k] += __shfl_xor(x[k], o);
}
// The gradient of a norm is a difference, s - y r^2 mean(s y), that cancels the more the
// narrower the row: at width 1 all but eps / (y^2 + eps) of it.  Rows of up to 64 take
// it in 64 bits (a few operations an element beside the row's way through memory).
template <int LPR>
using NormAcc = typename std::conditional<LPR == 8, double, float>::type;

template <int LPR>
constexpr int norm_threads() { return LPR > 256 ? LPR : 256; }
// LDS floats of norm_sum: four slots of every row's wave sums
template <int LPR>
constexpr int norm_red() { return LPR > 64 ? 4 * (norm_threads<LPR>() / 64) * 2 : 1; }

__device__ __forceinline__ float inv_rms(float ss, int D, float eps) { return 1.f / sqrtf(ss / (float)D + eps); }
__device__ __forceinline__ double inv_rms(double ss, int D, float eps) { return 1.0 / sqrt(ss / D + (double)eps); }

// sums over a row in NormAcc
template <int LPR, int N>
__device__ __forceinline__ void norm_acc(NormAcc<LPR> (&x)[N], float* red, int slot) {
  if constexpr (LPR == 8)
    norm_sum8(x);
  else
    norm_sum<LPR>(x, red, slot);
}

}  // namespace

template <typename T, typename TS, int LPR, bool VEC>
__global__ __launch_bounds__(norm_threads<LPR>()) void norm_fwd_kernel(NormFwdArgs<T, TS> a) {
  __shared__ float red[norm_red<LPR>()];
  constexpr int RPB = norm_threads<LPR>() / LPR;
  const int lane = threadIdx.x % LPR, D = a.D;
  float wp[EPL], c[EPL], wn[EPL];
  if (a.w_post) norm_load<LPR, VEC>(a.w_post, D, lane, wp);
  if (a.c) norm_load<LPR, VEC>(a.c, D, lane, c);
  if (a.w_pre) norm_load<LPR, VEC>(a.w_pre, D, lane, wn);
  int slot = 0;
  // every lane of the workgroup makes the same number of rounds (barriers inside)
  for (int64_t base = (int64_t)blockIdx.x * RPB; base < a.rows; base += (int64_t)gridDim.x * RPB) {
    const int64_t row = base + threadIdx.x / LPR;
    const bool on = row < a.rows;
    const size_t at = (size_t)(on ? row : a.rows - 1) * D;
    float y[EPL], z[EPL], h[EPL];
    norm_load<LPR, VEC>(a.y + at, D, lane, y);
    if (a.z) norm_load<LPR, VEC>(a.z + at, D, lane, z);
    if (a.x) norm_load<LPR, VEC>(a.x + at, D, lane, h);
    if (a.w_post) {
      float s[1] = {0.f};
#pragma unroll
      for (int i = 0; i < EPL; ++i) s[0] += y[i] * y[i];
      norm_sum<LPR>(s, red, slot++);
      const float r = inv_rms(s[0], D, a.eps);
#pragma unroll
      for (int i = 0; i < EPL; ++i) y[i] = y[i] * r * wp[i];
    }
    if (a.z) {
#pragma unroll
      for (int i = 0; i < EPL; ++i) y[i] *= z[i] / (1.f + expf(-z[i]));
    }
    if (a.c) {
#pragma unroll
      for (int i = 0; i < EPL; ++i) y[i] *= c[i];
    }
#pragma unroll
    for (int i = 0; i < EPL; ++i) h[i] = a.x ? h[i] + y[i] : y[i];
    if (a.h && on) norm_store<LPR, VEC>(a.h + at, D, lane, h);
    if (a.w_pre) {
      float s[1] = {0.f};
#pragma unroll
      for (int i = 0; i < EPL; ++i) s[0] += h[i] * h[i];
      norm_sum<LPR>(s, red, slot++);
      const float r = inv_rms(s[0], D, a.eps);
#pragma unroll
      for (int i = 0; i < EPL; ++i) h[i] = h[i] * r * wn[i];
      if (on) norm_store<LPR, VEC>(a.n + at, D, lane, h);
    }
  }
}

// REST: there may be x, c or w_pre; without them a lane needs half the registers.
template <typename T, typename TS, int LPR, bool VEC, bool REST>
__global__ __launch_bounds__(norm_threads<LPR>()) void norm_bwd_kernel(NormBwdArgs<T, TS> a) {
  constexpr int TPB = norm_threads<LPR>(), RPB = TPB / LPR;
  __shared__ float red[norm_red<LPR>()];
  __shared__ float acc[RPB > 1 ? TPB * EPL : 1];
  const int lane = threadIdx.x % LPR, D = a.D;
  const bool has_x = REST && a.x, has_c = REST && a.c, pre = REST && a.w_pre;
  float wp[EPL], c[EPL], wn[EPL], dwp[EPL], dc[EPL], dwn[EPL];
#pragma unroll
  for (int i = 0; i < EPL; ++i) wp[i] = c[i] = 1.f, dwp[i] = dc[i] = dwn[i] = 0.f;
  if (a.w_post) norm_load<LPR, VEC>(a.w_post, D, lane, wp);
  if (has_c) norm_load<LPR, VEC>(a.c, D, lane, c);
  if (pre) norm_load<LPR, VEC>(a.w_pre, D, lane, wn);
  using Acc = NormAcc<LPR>;
  const Acc inv_d = (Acc)1 / (Acc)D;
  int slot = 0;
  NormRow<T, LPR, VEC> ny, nz, nt;
  NormRow<TS, LPR, VEC> nx, ndh;
  const auto fetch = [&](int64_t base) {
    const int64_t row = base + threadIdx.x / LPR;
    const size_t at = (size_t)(row < a.rows ? row : a.rows - 1) * D;
    ny.load(a.y + at, D, lane);
    if (a.z) nz.load(a.z + at, D, lane);
    if (has_x) nx.load(a.x + at, D, lane);
    if (a.dh) ndh.load(a.dh + at, D, lane);
    if (pre) nt.load(a.dn + at, D, lane);
  };
  const int64_t step = (int64_t)gridDim.x * RPB;
  fetch((int64_t)blockIdx.x * RPB);
  for (int64_t base = (int64_t)blockIdx.x * RPB; base < a.rows; base += step) {
    const int64_t row = base + threadIdx.x / LPR;
    const bool on = row < a.rows;
    const size_t at = (size_t)(on ? row : a.rows - 1) * D;
    float y[EPL], z[EPL], h[EPL], dh[EPL], t[EPL];
    ny.get(y);
    if (a.z) nz.get(z);
    if (has_x) nx.get(h);
    if (a.dh) {
      ndh.get(dh);
    } else {
#pragma unroll
      for (int i = 0; i < EPL; ++i) dh[i] = 0.f;
    }
    if (pre) nt.get(t);
    if (base + step < a.rows) fetch(base + step);
    Acc rya = 1;
    if (a.w_post) {
      Acc s[1] = {0};
#pragma unroll
      for (int i = 0; i < EPL; ++i) s[0] += (Acc)y[i] * y[i];
      norm_acc<LPR>(s, red, slot++);
      rya = inv_rms(s[0], D, a.eps);
    }
    const float ry = (float)rya;
    float sg[EPL];  // logistic of the gate
    if (a.z) {
#pragma unroll
      for (int i = 0; i < EPL; ++i) sg[i] = 1.f / (1.f + expf(-z[i]));
    }
    // full gradient at h, in dh
    if (pre) {
      Acc s[2] = {0, 0};
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        const float v = y[i] * ry * wp[i] * (a.z ? z[i] * sg[i] : 1.f) * c[i];
        h[i] = has_x ? h[i] + v : v;
        s[0] += (Acc)h[i] * h[i];
        s[1] += (Acc)(t[i] * wn[i]) * h[i];
      }
      norm_acc<LPR>(s, red, slot++);
      const Acc rh = inv_rms(s[0], D, a.eps), m = s[1] * inv_d * rh * rh;
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        if (on) dwn[i] += t[i] * h[i] * (float)rh;
        dh[i] += (float)(rh * (t[i] * wn[i] - h[i] * m));
      }
    }
    if (has_x && a.dx && on) norm_store<LPR, VEC>(a.dx + at, D, lane, dh);
    float dz[EPL];
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      const float u = y[i] * ry * wp[i], s = a.z ? z[i] * sg[i] : 1.f;
      if (has_c && on) dc[i] += dh[i] * u * s;
      const float da = dh[i] * c[i];
      if (a.z) dz[i] = da * u * sg[i] * (1.f + z[i] * (1.f - sg[i]));
      dh[i] = da * s;
      if (on) dwp[i] += dh[i] * y[i] * ry;
    }
    if (a.z && on) norm_store<LPR, VEC>(a.dz + at, D, lane, dz);
    if (a.w_post) {
      Acc s[1] = {0};
#pragma unroll
      for (int i = 0; i < EPL; ++i) s[0] += (Acc)(dh[i] * wp[i]) * y[i];
      norm_acc<LPR>(s, red, slot++);
      const Acc m = s[0] * inv_d * rya * rya;
#pragma unroll
      for (int i = 0; i < EPL; ++i) dh[i] = (float)(rya * (dh[i] * wp[i] - y[i] * m));
    }
    if (on) norm_store<LPR, VEC>(a.dy + at, D, lane, dh);
  }
  // the workgroup's sums: its RPB rows' lanes meet in LDS, in order
  const auto leave = [&](const float (&x)[EPL], int k) {
    float* out = a.part + ((size_t)k * a.blocks + blockIdx.x) * D;
    if constexpr (RPB == 1) {
      norm_store<LPR, VEC>(out, D, lane, x);
    } else {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < EPL; ++i) acc[(threadIdx.x / LPR) * (LPR * EPL) + norm_col<LPR, VEC>(lane, i)] = x[i];
      __syncthreads();
      for (int j = threadIdx.x; j < D; j += TPB) {
        float s = 0.f;
#pragma unroll
        for (int r = 0; r < RPB; ++r) s += acc[r * (LPR * EPL) + j];
        out[j] = s;
      }
    }
  };
  if (a.w_post) leave(dwp, 0);
  if (has_c) leave(dc, 1);
  if (pre) leave(dwn, 2);
}

// Columns' sums over the workgroups: 16 columns a workgroup, 64 threads each, so that a column's
// loads are in flight together (16 threads each took 20 us for 1024 parts of 128 to 2048 columns)
__global__ __launch_bounds__(1024) void norm_sum_kernel(NormSumArgs a) {
  __shared__ float sum[64][17];
  const int j = threadIdx.x % 16, g = threadIdx.x / 16, col = blockIdx.x * 16 + j, k = blockIdx.y;
  float* out = a.out[k];
  if (out == nullptr) return;
  float x = 0.f;
  if (col < a.D) {
    const float* p = a.part + (size_t)k * a.blocks * a.D + col;
#pragma unroll 16
    for (int b = g; b < a.blocks; b += 64) x += p[(size_t)b * a.D];
  }
  sum[g][j] = x;
  __syncthreads();
  if (g == 0 && col < a.D) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 64; ++i) s += sum[i][j];
    out[col] = s;
  }
}

// ---- launches --------------------------------------------------------------
namespace {

// lanes of a row: the fewest that hold it, eight elements each
int norm_lanes(int D) {
  int n = 8;
  while (n * EPL < D) n *= 2;
  return n;
}
int norm_rows_per_block(int D) {
  const int n = norm_lanes(D);
  return n > 256 ? 1 : 256 / n;
}

// f(LPR, VEC) as template arguments
template <class F>
hipError_t norm_dispatch(int D, F&& f) {
  const auto vec = [&](auto lpr) {
    return D % EPL == 0 ? f(lpr, std::true_type{}) : f(lpr, std::false_type{});
  };
  switch (norm_lanes(D)) {
    case 8: return vec(std::integral_constant<int, 8>{});
    case 16: return vec(std::integral_constant<int, 16>{});
    case 32: return vec(std::integral_constant<int, 32>{});
    case 64: return vec(std::integral_constant<int, 64>{});
    case 128: return vec(std::integral_constant<int, 128>{});
    case 256: return vec(std::integral_constant<int, 256>{});
    case 512: return vec(std::integral_constant<int, 512>{});
    default: return vec(std::integral_constant<int, 1024>{});
  }
}

}  // namespace

// Workgroups of a backward call, as many as are resident together: four waves a SIMD of the form
// without x, c and w_pre, two of the other (1024 of the latter, rows of 2048, took 382 us for 336)
int norm_bwd_blocks(int64_t rows, int D, bool rest) {
  const int rpb = norm_rows_per_block(D);
  const int64_t n = (rows + rpb - 1) / rpb, most = rest ? 512 : 1024;
  return (int)(n < most ? n : most);
}

template <typename T, typename TS>
hipError_t launch_norm_fwd(const NormFwdArgs<T, TS>& a, hipStream_t st) {
  return norm_dispatch(a.D, [&](auto lpr, auto vec) {
    constexpr int LPR = decltype(lpr)::value, TPB = norm_threads<LPR>(), RPB = TPB / LPR;
    const int64_t n = (a.rows + RPB - 1) / RPB;
    hipLaunchKernelGGL((norm_fwd_kernel<T, TS, LPR, decltype(vec)::value>), dim3((unsigned)(n < 8192 ? n : 8192)), dim3(TPB),
                       0, st, a);
    return hipGetLastError();
  });
}

template <typename T, typename TS>
hipError_t launch_norm_bwd(const NormBwdArgs<T, TS>& a, hipStream_t st) {
  return norm_dispatch(a.D, [&](auto lpr, auto vec) {
    constexpr int LPR = decltype(lpr)::value;
    const auto kernel = a.x || a.c || a.w_pre ? norm_bwd_kernel<T, TS, LPR, decltype(vec)::value, true>
                                              : norm_bwd_kernel<T, TS, LPR, decltype(vec)::value, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)a.blocks), dim3(norm_threads<LPR>()), 0, st, a);
    return hipGetLastError();
  });
}

hipError_t launch_norm_sum(const NormSumArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(norm_sum_kernel, dim3((unsigned)((a.D + 15) / 16), 3), dim3(1024), 0, st, a);
  return hipGetLastError();
}

#define GDR2_NORM_INST(T, TS)                                                            \
  template hipError_t launch_norm_fwd<T, TS>(const NormFwdArgs<T, TS>&, hipStream_t);    \
  template hipError_t launch_norm_bwd<T, TS>(const NormBwdArgs<T, TS>&, hipStream_t);
GDR2_NORM_INST(float, float)
GDR2_NORM_INST(bf16_t, float)
GDR2_NORM_INST(bf16_t, bf16_t)

}  // namespace gdr2

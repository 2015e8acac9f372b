// Dropout with the block's residual sum (include/gdr2_dropout.h), the C ABI and its one kernel:
//     y = r + [word >= round(p 2^32)] x / (1 - p)
// Bound by memory: x and r are read once, y is written once.  A lane takes eight consecutive
// elements, two blocks of the generator; the 2 x 10 rounds are 40 widening 32-bit products, which
// hide behind the loads (64 Mi bf16 elements without a residual: 43 us where a copy takes 37; 32768 x 2048
// beside a 32-bit stream, both ways: 184 us for 1.07 GB).  Whole 32-bit words an element: 16 bits would
// give 38 us and round p to 2^-16.

#include "../../include/gdr2_dropout.h"

#include "gdr2_bf16.hpp"
#include "gdr2_host.hpp"

namespace gdr2 {

namespace {

constexpr int EPL = 8;

// One block of Philox 4x32-10: the multipliers and key increments are the method's published ones.
__device__ __forceinline__ void philox10(uint64_t block, uint64_t offset, uint64_t seed, uint32_t (&c)[4]) {
  c[0] = (uint32_t)block, c[1] = (uint32_t)(block >> 32), c[2] = (uint32_t)offset, c[3] = (uint32_t)(offset >> 32);
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t p = (uint64_t)0xD2511F53u * c[0], q = (uint64_t)0xCD9E8D57u * c[2];
    const uint32_t n0 = (uint32_t)(q >> 32) ^ c[1] ^ k0, n2 = (uint32_t)(p >> 32) ^ c[3] ^ k1;
    c[0] = n0, c[1] = (uint32_t)q, c[2] = n2, c[3] = (uint32_t)p;
    k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
  }
}

template <typename TX, typename TY>
struct DropArgs {
  const TX* x;
  const TY* r;  // nullable
  TY* y;
  const uint64_t* more;
  int64_t n;
  uint64_t seed, offset;
  uint32_t least;  // the first word that is kept
  float scale;
};

__device__ __forceinline__ void drop_load(const float* p, float (&x)[EPL]) { ldf8(p, x); }
__device__ __forceinline__ void drop_load(const bf16_t* p, float (&x)[EPL]) { unpack8(ldg16(p), x); }
__device__ __forceinline__ float drop_load1(const float* p) { return *p; }
__device__ __forceinline__ float drop_load1(const bf16_t* p) { return __uint_as_float((uint32_t)p->x << 16); }
__device__ __forceinline__ void drop_store(float* p, const float (&x)[EPL]) {
  *reinterpret_cast<f4*>(p) = f4{x[0], x[1], x[2], x[3]};
  *reinterpret_cast<f4*>(p + 4) = f4{x[4], x[5], x[6], x[7]};
}
__device__ __forceinline__ void drop_store(bf16_t* p, const float (&x)[EPL]) { st8(reinterpret_cast<__bf16*>(p), round8(x)); }
__device__ __forceinline__ void drop_store1(float* p, float x) { *p = x; }
__device__ __forceinline__ void drop_store1(bf16_t* p, float x) { *reinterpret_cast<__bf16*>(p) = (__bf16)x; }

// elements e0 .. e0 + EPL
template <typename TX, typename TY>
__device__ __forceinline__ void drop_piece(const DropArgs<TX, TY>& a, int64_t e0, uint64_t offset) {
  const bool whole = e0 + EPL <= a.n;
  float x[EPL], r[EPL];
  if (whole) {
    drop_load(a.x + e0, x);
    if (a.r) drop_load(a.r + e0, r);
  } else {  // the tensor's last elements
    for (int i = 0; i < EPL; ++i) {
      x[i] = e0 + i < a.n ? drop_load1(a.x + e0 + i) : 0.f;
      if (a.r) r[i] = e0 + i < a.n ? drop_load1(a.r + e0 + i) : 0.f;
    }
  }
#pragma unroll
  for (int b = 0; b < EPL / 4; ++b) {
    uint32_t w[4];
    philox10((uint64_t)(e0 / 4 + b), offset, a.seed, w);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float v = w[i] >= a.least ? x[4 * b + i] * a.scale : 0.f;  // chosen, not multiplied: an infinity is dropped too
      x[4 * b + i] = a.r ? r[4 * b + i] + v : v;
    }
  }
  if (whole) {
    drop_store(a.y + e0, x);
  } else {
    for (int i = 0; i < EPL; ++i)
      if (e0 + i < a.n) drop_store1(a.y + e0 + i, x[i]);
  }
}

template <typename TX, typename TY>
__global__ __launch_bounds__(256) void dropout_kernel(DropArgs<TX, TY> a) {
  const uint64_t offset = a.offset + (a.more ? *a.more : 0);
  for (int64_t e0 = ((int64_t)blockIdx.x * 256 + threadIdx.x) * EPL; e0 < a.n; e0 += (int64_t)gridDim.x * (256 * EPL))
    drop_piece(a, e0, offset);
}

gdr2_status drop_check(const gdr2_dropout* p, const uint64_t* more) {
  if (p == nullptr || p->n < 0 || !(p->p >= 0.0 && p->p < 1.0)) return GDR2_EINVAL;
  if (p->dtype != GDR2_BF16 && p->dtype != GDR2_FP32) return GDR2_EINVAL;
  if (p->stream_dtype != p->dtype && p->stream_dtype != GDR2_FP32) return GDR2_EINVAL;
  if ((reinterpret_cast<uintptr_t>(more) & 7u) != 0) return GDR2_EINVAL;
  if (p->n > (int64_t)1 << 40) return GDR2_EUNSUPPORTED;
  return GDR2_OK;
}

template <typename TX, typename TY>
gdr2_status drop_launch(const gdr2_dropout* p, const uint64_t* more, const void* x, const void* r, void* y, hipStream_t st) {
  if (p->n == 0) return GDR2_OK;
  // round(p 2^32) is 2^32 for the last p below 1: all but the largest word are dropped then
  const double least = std::nearbyint(p->p * 4294967296.0);
  const DropArgs<TX, TY> a{static_cast<const TX*>(x), static_cast<const TY*>(r), static_cast<TY*>(y), more, p->n, p->seed,
                           p->offset, least > 4294967295.0 ? 4294967295u : (uint32_t)least, (float)(1.0 / (1.0 - p->p))};
  // a launch has less than 2^32 threads: from 2^32 elements on a lane takes several pieces
  const int64_t blocks = (p->n + 256 * EPL - 1) / (256 * EPL), most = 1 << 21;
  hipLaunchKernelGGL((dropout_kernel<TX, TY>), dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, st, a);
  return hip_status(hipGetLastError(), st);
}

}  // namespace

}  // namespace gdr2

using namespace gdr2;

extern "C" {

gdr2_status gdr2_dropout_fwd(const gdr2_dropout* p, const uint64_t* more, const void* x, const void* r, void* y,
                             hipStream_t stream) {
  const gdr2_status s = drop_check(p, more);
  if (s != GDR2_OK) return s;
  if (p->n > 0 && (x == nullptr || y == nullptr)) return GDR2_EINVAL;
  if (!aligned16(x) || !aligned16(r) || !aligned16(y)) return GDR2_EINVAL;
  if (p->dtype == GDR2_FP32) return drop_launch<float, float>(p, more, x, r, y, stream);
  if (p->stream_dtype == GDR2_FP32) return drop_launch<bf16_t, float>(p, more, x, r, y, stream);
  return drop_launch<bf16_t, bf16_t>(p, more, x, r, y, stream);
}

gdr2_status gdr2_dropout_bwd(const gdr2_dropout* p, const uint64_t* more, const void* dy, void* dx, hipStream_t stream) {
  const gdr2_status s = drop_check(p, more);
  if (s != GDR2_OK) return s;
  if (p->n > 0 && (dy == nullptr || dx == nullptr)) return GDR2_EINVAL;
  if (!aligned16(dy) || !aligned16(dx)) return GDR2_EINVAL;
  if (p->dtype == GDR2_FP32) return drop_launch<float, float>(p, more, dy, nullptr, dx, stream);
  if (p->stream_dtype == GDR2_FP32) return drop_launch<float, bf16_t>(p, more, dy, nullptr, dx, stream);
  return drop_launch<bf16_t, bf16_t>(p, more, dy, nullptr, dx, stream);
}

}  // extern "C"

// C ABI of the gated feed-forward block (include/gdr2_gatedff.h): argument checks, workspace
// layout and launches.  Every check runs before the first HIP call.

#include "../../include/gdr2_gatedff.h"

#include "gdr2_gatedff.hpp"
#include "gdr2_host.hpp"

using namespace gdr2;

namespace {

constexpr int kMaxWidth = 65536;
constexpr int64_t kMaxRows = 1 << 24;

bool need(const void* x) { return x != nullptr && aligned16(x); }

gdr2_status ff_check(const gdr2_gatedff* p) {
  if (p == nullptr || p->rows < 0 || p->D <= 0 || p->F <= 0) return GDR2_EINVAL;
  if (p->dtype != GDR2_BF16 && p->dtype != GDR2_FP32) return GDR2_EINVAL;
  if (p->act != GDR2_ACT_SILU && p->act != GDR2_ACT_GELU) return GDR2_EINVAL;
  if (p->D % 8 != 0 || p->F % 8 != 0 || p->D > kMaxWidth || p->F > kMaxWidth || p->rows > kMaxRows) return GDR2_EUNSUPPORTED;
  return GDR2_OK;
}

// fp32 g and u (rows, F), first: what a saving forward leaves; h (rows, F); backward also dh in
// fp32, and the gradients at g and u
struct FfLayout {
  size_t g, u, h, dh, dg, du, total;
};
FfLayout ff_layout(const gdr2_gatedff* p, bool bwd) {
  const size_t n = (size_t)p->rows * p->F, e = p->dtype == GDR2_BF16 ? 2 : 4;
  FfLayout L{};
  size_t off = 0;
  const auto take = [&](size_t bytes) {
    const size_t at = off;
    off += round_up(bytes);
    return at;
  };
  L.g = take(4 * n);
  L.u = take(4 * n);
  L.h = take(e * n);
  if (bwd) {
    L.dh = take(4 * n);
    L.dg = take(e * n);
    L.du = take(e * n);
  }
  L.total = off + kAlign;
  return L;
}

// c (M, N) = a b^T with rows of a and b along the products' sum
template <typename T, typename TC>
hipError_t rows_by_rows(const T* a, const T* b, TC* c, int64_t M, int64_t N, int64_t K, hipStream_t st) {
  return launch_ff_gemm<T, TC>({{a, nullptr}, {b, nullptr}, K, 1, K, 1, 1, c, M, N, K}, st);
}
// c (M, N) = a0 b0 + a1 b1, a (M, K), b (K, N); a1 may be NULL
template <typename T, typename TC>
hipError_t rows_by_columns(const T* a0, const T* b0, const T* a1, const T* b1, TC* c, int64_t M, int64_t N, int64_t K,
                           hipStream_t st) {
  return launch_ff_gemm<T, TC>({{a0, a1}, {b0, b1}, K, 1, 1, N, a1 ? 2 : 1, c, M, N, K}, st);
}
// c (M, N) = a^T b, a (K, M), b (K, N)
template <typename T>
hipError_t columns_by_columns(const T* a, const T* b, T* c, int64_t M, int64_t N, int64_t K, hipStream_t st) {
  return launch_ff_gemm<T, T>({{a, nullptr}, {b, nullptr}, 1, M, 1, N, 1, c, M, N, K}, st);
}

}  // namespace

extern "C" {

gdr2_status gdr2_gatedff_workspace_bytes(const gdr2_gatedff* p, int for_backward, size_t* bytes) {
  if (bytes == nullptr) return GDR2_EINVAL;
  const gdr2_status s = ff_check(p);
  if (s != GDR2_OK) return s;
  *bytes = ff_layout(p, for_backward != 0).total;
  return GDR2_OK;
}

gdr2_status gdr2_gatedff_fwd(const gdr2_gatedff* p, const void* x, const void* Wg, const void* Wu, const void* Wd, void* y,
                             void* ws, size_t ws_bytes, int save, hipStream_t stream) {
  const gdr2_status s = ff_check(p);
  if (s != GDR2_OK) return s;
  if (!aligned16(x) || !need(Wg) || !need(Wu) || !need(Wd) || !aligned16(y) || !need(ws)) return GDR2_EINVAL;
  if (p->rows > 0 && (x == nullptr || y == nullptr)) return GDR2_EINVAL;
  const FfLayout L = ff_layout(p, save != 0);
  if (ws_bytes < L.total) return GDR2_EWORKSPACE;
  if (p->rows == 0) return GDR2_OK;
  const auto run = [&](auto t) {
    using T = decltype(t);
    const T *xs = static_cast<const T*>(x), *wg = static_cast<const T*>(Wg), *wu = static_cast<const T*>(Wu);
    const int64_t M = p->rows, D = p->D, F = p->F;
    hipError_t e = rows_by_rows<T, float>(xs, wg, at<float>(ws, L.g), M, F, D, stream);
    if (e == hipSuccess) e = rows_by_rows<T, float>(xs, wu, at<float>(ws, L.u), M, F, D, stream);
    if (e == hipSuccess)
      e = launch_ff_act<T>({at<float>(ws, L.g), at<float>(ws, L.u), nullptr, at<T>(ws, L.h), nullptr, nullptr, M * F, p->act},
                           stream);
    if (e == hipSuccess)
      e = rows_by_rows<T, T>(at<T>(ws, L.h), static_cast<const T*>(Wd), static_cast<T*>(y), M, D, F, stream);
    return e;
  };
  return hip_status(p->dtype == GDR2_FP32 ? run(0.f) : run(bf16_t{}), stream);
}

gdr2_status gdr2_gatedff_bwd(const gdr2_gatedff* p, const void* x, const void* Wg, const void* Wu, const void* Wd,
                             const void* dy, void* dx, void* dWg, void* dWu, void* dWd, void* ws, size_t ws_bytes, int saved,
                             hipStream_t stream) {
  const gdr2_status s = ff_check(p);
  if (s != GDR2_OK) return s;
  if (!aligned16(x) || !need(Wg) || !need(Wu) || !need(Wd) || !aligned16(dy) || !aligned16(dx) || !aligned16(dWg) ||
      !aligned16(dWu) || !aligned16(dWd) || !need(ws))
    return GDR2_EINVAL;
  const bool weights = dWg != nullptr;
  if ((dWu != nullptr) != weights || (dWd != nullptr) != weights || (dx == nullptr && !weights)) return GDR2_EINVAL;
  if (p->rows > 0 && (x == nullptr || dy == nullptr)) return GDR2_EINVAL;
  const FfLayout L = ff_layout(p, true);
  if (ws_bytes < L.total) return GDR2_EWORKSPACE;
  const auto run = [&](auto t) {
    using T = decltype(t);
    const T *xs = static_cast<const T*>(x), *wg = static_cast<const T*>(Wg), *wu = static_cast<const T*>(Wu);
    const T *wd = static_cast<const T*>(Wd), *d = static_cast<const T*>(dy);
    float *g = at<float>(ws, L.g), *u = at<float>(ws, L.u), *dh = at<float>(ws, L.dh);
    T *h = at<T>(ws, L.h), *dg = at<T>(ws, L.dg), *du = at<T>(ws, L.du);
    const int64_t M = p->rows, D = p->D, F = p->F;
    hipError_t e = hipSuccess;
    if (M > 0) {
      if (!saved) {
        e = rows_by_rows<T, float>(xs, wg, g, M, F, D, stream);
        if (e == hipSuccess) e = rows_by_rows<T, float>(xs, wu, u, M, F, D, stream);
      }
      if (e == hipSuccess) e = rows_by_columns<T, float>(d, wd, nullptr, nullptr, dh, M, F, D, stream);
      if (e == hipSuccess) e = launch_ff_act<T>({g, u, dh, h, dg, du, M * F, p->act}, stream);
      if (e == hipSuccess && dx) e = rows_by_columns<T, T>(dg, wg, du, wu, static_cast<T*>(dx), M, D, F, stream);
    }
    if (e == hipSuccess && weights) {  // no row: zero
      e = columns_by_columns<T>(dg, xs, static_cast<T*>(dWg), F, D, M, stream);
      if (e == hipSuccess) e = columns_by_columns<T>(du, xs, static_cast<T*>(dWu), F, D, M, stream);
      if (e == hipSuccess) e = columns_by_columns<T>(d, h, static_cast<T*>(dWd), D, F, M, stream);
    }
    return e;
  };
  return hip_status(p->dtype == GDR2_FP32 ? run(0.f) : run(bf16_t{}), stream);
}

}  // extern "C"

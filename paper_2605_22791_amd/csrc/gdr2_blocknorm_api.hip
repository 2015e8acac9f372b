// C ABI of the block norms (include/gdr2_blocknorm.h): argument checks and launches.
// Every check runs before the first HIP call.

#include "../../include/gdr2_blocknorm.h"

#include "gdr2_blocknorm.hpp"
#include "gdr2_host.hpp"

using namespace gdr2;

namespace {

constexpr int kMaxWidth = 8192;

bool need(const void* x) { return x != nullptr && aligned16(x); }
bool may(const void* x) { return x == nullptr || aligned16(x); }

gdr2_status norm_check(const gdr2_blocknorm* p) {
  if (p == nullptr || p->rows < 0 || p->D <= 0) return GDR2_EINVAL;
  if (!std::isfinite(p->eps) || p->eps < 0.f) return GDR2_EINVAL;
  if (p->dtype != GDR2_BF16 && p->dtype != GDR2_FP32) return GDR2_EINVAL;
  if (p->stream_dtype != p->dtype && p->stream_dtype != GDR2_FP32) return GDR2_EINVAL;
  if (p->D > kMaxWidth) return GDR2_EUNSUPPORTED;
  if ((double)p->rows * p->D >= 1099511627776.0) return GDR2_EUNSUPPORTED;  // 2^40 elements
  return GDR2_OK;
}

size_t norm_ws(const gdr2_blocknorm* p) { return round_up((size_t)3 * norm_bwd_blocks(p->rows, p->D, false) * p->D * 4); }

// f(T{}, TS{}): the types of y and of h
template <class F>
hipError_t norm_types(const gdr2_blocknorm* p, bool stream, F&& f) {
  if (p->dtype == GDR2_FP32) return f(0.f, 0.f);
  return stream && p->stream_dtype == GDR2_FP32 ? f(bf16_t{}, 0.f) : f(bf16_t{}, bf16_t{});
}

}  // namespace

extern "C" {

gdr2_status gdr2_blocknorm_fwd(const gdr2_blocknorm* p, const void* y, const float* w_post, const void* z, const void* x,
                               const float* c, const float* w_pre, void* h, void* n, hipStream_t stream) {
  const gdr2_status s = norm_check(p);
  if (s != GDR2_OK) return s;
  if (!need(y) || !may(w_post) || !may(z) || !may(x) || !may(c) || !may(w_pre) || !may(h) || !may(n)) return GDR2_EINVAL;
  if ((n != nullptr) != (w_pre != nullptr) || (h == nullptr && n == nullptr)) return GDR2_EINVAL;
  if (p->rows == 0) return GDR2_OK;
  const hipError_t e = norm_types(p, x != nullptr, [&](auto t, auto ts) {
    using T = decltype(t);
    using TS = decltype(ts);
    return launch_norm_fwd<T, TS>({static_cast<const T*>(y), static_cast<const T*>(z), static_cast<const TS*>(x), w_post, c,
                                   w_pre, static_cast<TS*>(h), static_cast<T*>(n), p->rows, p->D, p->eps}, stream);
  });
  return hip_status(e, stream);
}

gdr2_status gdr2_blocknorm_workspace_bytes(const gdr2_blocknorm* p, size_t* bytes) {
  if (bytes == nullptr) return GDR2_EINVAL;
  const gdr2_status s = norm_check(p);
  if (s != GDR2_OK) return s;
  *bytes = norm_ws(p);
  return GDR2_OK;
}

gdr2_status gdr2_blocknorm_bwd(const gdr2_blocknorm* p, const void* y, const float* w_post, const void* z, const void* x,
                               const float* c, const float* w_pre, const void* dh, const void* dn, void* dy,
                               float* dw_post, void* dz, void* dx, float* dc, float* dw_pre, void* ws, size_t ws_bytes,
                               hipStream_t stream) {
  const gdr2_status s = norm_check(p);
  if (s != GDR2_OK) return s;
  if (!need(y) || !may(w_post) || !may(z) || !may(x) || !may(c) || !may(w_pre) || !may(dh) || !may(dn) || !need(dy) ||
      !may(dw_post) || !may(dz) || !may(dx) || !may(dc) || !may(dw_pre) || !may(ws))
    return GDR2_EINVAL;
  const auto both = [](const void* a, const void* b) { return (a != nullptr) == (b != nullptr); };
  if (!both(dn, w_pre) || !both(dw_post, w_post) || !both(dz, z) || !both(dc, c) || !both(dw_pre, w_pre)) return GDR2_EINVAL;
  if ((dx != nullptr && x == nullptr) || (dh == nullptr && dn == nullptr)) return GDR2_EINVAL;
  const bool sums = w_post != nullptr || c != nullptr || w_pre != nullptr;
  if (sums && p->rows > 0 && ws == nullptr) return GDR2_EINVAL;
  if (sums && ws_bytes < norm_ws(p)) return GDR2_EWORKSPACE;
  const int blocks = norm_bwd_blocks(p->rows, p->D, x != nullptr || c != nullptr || w_pre != nullptr);
  hipError_t e = hipSuccess;
  if (p->rows > 0)
    e = norm_types(p, x != nullptr, [&](auto t, auto ts) {
      using T = decltype(t);
      using TS = decltype(ts);
      NormBwdArgs<T, TS> a{};
      a.y = static_cast<const T*>(y);
      a.z = static_cast<const T*>(z);
      a.dn = static_cast<const T*>(dn);
      a.x = static_cast<const TS*>(x);
      a.dh = static_cast<const TS*>(dh);
      a.w_post = w_post;
      a.c = c;
      a.w_pre = w_pre;
      a.dy = static_cast<T*>(dy);
      a.dz = static_cast<T*>(dz);
      a.dx = static_cast<TS*>(dx);
      a.part = static_cast<float*>(ws);
      a.rows = p->rows;
      a.D = p->D;
      a.blocks = blocks;
      a.eps = p->eps;
      return launch_norm_bwd<T, TS>(a, stream);
    });
  if (e == hipSuccess && sums)  // no row: no block, and the sums are zero
    e = launch_norm_sum({static_cast<const float*>(ws), {dw_post, dc, dw_pre}, p->D, blocks}, stream);
  return hip_status(e, stream);
}

}  // extern "C"

// C ABI of the gated feed-forward block (include/gdr2_gatedff.h): argument checks, workspace
// layout and launches.  Every check runs before the first HIP call.

#include "../../include/gdr2_gatedff.h"

#include <algorithm>

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

// The six products of the block, by what they take
template <typename T>
FfArgs<T> ff_args(int64_t M, int64_t N, int64_t K, const void* a, int64_t lda, const void* b0, const void* b1, int64_t ldb,
                  void* part) {
  FfArgs<T> p{};
  p.a = static_cast<const T*>(a);
  p.b[0] = static_cast<const T*>(b0);
  p.b[1] = static_cast<const T*>(b1);
  p.lda = lda;
  p.ldb = ldb;
  p.M = M;
  p.N = N;
  p.K = K;
  p.pairs = 1;
  p.cut = M;
  p.part = static_cast<float*>(part);
  return p;
}

// h (rows, F), and for a backward g and u with it, first: what a saving forward leaves; the gradients
// at g and u (rows, 2 F); partial tiles of the products
struct FfLayout {
  size_t h, g, u, ge, ue, dgu, part, total;
};
template <typename T>
FfLayout ff_layout_of(const gdr2_gatedff* p, bool bwd) {
  const int64_t M = p->rows, D = p->D, F = p->F;
  const size_t n = (size_t)M * F, e = sizeof(T);
  FfLayout L{};
  size_t off = 0;
  const auto take = [&](size_t bytes) {
    const size_t at = off;
    off += round_up(bytes);
    return at;
  };
  L.h = take(e * n);
  if (bwd) {
    L.g = take(e * n);
    L.u = take(e * n);
    const size_t powers = e == 2 ? (size_t)M * ((F + kFfBlock - 1) / kFfBlock) : 0;
    L.ge = take(powers);
    L.ue = take(powers);
    L.dgu = take(2 * e * n);
  }
  size_t part = 0;
  const auto product = [&](int form, int end, int64_t M, int64_t N, int64_t K, int pairs) {
    part = std::max(part, ff_part_bytes<T>(form, end, M, N, K, pairs));
  };
  if (M > 0) {
    product(FF_ROWS, FF_GATE, M, F, D, 1);
    product(FF_ROWS, FF_STORE, M, D, F, 1);
    if (bwd) {
      product(FF_MIXED, FF_GRAD, M, F, D, 1);
      product(FF_MIXED, FF_STORE, M, D, F, 2);
      product(FF_COLUMNS, FF_STORE, 2 * F, D, M, 1);
      product(FF_COLUMNS, FF_STORE, D, F, M, 1);
    }
  }
  L.part = take(part);
  L.total = off + kAlign;
  return L;
}
FfLayout ff_layout(const gdr2_gatedff* p, bool bwd) {
  return p->dtype == GDR2_FP32 ? ff_layout_of<float>(p, bwd) : ff_layout_of<bf16_t>(p, bwd);
}

template <typename T>
FfHidden<T> ff_hidden(void* ws, const FfLayout& L) {
  return {at<char>(ws, L.g), at<char>(ws, L.u), at<int8_t>(ws, L.ge), at<int8_t>(ws, L.ue)};
}

// h and, where they are asked for, g and u
template <typename T>
hipError_t ff_gate(const gdr2_gatedff* p, const void* x, const void* Wg, const void* Wu, T* h, const FfHidden<T>& hid,
                   void* part, hipStream_t st) {
  FfArgs<T> a = ff_args<T>(p->rows, p->F, p->D, x, p->D, Wg, Wu, p->D, part);
  a.hid = hid;
  a.h = h;
  a.act = p->act;
  return launch_ff<T, FF_ROWS, FF_GATE>(a, st);
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
    T* h = at<T>(ws, L.h);
    void* part = at<char>(ws, L.part);
    hipError_t e = ff_gate<T>(p, x, Wg, Wu, h, save ? ff_hidden<T>(ws, L) : FfHidden<T>{}, part, stream);
    if (e != hipSuccess) return e;
    FfArgs<T> a = ff_args<T>(p->rows, p->D, p->F, h, p->F, Wd, nullptr, p->F, part);
    a.c[0] = static_cast<T*>(y);
    return launch_ff<T, FF_ROWS, FF_STORE>(a, stream);
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
    const FfHidden<T> hid = ff_hidden<T>(ws, L);
    T *h = at<T>(ws, L.h), *dgu = at<T>(ws, L.dgu);
    void* part = at<char>(ws, L.part);
    const int64_t M = p->rows, D = p->D, F = p->F;
    hipError_t e = hipSuccess;
    if (M > 0) {
      if (!saved) e = ff_gate<T>(p, x, Wg, Wu, weights ? h : nullptr, hid, part, stream);
      if (e != hipSuccess) return e;
      FfArgs<T> a = ff_args<T>(M, F, D, dy, D, Wd, nullptr, F, part);
      a.hid = hid;
      a.dgu = dgu;
      a.act = p->act;
      e = launch_ff<T, FF_MIXED, FF_GRAD>(a, stream);
      if (e == hipSuccess && dx) {
        FfArgs<T> b = ff_args<T>(M, D, F, dgu, 2 * F, Wg, Wu, D, part);
        b.pairs = 2;
        b.a2 = F;
        b.c[0] = static_cast<T*>(dx);
        e = launch_ff<T, FF_MIXED, FF_STORE>(b, stream);
      }
    }
    if (e == hipSuccess && weights) {  // no row: zero
      FfArgs<T> a = ff_args<T>(2 * F, D, M, dgu, 2 * F, x, nullptr, D, part);
      a.c[0] = static_cast<T*>(dWg);
      a.c[1] = static_cast<T*>(dWu);
      a.cut = F;
      e = launch_ff<T, FF_COLUMNS, FF_STORE>(a, stream);
      if (e != hipSuccess) return e;
      FfArgs<T> b = ff_args<T>(D, F, M, dy, D, h, nullptr, F, part);
      b.c[0] = static_cast<T*>(dWd);
      e = launch_ff<T, FF_COLUMNS, FF_STORE>(b, stream);
    }
    return e;
  };
  return hip_status(p->dtype == GDR2_FP32 ? run(0.f) : run(bf16_t{}), stream);
}

}  // extern "C"

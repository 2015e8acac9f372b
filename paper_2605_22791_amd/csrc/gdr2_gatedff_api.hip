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
  // a launch has less than 2^32 threads: ff_plan has tiles for every call within these
  if ((double)p->rows * std::max(p->D, p->F) >= 68719476736.0) return GDR2_EUNSUPPORTED;  // 2^36 values
  return GDR2_OK;
}

// ---- the block's products; x, h and the others may be NULL where only sizes count ----
template <typename T>
FfProduct<T> ff_product(int64_t M, int64_t N, const void* a, int64_t lda, const void* b0, const void* b1, int64_t ldb,
                        void* c0, void* c1) {
  FfProduct<T> p{};
  p.a = static_cast<const T*>(a);
  p.b[0] = static_cast<const T*>(b0);
  p.b[1] = static_cast<const T*>(b1);
  p.lda = lda;
  p.ldb = ldb;
  p.M = M;
  p.N = N;
  p.c[0] = static_cast<T*>(c0);
  p.c[1] = static_cast<T*>(c1);
  p.cut = c1 ? M / 2 : M;
  return p;
}
template <typename T>
FfArgs<T> ff_args(const FfProduct<T>& one, int64_t K) {
  FfArgs<T> p{};
  static_cast<FfProduct<T>&>(p) = one;
  p.K = K;
  p.pairs = 1;
  return p;
}
// g, u and h = act(g) u
template <typename T>
FfArgs<T> ff_gate(const gdr2_gatedff* p, const void* x, const void* Wg, const void* Wu) {
  FfArgs<T> a = ff_args(ff_product<T>(p->rows, p->F, x, p->D, Wg, Wu, p->D, nullptr, nullptr), p->D);
  a.act = p->act;
  return a;
}
// y = h Wd^T
template <typename T>
FfArgs<T> ff_down(const gdr2_gatedff* p, const T* h, const void* Wd, void* y) {
  return ff_args(ff_product<T>(p->rows, p->D, h, p->F, Wd, nullptr, p->F, y, nullptr), p->F);
}
// dh = dy Wd, and dg, du from it
template <typename T>
FfArgs<T> ff_grad(const gdr2_gatedff* p, const void* dy, const void* Wd) {
  FfArgs<T> a = ff_args(ff_product<T>(p->rows, p->F, dy, p->D, Wd, nullptr, p->F, nullptr, nullptr), p->D);
  a.act = p->act;
  return a;
}
// dx = dg Wg + du Wu
template <typename T>
FfArgs<T> ff_dx(const gdr2_gatedff* p, const T* dgu, const void* Wg, const void* Wu, void* dx) {
  FfArgs<T> a = ff_args(ff_product<T>(p->rows, p->D, dgu, 2 * (int64_t)p->F, Wg, Wu, p->D, dx, nullptr), p->F);
  a.pairs = 2;
  a.a2 = p->F;
  return a;
}
// dWg = dg^T x, dWu = du^T x, dWd = dy^T h
template <typename T>
FfArgs<T> ff_dw(const gdr2_gatedff* p, const T* dgu, const void* x, const void* dy, const T* h, void* dWg, void* dWu,
                void* dWd) {
  FfArgs<T> a = ff_args(ff_product<T>(2 * (int64_t)p->F, p->D, dgu, 2 * (int64_t)p->F, x, nullptr, p->D, dWg, dWu), p->rows);
  a.cut = p->F;
  a.also = ff_product<T>(p->D, p->F, dy, p->D, h, nullptr, p->F, dWd, nullptr);
  return a;
}

// h (rows, F), and for a backward g and u with it, first: what a saving forward leaves; the gradients
// at g and u (rows, 2 F); partial tiles of the products
struct FfLayout {
  size_t h, g, u, ge, ue, dgu, part, total;
};
template <typename T>
FfLayout ff_layout_of(const gdr2_gatedff* p, bool bwd) {
  const size_t rows = (size_t)p->rows, n = rows * p->F, e = sizeof(T);
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
    const size_t powers = e == 2 ? rows * ((p->F + kFfBlock - 1) / kFfBlock) : 0;
    L.ge = take(powers);
    L.ue = take(powers);
    L.dgu = take(2 * e * n);
  }
  const T* none = nullptr;
  size_t part = std::max(ff_part_bytes<T, FF_ROWS, FF_GATE>(ff_gate<T>(p, none, none, none)),
                         ff_part_bytes<T, FF_ROWS, FF_STORE>(ff_down<T>(p, none, none, nullptr)));
  if (bwd) {
    part = std::max(part, ff_part_bytes<T, FF_MIXED, FF_GRAD>(ff_grad<T>(p, none, none)));
    part = std::max(part, ff_part_bytes<T, FF_MIXED, FF_STORE>(ff_dx<T>(p, none, none, none, nullptr)));
    part = std::max(part, ff_part_bytes<T, FF_COLUMNS, FF_STORE>(ff_dw<T>(p, none, none, none, none, nullptr, nullptr, nullptr)));
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

template <typename T>
hipError_t ff_forward(const gdr2_gatedff* p, const void* x, const void* Wg, const void* Wu, const void* Wd, void* y, void* ws,
                      const FfLayout& L, bool save, hipStream_t st) {
  FfArgs<T> gate = ff_gate<T>(p, x, Wg, Wu), down = ff_down<T>(p, at<T>(ws, L.h), Wd, y);
  gate.part = down.part = at<float>(ws, L.part);
  gate.h = at<T>(ws, L.h);
  if (save) gate.hid = ff_hidden<T>(ws, L);
  const hipError_t e = launch_ff<T, FF_ROWS, FF_GATE>(gate, st);
  return e == hipSuccess ? launch_ff<T, FF_ROWS, FF_STORE>(down, st) : e;
}

template <typename T>
hipError_t ff_backward(const gdr2_gatedff* p, const void* x, const void* Wg, const void* Wu, const void* Wd, const void* dy,
                       void* dx, void* dWg, void* dWu, void* dWd, void* ws, const FfLayout& L, bool saved, hipStream_t st) {
  T *h = at<T>(ws, L.h), *dgu = at<T>(ws, L.dgu);
  float* part = at<float>(ws, L.part);
  hipError_t e = hipSuccess;
  if (p->rows > 0) {
    if (!saved) {
      FfArgs<T> gate = ff_gate<T>(p, x, Wg, Wu);
      gate.hid = ff_hidden<T>(ws, L);
      gate.h = dWd ? h : nullptr;
      gate.part = part;
      e = launch_ff<T, FF_ROWS, FF_GATE>(gate, st);
      if (e != hipSuccess) return e;
    }
    FfArgs<T> grad = ff_grad<T>(p, dy, Wd);
    grad.hid = ff_hidden<T>(ws, L);
    grad.dgu = dgu;
    grad.part = part;
    e = launch_ff<T, FF_MIXED, FF_GRAD>(grad, st);
    if (e == hipSuccess && dx) {
      FfArgs<T> back = ff_dx<T>(p, dgu, Wg, Wu, dx);
      back.part = part;
      e = launch_ff<T, FF_MIXED, FF_STORE>(back, st);
    }
  }
  if (e == hipSuccess && dWd) {  // no row: zero
    FfArgs<T> w = ff_dw<T>(p, dgu, x, dy, h, dWg, dWu, dWd);
    w.part = part;
    e = launch_ff<T, FF_COLUMNS, FF_STORE>(w, st);
  }
  return e;
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
  const hipError_t e = p->dtype == GDR2_FP32 ? ff_forward<float>(p, x, Wg, Wu, Wd, y, ws, L, save != 0, stream)
                                             : ff_forward<bf16_t>(p, x, Wg, Wu, Wd, y, ws, L, save != 0, stream);
  return hip_status(e, stream);
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
  const hipError_t e = p->dtype == GDR2_FP32
                           ? ff_backward<float>(p, x, Wg, Wu, Wd, dy, dx, dWg, dWu, dWd, ws, L, saved != 0, stream)
                           : ff_backward<bf16_t>(p, x, Wg, Wu, Wd, dy, dx, dWg, dWu, dWd, ws, L, saved != 0, stream);
  return hip_status(e, stream);
}

}  // extern "C"

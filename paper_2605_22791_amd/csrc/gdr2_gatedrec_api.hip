// C ABI of the gated linear recurrence (include/gdr2_gatedrec.h): argument checks, workspace
// layout and launches.  Every check runs before the first HIP call.

#include "../../include/gdr2_gatedrec.h"

#include "gdr2_gatedrec.hpp"
#include "gdr2_host.hpp"

using namespace gdr2;

namespace {

constexpr int kMaxChannels = 65536;

gdr2_status rec_check(const gdr2_gatedrec* p, const int32_t* cu, int nseq, bool with_cu) {
  if (p == nullptr || p->B <= 0 || p->T <= 0 || p->D <= 0) return GDR2_EINVAL;
  if (p->dtype != GDR2_BF16 && p->dtype != GDR2_FP32) return GDR2_EINVAL;
  if (p->normalize != 0 && p->normalize != 1) return GDR2_EINVAL;
  if (nseq < 0 || (nseq > 0 && p->B != 1)) return GDR2_EINVAL;
  if (with_cu && nseq > 0 && (cu == nullptr || (reinterpret_cast<uintptr_t>(cu) & 3u) != 0)) return GDR2_EINVAL;
  if (p->D > kMaxChannels || nseq > kMaxSeqs) return GDR2_EUNSUPPORTED;
  if ((double)p->B * p->T >= 2147483648.0) return GDR2_EUNSUPPORTED;
  // (sequence, 256 channels) pairs are workgroups of one launch
  if ((double)(nseq > 0 ? nseq : p->B) * ((p->D + 255) / 256) >= 2147483648.0) return GDR2_EUNSUPPORTED;
  return GDR2_OK;
}

size_t rec_ws(const gdr2_gatedrec* p, bool bwd) { return bwd ? round_up((size_t)p->B * p->T * p->D * 4) : kAlign; }

bool need(const void* x) { return x != nullptr && aligned16(x); }

template <typename T>
RecArgs<T> rec_args(const gdr2_gatedrec* p, const int32_t* cu, int n, const void* x, const float* g, const void* i,
                    const float* h0) {
  RecArgs<T> a{};
  a.x = static_cast<const T*>(x);
  a.i = static_cast<const T*>(i);
  a.g = g;
  a.h0 = h0;
  a.cu = n > 0 ? cu : nullptr;
  a.nseq = n > 0 ? n : p->B;
  a.len = p->T;
  a.D = p->D;
  a.normalize = p->normalize;
  return a;
}

template <typename T>
hipError_t rec_fwd(const gdr2_gatedrec* p, const int32_t* cu, int n, const void* x, const float* g, const void* i,
                   const float* h0, void* o, float* hT, float* hs, hipStream_t st) {
  RecArgs<T> a = rec_args<T>(p, cu, n, x, g, i, h0);
  a.o = static_cast<T*>(o);
  a.hT = hT;
  a.hs = hs;
  return launch_rec_fwd<T>(a, st);
}

}  // namespace

extern "C" {

gdr2_status gdr2_gatedrec_workspace_bytes(const gdr2_gatedrec* p, int32_t n_seqs, int for_backward, size_t* bytes) {
  if (bytes == nullptr) return GDR2_EINVAL;
  const gdr2_status s = rec_check(p, nullptr, n_seqs, false);
  if (s != GDR2_OK) return s;
  *bytes = rec_ws(p, for_backward != 0);
  return GDR2_OK;
}

gdr2_status gdr2_gatedrec_fwd(const gdr2_gatedrec* p, const int32_t* cu, int32_t n, const void* x, const float* g,
                              const void* i, const float* h0, void* o, float* hT, void* ws, size_t ws_bytes, int save,
                              hipStream_t stream) {
  const gdr2_status s = rec_check(p, cu, n, true);
  if (s != GDR2_OK) return s;
  if (!need(x) || !need(g) || !aligned16(i) || !aligned16(h0) || !need(o) || !aligned16(hT) || !need(ws)) return GDR2_EINVAL;
  if (ws_bytes < rec_ws(p, save != 0)) return GDR2_EWORKSPACE;
  float* hs = save ? static_cast<float*>(ws) : nullptr;
  const hipError_t e = p->dtype == GDR2_FP32 ? rec_fwd<float>(p, cu, n, x, g, i, h0, o, hT, hs, stream)
                                             : rec_fwd<bf16_t>(p, cu, n, x, g, i, h0, o, hT, hs, stream);
  return hip_status(e, stream);
}

gdr2_status gdr2_gatedrec_bwd(const gdr2_gatedrec* p, const int32_t* cu, int32_t n, const void* x, const float* g,
                              const void* i, const float* h0, const void* dout, const float* dhT, void* dx, float* dg,
                              void* di, float* dh0, void* ws, size_t ws_bytes, int saved, hipStream_t stream) {
  const gdr2_status s = rec_check(p, cu, n, true);
  if (s != GDR2_OK) return s;
  if (!need(x) || !need(g) || !aligned16(i) || !aligned16(h0) || !need(dout) || !aligned16(dhT) || !need(dx) || !need(dg) ||
      !aligned16(di) || !aligned16(dh0) || !need(ws))
    return GDR2_EINVAL;
  if ((i != nullptr) != (di != nullptr)) return GDR2_EINVAL;
  if (ws_bytes < rec_ws(p, true)) return GDR2_EWORKSPACE;
  const auto run = [&](auto t) {
    using T = decltype(t);
    float* hs = static_cast<float*>(ws);
    if (!saved) {
      const hipError_t e = rec_fwd<T>(p, cu, n, x, g, i, h0, nullptr, nullptr, hs, stream);
      if (e != hipSuccess) return e;
    }
    RecBwdArgs<T> a{};
    a.x = static_cast<const T*>(x);
    a.i = static_cast<const T*>(i);
    a.dout = static_cast<const T*>(dout);
    a.g = g;
    a.h0 = h0;
    a.dhT = dhT;
    a.hs = hs;
    a.cu = n > 0 ? cu : nullptr;
    a.dx = static_cast<T*>(dx);
    a.di = static_cast<T*>(di);
    a.dg = dg;
    a.dh0 = dh0;
    a.nseq = n > 0 ? n : p->B;
    a.len = p->T;
    a.D = p->D;
    a.normalize = p->normalize;
    return launch_rec_bwd<T>(a, stream);
  };
  return hip_status(p->dtype == GDR2_FP32 ? run(0.f) : run(bf16_t{}), stream);
}

gdr2_status gdr2_gatedrec_step(const gdr2_gatedrec* p, const int32_t* cu, int32_t n, const void* x, const float* g,
                               const void* i, float* h, void* o, hipStream_t stream) {
  const gdr2_status s = rec_check(p, cu, n, true);
  if (s != GDR2_OK) return s;
  if (!need(x) || !need(g) || !aligned16(i) || !need(h) || !need(o)) return GDR2_EINVAL;
  const hipError_t e = p->dtype == GDR2_FP32 ? rec_fwd<float>(p, cu, n, x, g, i, h, o, h, nullptr, stream)
                                             : rec_fwd<bf16_t>(p, cu, n, x, g, i, h, o, h, nullptr, stream);
  return hip_status(e, stream);
}

}  // extern "C"

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
  // workgroups of one launch: (tile, 64 channels) and, token by token, (sequence, 256 channels)
  if (((double)p->B * p->T / kRecTile + 1) * ((p->D + 63) / 64) >= 2147483648.0) return GDR2_EUNSUPPORTED;
  if ((double)(nseq > 0 ? nseq : p->B) * ((p->D + 255) / 256) >= 2147483648.0) return GDR2_EUNSUPPORTED;
  return GDR2_OK;
}

// Workspace: the forward chain (a line for its counter, states behind the tiles, factors and
// addends), and for a backward the reverse chain behind it.  One tile needs no chain.
struct RecLayout {
  size_t half, pref, agg, total;  // one chain's bytes, and the offsets in it
  int tiles;
};
RecLayout rec_layout(const gdr2_gatedrec* p, bool bwd) {
  RecLayout L{};
  L.tiles = (int)(((int64_t)p->B * p->T + kRecTile - 1) / kRecTile);
  const size_t n = (size_t)L.tiles * p->D;
  L.pref = kAlign;
  L.agg = L.pref + round_up(4 * n);
  L.half = L.tiles > 1 ? L.agg + round_up(8 * n) : kAlign;
  L.total = (bwd ? 2 : 1) * L.half;
  return L;
}
RecChain rec_chain_at(void* ws, size_t off, const RecLayout& L) {
  return {at<float>(ws, off + L.pref), at<float>(ws, off + L.agg), at<uint32_t>(ws, off)};
}
// chains [from, to) of the workspace as a launch finds them: nothing published, counters at zero
hipError_t rec_clear(void* ws, const RecLayout& L, int from, int to, hipStream_t st) {
  if (L.tiles <= 1) return hipSuccess;
  return launch_rec_clear(at<char>(ws, from * L.half), L.half / 16, to - from, st);
}

bool need(const void* x) { return x != nullptr && aligned16(x); }

// what the arguments of the three kernels share
template <class A>
void rec_shape(A& a, const gdr2_gatedrec* p, const int32_t* cu, int n) {
  a.cu = n > 0 ? cu : nullptr;
  a.nseq = n > 0 ? n : p->B;
  a.len = p->T;
  a.D = p->D;
  a.normalize = p->normalize;
}

template <typename T>
hipError_t rec_fwd(const gdr2_gatedrec* p, const int32_t* cu, int n, const void* x, const float* g, const void* i,
                   const float* h0, void* o, float* hT, const RecChain& chain, hipStream_t st) {
  RecArgs<T> a{};
  rec_shape(a, p, cu, n);
  a.x = static_cast<const T*>(x);
  a.i = static_cast<const T*>(i);
  a.g = g;
  a.h0 = h0;
  a.o = static_cast<T*>(o);
  a.hT = hT;
  a.chain = chain;
  a.rows = p->B * p->T;
  return launch_rec_fwd<T>(a, st);
}

template <typename T>
hipError_t rec_step(const gdr2_gatedrec* p, const int32_t* cu, int n, const void* x, const float* g, const void* i, float* h,
                    void* o, hipStream_t st) {
  RecStepArgs<T> a{};
  rec_shape(a, p, cu, n);
  a.x = static_cast<const T*>(x);
  a.i = static_cast<const T*>(i);
  a.g = g;
  a.o = static_cast<T*>(o);
  a.h = h;
  return launch_rec_step<T>(a, st);
}

}  // namespace

extern "C" {

gdr2_status gdr2_gatedrec_workspace_bytes(const gdr2_gatedrec* p, int32_t n_seqs, int for_backward, size_t* bytes) {
  if (bytes == nullptr) return GDR2_EINVAL;
  const gdr2_status s = rec_check(p, nullptr, n_seqs, false);
  if (s != GDR2_OK) return s;
  *bytes = rec_layout(p, for_backward != 0).total;
  return GDR2_OK;
}

gdr2_status gdr2_gatedrec_fwd(const gdr2_gatedrec* p, const int32_t* cu, int32_t n, const void* x, const float* g,
                              const void* i, const float* h0, void* o, float* hT, void* ws, size_t ws_bytes, int save,
                              hipStream_t stream) {
  const gdr2_status s = rec_check(p, cu, n, true);
  if (s != GDR2_OK) return s;
  if (!need(x) || !need(g) || !aligned16(i) || !aligned16(h0) || !need(o) || !aligned16(hT) || !need(ws)) return GDR2_EINVAL;
  const RecLayout L = rec_layout(p, save != 0);
  if (ws_bytes < L.total) return GDR2_EWORKSPACE;
  const RecChain chain = rec_chain_at(ws, 0, L);
  hipError_t e = rec_clear(ws, L, 0, 1, stream);
  if (e == hipSuccess)
    e = p->dtype == GDR2_FP32 ? rec_fwd<float>(p, cu, n, x, g, i, h0, o, hT, chain, stream)
                              : rec_fwd<bf16_t>(p, cu, n, x, g, i, h0, o, hT, chain, stream);
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
  const RecLayout L = rec_layout(p, true);
  if (ws_bytes < L.total) return GDR2_EWORKSPACE;
  const auto run = [&](auto t) {
    using T = decltype(t);
    const RecChain forward = rec_chain_at(ws, 0, L);
    hipError_t e = rec_clear(ws, L, saved ? 1 : 0, 2, stream);
    if (e == hipSuccess && !saved && L.tiles > 1) e = rec_fwd<T>(p, cu, n, x, g, i, h0, nullptr, nullptr, forward, stream);
    if (e != hipSuccess) return e;
    RecBwdArgs<T> a{};
    rec_shape(a, p, cu, n);
    a.x = static_cast<const T*>(x);
    a.i = static_cast<const T*>(i);
    a.dout = static_cast<const T*>(dout);
    a.g = g;
    a.h0 = h0;
    a.dhT = dhT;
    a.states = forward.pref;
    a.dx = static_cast<T*>(dx);
    a.di = static_cast<T*>(di);
    a.dg = dg;
    a.dh0 = dh0;
    a.chain = rec_chain_at(ws, L.half, L);
    a.rows = p->B * p->T;
    return launch_rec_bwd<T>(a, stream);
  };
  return hip_status(p->dtype == GDR2_FP32 ? run(0.f) : run(bf16_t{}), stream);
}

gdr2_status gdr2_gatedrec_step(const gdr2_gatedrec* p, const int32_t* cu, int32_t n, const void* x, const float* g,
                               const void* i, float* h, void* o, hipStream_t stream) {
  const gdr2_status s = rec_check(p, cu, n, true);
  if (s != GDR2_OK) return s;
  if (!need(x) || !need(g) || !aligned16(i) || !need(h) || !need(o)) return GDR2_EINVAL;
  const hipError_t e = p->dtype == GDR2_FP32 ? rec_step<float>(p, cu, n, x, g, i, h, o, stream)
                                             : rec_step<bf16_t>(p, cu, n, x, g, i, h, o, stream);
  return hip_status(e, stream);
}

}  // extern "C"

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
  // a launch has less than 2^32 threads: 512 for 64 tokens and 64 or 128 channels, and token by token
  // 256 for a sequence and 256 channels
  const double groups = (p->D + rec_channels(p->D) - 1) / rec_channels(p->D);
  if (((double)p->B * p->T / kRecBlock + 1) * groups * (64 * kRecWaves) >= 4294967296.0) return GDR2_EUNSUPPORTED;
  if ((double)(nseq > 0 ? nseq : p->B) * ((p->D + 255) / 256) * 256 >= 4294967296.0) return GDR2_EUNSUPPORTED;
  return GDR2_OK;
}

// Workspace: the chains of the forward's and the backward's tiles (counters, states behind the tiles,
// factors and addends), and the states that a backward starts from.  One tile needs no chain.
struct RecLayout {
  struct Chain {
    size_t at, pref, agg, bytes;
    int tiles;
  } chain[2];  // forward, backward
  size_t states, total;
};
RecLayout rec_layout(const gdr2_gatedrec* p, int nseq, bool bwd) {
  RecLayout L{};
  const int64_t rows = (int64_t)p->B * p->T;
  size_t off = 0;
  for (int k = 0; k < (bwd ? 2 : 1); ++k) {
    RecLayout::Chain& c = L.chain[k];
    const int tile = k == 0 ? rec_tile(nseq > 0 ? p->T / nseq : p->T, rows, p->D) : kRecBlock;
    c.tiles = (int)((rows + tile - 1) / tile);
    c.at = off;
    if (c.tiles > 1) {
      const size_t n = (size_t)c.tiles * p->D;
      c.pref = round_up((size_t)(p->D + 63) / 64 * 64);  // a counter for 64 channels, 64 bytes apart
      c.agg = c.pref + round_up(4 * n);
      c.bytes = c.agg + round_up(8 * n);
    }
    off += c.bytes;
  }
  L.states = off;
  if (bwd) off += round_up((size_t)L.chain[1].tiles * p->D * 4);
  L.total = off + kAlign;
  return L;
}
RecChain rec_chain_at(void* ws, const RecLayout::Chain& c) {
  return {at<float>(ws, c.at + c.pref), at<float>(ws, c.at + c.agg), at<uint32_t>(ws, c.at)};
}
RecClear rec_clear(void* ws, const RecLayout::Chain& c) { return {at<char>(ws, c.at), c.bytes / 16, c.pref / 16}; }

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
                   const float* h0, void* o, float* hT, const RecLayout& L, void* ws, bool save, hipStream_t st) {
  RecArgs<T> a{};
  rec_shape(a, p, cu, n);
  a.x = static_cast<const T*>(x);
  a.i = static_cast<const T*>(i);
  a.g = g;
  a.h0 = h0;
  a.o = static_cast<T*>(o);
  a.hT = hT;
  a.states = save ? at<float>(ws, L.states) : nullptr;
  a.chain = rec_chain_at(ws, L.chain[0]);
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
  *bytes = rec_layout(p, n_seqs, for_backward != 0).total;
  return GDR2_OK;
}

gdr2_status gdr2_gatedrec_fwd(const gdr2_gatedrec* p, const int32_t* cu, int32_t n, const void* x, const float* g,
                              const void* i, const float* h0, void* o, float* hT, void* ws, size_t ws_bytes, int save,
                              hipStream_t stream) {
  const gdr2_status s = rec_check(p, cu, n, true);
  if (s != GDR2_OK) return s;
  if (!need(x) || !need(g) || !aligned16(i) || !aligned16(h0) || !need(o) || !aligned16(hT) || !need(ws)) return GDR2_EINVAL;
  const RecLayout L = rec_layout(p, n, save != 0);
  if (ws_bytes < L.total) return GDR2_EWORKSPACE;
  hipError_t e = launch_rec_clear(rec_clear(ws, L.chain[0]), {}, stream);
  if (e == hipSuccess)
    e = p->dtype == GDR2_FP32 ? rec_fwd<float>(p, cu, n, x, g, i, h0, o, hT, L, ws, save != 0, stream)
                              : rec_fwd<bf16_t>(p, cu, n, x, g, i, h0, o, hT, L, ws, save != 0, stream);
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
  const RecLayout L = rec_layout(p, n, true);
  if (ws_bytes < L.total) return GDR2_EWORKSPACE;
  const auto run = [&](auto t) {
    using T = decltype(t);
    const bool states = !saved && L.chain[1].tiles > 1;
    hipError_t e = launch_rec_clear(rec_clear(ws, L.chain[1]), states ? rec_clear(ws, L.chain[0]) : RecClear{}, stream);
    if (e == hipSuccess && states) e = rec_fwd<T>(p, cu, n, x, g, i, h0, nullptr, nullptr, L, ws, true, stream);
    if (e != hipSuccess) return e;
    RecBwdArgs<T> a{};
    rec_shape(a, p, cu, n);
    a.x = static_cast<const T*>(x);
    a.i = static_cast<const T*>(i);
    a.dout = static_cast<const T*>(dout);
    a.g = g;
    a.h0 = h0;
    a.dhT = dhT;
    a.states = at<float>(ws, L.states);
    a.dx = static_cast<T*>(dx);
    a.di = static_cast<T*>(di);
    a.dg = dg;
    a.dh0 = dh0;
    a.chain = rec_chain_at(ws, L.chain[1]);
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

// C ABI of linear attention with a decay for each head (include/gdr2_linattn.h):
// argument checks, workspace layout and launches.  Every check runs before the first
// HIP call.

#include "../../include/gdr2_linattn.h"

#include "gdr2_host.hpp"
#include "gdr2_linattn.hpp"

using namespace gdr2;

namespace {

bool decay_ok(int d) { return d == GDR2_DECAY_TOKEN || d == GDR2_DECAY_HEAD; }

// Workspace: chunk states N (and the gradients M of the chunks' end states), exp(G_C),
// the chunk table of a packed call and, backward, the per-value-head parts of grouped
// heads and the per-token decay gradients of per-head decays.
struct LaLayout {
  size_t N, M, eGC, coff, ct0, clen, sord, Pq, Pk, dg, total;
  int NT;
};

LaLayout la_layout(const gdr2_problem* p, bool bwd, int nseq) {
  const gdr2_problem v = value_view(p);
  const int G = group_of(p);
  LaLayout L{};
  L.NT = nseq > 0 ? varlen_slots(p, nseq) : chunks_per_seq(p);
  const size_t NC = (size_t)v.H * L.NT * (nseq > 0 ? 1 : p->B), state = (size_t)p->Dk * p->Dv;
  size_t off = 0;
  const auto take = [&](size_t words) {
    const size_t at = off;
    off += round_up(4 * words);
    return at;
  };
  L.N = take(NC * state);
  L.eGC = take(NC);
  if (nseq > 0) {
    L.coff = take((size_t)nseq + 1);
    L.ct0 = take(L.NT);
    L.clen = take(L.NT);
    L.sord = take(nseq);
  }
  if (bwd) {
    const size_t rows = (size_t)p->B * p->T;
    L.M = take(NC * state);
    if (G > 1) {
      L.Pq = take(rows * v.H * p->Dk);
      L.Pk = take(rows * v.H * p->Dk);
    }
    L.dg = take(rows * v.H);
  }
  L.total = off;
  return L;
}

LaGeo la_geo(const gdr2_problem* p, const LaLayout& L, int decay, const int32_t* cu, int nseq, const float* g, void* ws) {
  LaGeo a{};
  const gdr2_problem v = value_view(p);
  if (nseq > 0) {
    a.vl.cu = cu;
    a.vl.coff = at<int>(ws, L.coff);
    a.vl.ct0 = at<int>(ws, L.ct0);
    a.vl.clen = at<int>(ws, L.clen);
    a.vl.sorder = nullptr;  // no kernel here walks the sequences by length
    a.vl.nseq = nseq;
    a.vl.ncmax = L.NT;
  }
  a.B = p->B;
  a.T = p->T;
  a.H = v.H;
  a.G = group_of(p);
  a.NT = L.NT;
  a.scale = p->scale;
  a.g = g;
  a.per_head = decay == GDR2_DECAY_HEAD;
  return a;
}

hipError_t la_table(const gdr2_problem* p, const LaLayout& L, const int32_t* cu, int nseq, void* ws, hipStream_t st) {
  if (nseq == 0) return hipSuccess;
  return launch_varlen_table(cu, nseq, p->T, L.NT, at<int>(ws, L.coff), at<int>(ws, L.ct0), at<int>(ws, L.clen),
                             at<int>(ws, L.sord), st);
}

// the states that enter the chunks, from k and v (rev: the gradients of the end states, from q and dout)
template <int DK, int DV, typename TIn>
hipError_t la_states(const LaGeo& geo, int ns, const void* x, const void* z, float* N, float* eGC, const float* init,
                     float* fin, bool rev, hipStream_t st) {
  const LaStateArgs<TIn> sa{geo, static_cast<const TIn*>(x), static_cast<const TIn*>(z), N, eGC};
  hipError_t e = launch_la_state<DK, DV, TIn>(sa, rev, st);
  if (e != hipSuccess) return e;
  return launch_la_combine({geo, N, eGC, init, fin, ns, DK * DV, rev ? 1 : 0}, st);
}

template <int DK, int DV, typename TIn>
hipError_t la_fwd(const gdr2_problem* p, const LaLayout& L, const LaGeo& geo, int ns, const void* q, const void* k,
                  const void* v, const float* S0, void* o, float* ST, void* ws, hipStream_t st) {
  float *N = at<float>(ws, L.N), *eGC = at<float>(ws, L.eGC);
  hipError_t e = la_states<DK, DV, TIn>(geo, ns, k, v, N, eGC, S0, ST, false, st);
  if (e != hipSuccess) return e;
  return launch_la_fwd<DK, DV, TIn>({geo, static_cast<const TIn*>(q), static_cast<const TIn*>(k),
                                     static_cast<const TIn*>(v), static_cast<TIn*>(o), S0, N, eGC}, st);
}

struct LaGrads {
  void *dq, *dk, *dv;
  float *dg, *dS0;
};

template <int DK, int DV, typename TIn>
hipError_t la_bwd(const gdr2_problem* p, const LaLayout& L, const LaGeo& geo, int ns, const void* q, const void* k,
                  const void* v, const float* S0, const void* dout, const float* dST, const LaGrads& d, void* ws,
                  bool saved, hipStream_t st) {
  float *N = at<float>(ws, L.N), *M = at<float>(ws, L.M), *eGC = at<float>(ws, L.eGC);
  hipError_t e = hipSuccess;
  if (!saved) e = la_states<DK, DV, TIn>(geo, ns, k, v, N, eGC, S0, nullptr, false, st);
  if (e == hipSuccess) e = la_states<DK, DV, TIn>(geo, ns, q, dout, M, eGC, dST, d.dS0, true, st);
  if (e != hipSuccess) return e;
  const size_t rows = (size_t)p->B * p->T;
  LaBwdArgs<TIn> a{};
  a.geo = geo;
  a.q = static_cast<const TIn*>(q);
  a.k = static_cast<const TIn*>(k);
  a.v = static_cast<const TIn*>(v);
  a.dout = static_cast<const TIn*>(dout);
  a.dq = static_cast<TIn*>(d.dq);
  a.dk = static_cast<TIn*>(d.dk);
  a.dv = static_cast<TIn*>(d.dv);
  if (geo.G > 1) {
    a.Pq = at<float>(ws, L.Pq);
    a.Pk = at<float>(ws, L.Pk);
  }
  a.dg = geo.per_head ? at<float>(ws, L.dg) : d.dg;
  a.N = N;
  a.M = M;
  a.eGC = eGC;
  e = launch_la_bwd<DK, DV, TIn>(a, st);
  if (e == hipSuccess && geo.G > 1) e = launch_la_group<TIn>(a.Pq, a.dq, rows, geo.H / geo.G, geo.G, DK, st);
  if (e == hipSuccess && geo.G > 1) e = launch_la_group<TIn>(a.Pk, a.dk, rows, geo.H / geo.G, geo.G, DK, st);
  if (e == hipSuccess && geo.per_head) e = launch_la_headsum(a.dg, d.dg, rows, geo.H, st);
  return e;
}

// f(<Dk>, <Dv>, <type>) as template arguments
template <class F>
hipError_t la_dispatch(const gdr2_problem* p, F&& f) {
  const auto dims = [&](auto t) {
    if (p->Dk == 128)
      return p->Dv == 128 ? f(std::integral_constant<int, 128>{}, std::integral_constant<int, 128>{}, t)
                          : f(std::integral_constant<int, 128>{}, std::integral_constant<int, 64>{}, t);
    return p->Dv == 128 ? f(std::integral_constant<int, 64>{}, std::integral_constant<int, 128>{}, t)
                        : f(std::integral_constant<int, 64>{}, std::integral_constant<int, 64>{}, t);
  };
  return p->dtype == GDR2_BF16 ? dims(bf16_t{}) : dims(0.f);
}

// n_seqs as the calls take it: 0 for a fixed-length batch
gdr2_status la_check(const gdr2_problem* p, int decay, const int32_t* cu, int n_seqs, bool chunked) {
  if (n_seqs < 0) return GDR2_EINVAL;
  const gdr2_status s = check_problem(p, chunked, n_seqs);
  if (s != GDR2_OK) return s;
  if (!decay_ok(decay)) return GDR2_EINVAL;
  if (n_seqs > 0 && (cu == nullptr || (reinterpret_cast<uintptr_t>(cu) & 3u) != 0)) return GDR2_EINVAL;
  return GDR2_OK;
}

bool need(const void* x) { return x != nullptr && aligned16(x); }
bool may(const void* x) { return x == nullptr || aligned16(x); }

}  // namespace

extern "C" {

gdr2_status gdr2_linattn_workspace_bytes(const gdr2_problem* p, int32_t n_seqs, int for_backward, size_t* bytes) {
  if (bytes == nullptr || n_seqs < 0) return GDR2_EINVAL;
  const gdr2_status s = check_problem(p, true, n_seqs);
  if (s != GDR2_OK) return s;
  *bytes = la_layout(p, for_backward != 0, n_seqs).total;
  return GDR2_OK;
}

gdr2_status gdr2_linattn_fwd(const gdr2_problem* p, int32_t decay, const int32_t* cu, int32_t n_seqs, const void* q,
                             const void* k, const void* v, const float* g, const float* S0, void* o, float* S_T,
                             void* ws, size_t ws_bytes, int save, hipStream_t stream) {
  const gdr2_status s = la_check(p, decay, cu, n_seqs, true);
  if (s != GDR2_OK) return s;
  if (!need(q) || !need(k) || !need(v) || !need(g) || !may(S0) || !need(o) || !may(S_T) || !need(ws)) return GDR2_EINVAL;
  const LaLayout L = la_layout(p, save != 0, n_seqs);
  if (ws_bytes < L.total) return GDR2_EWORKSPACE;
  const LaGeo geo = la_geo(p, L, decay, cu, n_seqs, g, ws);
  const int ns = n_seqs > 0 ? n_seqs : p->B;
  hipError_t e = la_table(p, L, cu, n_seqs, ws, stream);
  if (e == hipSuccess)
    e = la_dispatch(p, [&](auto dk, auto dv, auto t) {
      return la_fwd<decltype(dk)::value, decltype(dv)::value, decltype(t)>(p, L, geo, ns, q, k, v, S0, o, S_T, ws, stream);
    });
  return hip_status(e, stream);
}

gdr2_status gdr2_linattn_bwd(const gdr2_problem* p, int32_t decay, const int32_t* cu, int32_t n_seqs, const void* q,
                             const void* k, const void* v, const float* g, const float* S0, const void* dout,
                             const float* dS_T, void* dq, void* dk, void* dv, float* dg, float* dS0, void* ws,
                             size_t ws_bytes, int saved, hipStream_t stream) {
  const gdr2_status s = la_check(p, decay, cu, n_seqs, true);
  if (s != GDR2_OK) return s;
  if (!need(q) || !need(k) || !need(v) || !need(g) || !may(S0) || !need(dout) || !may(dS_T) || !need(dq) || !need(dk) ||
      !need(dv) || !need(dg) || !may(dS0) || !need(ws))
    return GDR2_EINVAL;
  const LaLayout L = la_layout(p, true, n_seqs);
  if (ws_bytes < L.total) return GDR2_EWORKSPACE;
  const LaGeo geo = la_geo(p, L, decay, cu, n_seqs, g, ws);
  const int ns = n_seqs > 0 ? n_seqs : p->B;
  const LaGrads d{dq, dk, dv, dg, dS0};
  hipError_t e = saved ? hipSuccess : la_table(p, L, cu, n_seqs, ws, stream);
  if (e == hipSuccess)
    e = la_dispatch(p, [&](auto ck, auto cv, auto t) {
      return la_bwd<decltype(ck)::value, decltype(cv)::value, decltype(t)>(p, L, geo, ns, q, k, v, S0, dout, dS_T, d, ws,
                                                                           saved != 0, stream);
    });
  return hip_status(e, stream);
}

gdr2_status gdr2_linattn_step(const gdr2_problem* p, int32_t decay, const int32_t* cu, int32_t n_seqs, const void* q,
                              const void* k, const void* v, const float* g, float* S, void* o, hipStream_t stream) {
  const gdr2_status s = la_check(p, decay, cu, n_seqs, false);
  if (s != GDR2_OK) return s;
  if (!need(q) || !need(k) || !need(v) || !need(g) || !need(S) || !need(o)) return GDR2_EINVAL;
  const hipError_t e = la_dispatch(p, [&](auto dk, auto dv, auto t) {
    using T = decltype(t);
    const LaStepArgs<T> a{static_cast<const T*>(q), static_cast<const T*>(k), static_cast<const T*>(v), g, S,
                          static_cast<T*>(o), n_seqs > 0 ? cu : nullptr, n_seqs > 0 ? n_seqs : p->B, p->T,
                          value_view(p).H, group_of(p), decay == GDR2_DECAY_HEAD, p->scale};
    return launch_la_step<decltype(dk)::value, decltype(dv)::value, T>(a, stream);
  });
  return hip_status(e, stream);
}

}  // extern "C"

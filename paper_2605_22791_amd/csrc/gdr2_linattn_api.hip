// C ABI of linear attention with a decay for each head (include/gdr2_linattn.h):
// argument checks, workspace layout and launches.  Every check runs before the first
// HIP call.

#include "../../include/gdr2_linattn.h"

#include <algorithm>

#include "gdr2_host.hpp"
#include "gdr2_linattn.hpp"

using namespace gdr2;

namespace {

constexpr double kMaxRow = 1 << 22;  // values of one token over all heads

bool decay_ok(int d) { return d == GDR2_DECAY_TOKEN || d == GDR2_DECAY_HEAD; }

// fp32 problems: chunk states N (and the gradients M of the chunks' end states), exp(G_C)
// and the chunk table of a packed call.  bf16 problems: the states behind the segments (the
// gradients before them), the segments' decays, the segment table of a packed call and,
// backward, the terms of the decays' gradient with S and dS at its anchors.  Both, backward:
// the per-value-head parts of grouped heads, the per-token gradients of per-head decays.
struct LaLayout {
  size_t N, M, eGC, coff, ct0, clen, sord, Pq, Pk, dg, total;
  size_t S, dS, dec, st0, slen, sseq, soff, pa, pb, ca, cb, aS, aD;
  int NT;
  LaSegs segs;
  int anchors;
  bool multi;  // sequences of more than one segment
};

// Tokens of a segment.  A workgroup scans one head's segment, two are on a CU at a time: sequences
// are cut into as many as fill the 256 CUs once.  (Twice as many, in two rounds, took 95 us where
// one round took 84, nine packed prompts of 8192 tokens in all, 16 value heads, and 809 where one
// took 738, training at 8 x 4096 tokens: each segment costs its state's way to memory and back.)
// A packed batch counts as one sequence of its total length, beside a slot for the end of each, for
// its lengths are on the device.  Cutting takes two more launches: up to three chunks (T 192, 16
// heads: 18 us a call whole, 24 cut) are left whole.
int la_seg_tokens(const gdr2_problem* p, int nseq) {
  const int NT = chunks_per_seq(p);
  const long long H = value_view(p).H, base = (nseq > 0 ? 1 : p->B) * H;
  const long long most = nseq > 0 ? std::max(512 - nseq * H, 256LL) : 512;
  const int nseg = (int)std::max(1LL, std::min(most / base, (long long)NT));
  int chunks = NT <= 3 ? NT : (NT + nseg - 1) / nseg;
  // a segment's rows, the widest in fp32, are one buffer of at most 2^31 bytes
  const long long row = 4LL * H * std::max(p->Dk, p->Dv);
  while (chunks > 1 && chunks * CH * row > (1LL << 31)) chunks = (chunks + 1) / 2;
  return chunks * CH;
}

LaLayout la_layout(const gdr2_problem* p, bool bwd, int nseq) {
  const gdr2_problem v = value_view(p);
  const int G = group_of(p);
  const size_t state = (size_t)p->Dk * p->Dv, rows = (size_t)p->B * p->T;
  LaLayout L{};
  size_t off = 0;
  const auto take = [&](size_t words) {
    const size_t at = off;
    off += round_up(4 * words);
    return at;
  };
  if (p->dtype == GDR2_BF16) {
    LaSegs& s = L.segs;
    s.seg_tokens = la_seg_tokens(p, nseq);
    s.nseq = nseq > 0 ? nseq : p->B;
    s.nseg = (p->T + s.seg_tokens - 1) / s.seg_tokens;
    s.nslot = nseq > 0 ? p->T / s.seg_tokens + nseq : p->B * s.nseg;
    L.anchors = (s.seg_tokens / CH + kLaAnchor - 1) / kLaAnchor;
    L.multi = s.nseg > 1;
    const size_t units = (size_t)s.nslot * v.H;
    if (nseq > 0) {
      L.st0 = take(s.nslot);
      L.slen = take(s.nslot);
      L.sseq = take(s.nslot);
      L.soff = take((size_t)nseq + 1);
    }
    if (L.multi) {
      L.S = take(units * state);
      L.dec = take(units);
    }
    if (bwd) {
      if (L.multi) L.dS = take(units * state);
      L.aS = take(units * L.anchors * state);
      L.aD = take(units * L.anchors * state);
      L.pa = take(rows * v.H);
      L.pb = take(rows * v.H);
      L.ca = take(units * (s.seg_tokens / CH) * 16);
      L.cb = take(units * (s.seg_tokens / CH) * 16);
    }
  } else {
    L.NT = nseq > 0 ? varlen_slots(p, nseq) : chunks_per_seq(p);
    const size_t NC = (size_t)v.H * L.NT * (nseq > 0 ? 1 : p->B);
    L.N = take(NC * state);
    L.eGC = take(NC);
    if (nseq > 0) {
      L.coff = take((size_t)nseq + 1);
      L.ct0 = take(L.NT);
      L.clen = take(L.NT);
      L.sord = take(nseq);
    }
    if (bwd) L.M = take(NC * state);
  }
  if (bwd) {
    if (G > 1) {
      L.Pq = take(rows * v.H * p->Dk);
      L.Pk = take(rows * v.H * p->Dk);
    }
    L.dg = take(rows * v.H);
  }
  L.total = off > 0 ? off : kAlign;  // a call always takes a workspace
  return L;
}

LaGeo la_geo(const gdr2_problem* p, const LaLayout& L, int decay, const int32_t* cu, int nseq, const float* g, void* ws) {
  LaGeo a{};
  const gdr2_problem v = value_view(p);
  if (nseq > 0 && p->dtype == GDR2_FP32) {
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
  if (p->dtype == GDR2_BF16 && nseq <= 64) return hipSuccess;
  if (p->dtype == GDR2_BF16)
    return launch_la_segtable(cu, L.segs, p->T, at<int>(ws, L.st0), at<int>(ws, L.slen), at<int>(ws, L.sseq),
                              at<int>(ws, L.soff), st);
  return launch_varlen_table(cu, nseq, p->T, L.NT, at<int>(ws, L.coff), at<int>(ws, L.ct0), at<int>(ws, L.clen),
                             at<int>(ws, L.sord), st);
}

// the states that enter the chunks, from k and v, and the gradients of their end states, from q and
// dout: those of them whose N is given
template <int DK, int DV>
hipError_t la_states(const LaStateArgs& fwd, const LaStateArgs& rev, const LaCombineArgs& cf, const LaCombineArgs& cr,
                     hipStream_t st) {
  const hipError_t e = launch_la_state<DK, DV>(fwd, rev, st);
  return e != hipSuccess ? e : launch_la_combine(cf, cr, st);
}

LaScanArgs la_scan_args(const LaLayout& L, const LaGeo& geo, const int32_t* cu, int nseq, const void* q, const void* k, const void* v,
                        const float* S0, void* ws) {
  LaScanArgs a{};
  a.geo = geo;
  a.segs = L.segs;
  if (nseq > 0 && nseq <= 64) {
    a.segs.cu = cu;
  } else if (nseq > 0) {
    a.segs.t0 = at<int>(ws, L.st0);
    a.segs.len = at<int>(ws, L.slen);
    a.segs.seq = at<int>(ws, L.sseq);
    a.segs.off = at<int>(ws, L.soff);
  }
  a.q = static_cast<const bf16_t*>(q);
  a.k = static_cast<const bf16_t*>(k);
  a.v = static_cast<const bf16_t*>(v);
  a.S0 = S0;
  a.S = at<float>(ws, L.S);
  a.dS = at<float>(ws, L.dS);
  a.dec = at<float>(ws, L.dec);
  a.anchors = L.anchors;
  return a;
}

// the states behind the segments (rev: the gradients before them)
template <int DK, int DV>
hipError_t la_seg_states(const LaScanArgs& a, bool rev, hipStream_t st) {
  const hipError_t e = launch_la_segstate<DK, DV>(a, rev, st);
  return e != hipSuccess ? e : launch_la_segcombine(a, DK * DV, rev, st);
}

template <int DK, int DV, typename TIn>
hipError_t la_fwd(const gdr2_problem* p, const LaLayout& L, const LaGeo& geo, const int32_t* cu, int nseq, const void* q, const void* k,
                  const void* v, const float* S0, void* o, float* ST, void* ws, hipStream_t st) {
  if constexpr (std::is_same<TIn, bf16_t>::value) {
    LaScanArgs a = la_scan_args(L, geo, cu, nseq, q, k, v, S0, ws);
    a.o = static_cast<bf16_t*>(o);
    a.ST = ST;
    hipError_t e = L.multi ? la_seg_states<DK, DV>(a, false, st) : hipSuccess;
    return e != hipSuccess ? e : launch_la_scan_fwd<DK, DV>(a, st);
  } else {
    float *N = at<float>(ws, L.N), *eGC = at<float>(ws, L.eGC);
    hipError_t e = la_states<DK, DV>({geo, static_cast<const float*>(k), static_cast<const float*>(v), N, eGC}, {},
                                     {geo, N, eGC, S0, ST, nseq > 0 ? nseq : p->B, DK * DV, 0}, {}, st);
    if (e != hipSuccess) return e;
    return launch_la_fwd<DK, DV>({geo, static_cast<const float*>(q), static_cast<const float*>(k),
                                  static_cast<const float*>(v), static_cast<float*>(o), N}, st);
  }
}

struct LaGrads {
  void *dq, *dk, *dv;
  float *dg, *dS0;
};

template <int DK, int DV, typename TIn>
hipError_t la_bwd(const gdr2_problem* p, const LaLayout& L, const LaGeo& geo, const int32_t* cu, int nseq, const void* q, const void* k,
                  const void* v, const float* S0, const void* dout, const float* dST, const LaGrads& d, void* ws,
                  bool saved, hipStream_t st) {
  const size_t rows = (size_t)p->B * p->T;
  float *Pq = geo.G > 1 ? at<float>(ws, L.Pq) : nullptr, *Pk = geo.G > 1 ? at<float>(ws, L.Pk) : nullptr;
  float* dg = geo.per_head ? at<float>(ws, L.dg) : d.dg;
  hipError_t e = hipSuccess;
  if constexpr (std::is_same<TIn, bf16_t>::value) {
    LaScanArgs a = la_scan_args(L, geo, cu, nseq, q, k, v, S0, ws);
    a.dout = static_cast<const bf16_t*>(dout);
    a.dST = dST;
    a.dS0 = d.dS0;
    a.dq = static_cast<bf16_t*>(d.dq);
    a.dk = static_cast<bf16_t*>(d.dk);
    a.dv = static_cast<bf16_t*>(d.dv);
    a.Pq = Pq;
    a.Pk = Pk;
    a.pa = at<float>(ws, L.pa);
    a.pb = at<float>(ws, L.pb);
    a.ca = at<float>(ws, L.ca);
    a.cb = at<float>(ws, L.cb);
    a.aS = at<float>(ws, L.aS);
    a.aD = at<float>(ws, L.aD);
    a.dg = dg;
    if (L.multi && !saved) e = la_seg_states<DK, DV>(a, false, st);
    if (L.multi && e == hipSuccess) e = la_seg_states<DK, DV>(a, true, st);
    if (e == hipSuccess) e = launch_la_scan_bwd<DK, DV>(a, st);
  } else {
    const int ns = nseq > 0 ? nseq : p->B;
    float *N = at<float>(ws, L.N), *M = at<float>(ws, L.M), *eGC = at<float>(ws, L.eGC);
    LaStateArgs fwd{};
    LaCombineArgs cf{};
    if (!saved) {
      fwd = {geo, static_cast<const float*>(k), static_cast<const float*>(v), N, eGC};
      cf = {geo, N, eGC, S0, nullptr, ns, DK * DV, 0};
    }
    e = la_states<DK, DV>(fwd, {geo, static_cast<const float*>(q), static_cast<const float*>(dout), M, eGC}, cf,
                          {geo, M, eGC, dST, d.dS0, ns, DK * DV, 1}, st);
    if (e != hipSuccess) return e;
    e = launch_la_bwd<DK, DV>({geo, static_cast<const float*>(q), static_cast<const float*>(k),
                               static_cast<const float*>(v), static_cast<const float*>(dout), static_cast<float*>(d.dq),
                               static_cast<float*>(d.dk), static_cast<float*>(d.dv), Pq, Pk, dg, N, M}, st);
  }
  if (e == hipSuccess && geo.G > 1)
    e = launch_la_group<TIn>(Pq, Pk, static_cast<TIn*>(d.dq), static_cast<TIn*>(d.dk), rows, geo.H / geo.G, geo.G, DK, st);
  if (e == hipSuccess && geo.per_head) e = launch_la_headsum(dg, d.dg, rows, geo.H, st);
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

// a chunk's rows are reached by 32-bit byte offsets (fp32 parts of grouped heads among them)
bool la_wide(const gdr2_problem* p) { return (double)value_view(p).H * std::max(p->Dk, p->Dv) > kMaxRow; }

// n_seqs as the calls take it: 0 for a fixed-length batch
gdr2_status la_check(const gdr2_problem* p, int decay, const int32_t* cu, int n_seqs, bool chunked) {
  if (n_seqs < 0) return GDR2_EINVAL;
  const gdr2_status s = check_problem(p, chunked, n_seqs);
  if (s != GDR2_OK) return s;
  if (!decay_ok(decay)) return GDR2_EINVAL;
  if (chunked && la_wide(p)) return GDR2_EUNSUPPORTED;
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
  if (la_wide(p)) return GDR2_EUNSUPPORTED;
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
  hipError_t e = la_table(p, L, cu, n_seqs, ws, stream);
  if (e == hipSuccess)
    e = la_dispatch(p, [&](auto dk, auto dv, auto t) {
      return la_fwd<decltype(dk)::value, decltype(dv)::value, decltype(t)>(p, L, geo, cu, n_seqs, q, k, v, S0, o, S_T, ws,
                                                                           stream);
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
  const LaGrads d{dq, dk, dv, dg, dS0};
  hipError_t e = saved ? hipSuccess : la_table(p, L, cu, n_seqs, ws, stream);
  if (e == hipSuccess)
    e = la_dispatch(p, [&](auto ck, auto cv, auto t) {
      return la_bwd<decltype(ck)::value, decltype(cv)::value, decltype(t)>(p, L, geo, cu, n_seqs, q, k, v, S0, dout, dS_T, d,
                                                                           ws, saved != 0, stream);
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

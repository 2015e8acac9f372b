// Host-side pieces that the C ABI files share: argument checks, workspace
// offsets and the status of a call's launches.
#pragma once

#include "../../include/gdr2.h"

#include <cmath>
#include <cstdlib>

#include "gdr2_kernels.hpp"

namespace gdr2 {

constexpr size_t kAlign = 256;

inline size_t round_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

constexpr int kMaxSeqs = 1 << 24;  // sequences of one packed call

// nseq > 0: a packed variable-length call of nseq sequences (B must be 1).
inline gdr2_status check_problem(const gdr2_problem* p, bool chunked, int nseq = 0) {
  if (p == nullptr) return GDR2_EINVAL;
  if (p->B <= 0 || p->T <= 0 || p->H <= 0 || p->Dk <= 0 || p->Dv <= 0) return GDR2_EINVAL;
  if (!std::isfinite(p->scale)) return GDR2_EINVAL;
  if (p->dtype != GDR2_BF16 && p->dtype != GDR2_FP32) return GDR2_EINVAL;
  if (nseq < 0 || (nseq > 0 && p->B != 1)) return GDR2_EINVAL;
  if (p->Hv < 0 || (p->Hv > 0 && p->Hv % p->H != 0)) return GDR2_EINVAL;
  if ((p->Dk != 64 && p->Dk != 128) || (p->Dv != 64 && p->Dv != 128)) return GDR2_EUNSUPPORTED;
  if (chunked && p->chunk != CH) return GDR2_EUNSUPPORTED;
  if (nseq > kMaxSeqs) return GDR2_EUNSUPPORTED;
  const double Hv = p->Hv > 0 ? p->Hv : p->H;
  const double rows = (double)p->B * (double)p->T * Hv;
  const int dmax = p->Dk > p->Dv ? p->Dk : p->Dv;
  if (rows * dmax >= 2147483648.0) return GDR2_EUNSUPPORTED;
  const double states = nseq > 0 ? (double)nseq : (double)p->B;
  if (states * Hv * (double)p->Dk * p->Dv >= 2147483648.0) return GDR2_EUNSUPPORTED;
  return GDR2_OK;
}

// The problem seen from the value heads: every kernel runs per value head
// (H := Hv) and reads the key-side tensors q, k, g, b at key head h / G.
inline gdr2_problem value_view(const gdr2_problem* p) {
  gdr2_problem v = *p;
  v.H = p->Hv > 0 ? p->Hv : p->H;
  v.Hv = 0;
  return v;
}
inline int group_of(const gdr2_problem* p) { return p->Hv > 0 ? p->Hv / p->H : 1; }

// Chunks per sequence of a fixed-length call (the last one partial when 64 does not divide T).
inline int chunks_per_seq(const gdr2_problem* p) { return (p->T + CH - 1) / CH; }
// Chunk slots of a packed call: sum_s ceil(L_s / 64) <= floor(T / 64) + nseq.
inline int varlen_slots(const gdr2_problem* p, int nseq) { return p->T / CH + nseq; }

template <typename T>
T* at(void* ws, size_t off) {
  return reinterpret_cast<T*>(static_cast<char*>(ws) + off);
}

inline bool debug_sync() {
  static const bool on = [] {
    const char* e = std::getenv("GDR2_DEBUG_SYNC");
    return e != nullptr && e[0] == '1';
  }();
  return on;
}

inline gdr2_status hip_status(hipError_t e, hipStream_t st) {
  if (e != hipSuccess) return GDR2_EHIP;
  if (debug_sync()) {
    if (hipStreamSynchronize(st) != hipSuccess) return GDR2_EHIP;
    if (hipGetLastError() != hipSuccess) return GDR2_EHIP;
  }
  return GDR2_OK;
}

}  // namespace gdr2

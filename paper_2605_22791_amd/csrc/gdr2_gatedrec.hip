// Gated linear recurrence (include/gdr2_gatedrec.h), one pass over the tokens each way:
//     h = a h + m i x;   dh = do + a_next dh_next,  dx = m i dh,  di = m x dh,
//     dg = a h_before dh - (a^2 / m) i x dh
// bound by memory: the forward reads x, i and g and writes o, 10 bytes an element in bf16, the
// backward reads do besides and writes three gradients, 18.
//
// A workgroup takes a tile of 128 tokens and 64 or 128 channels, each wave R of the tokens in
// registers, a lane one or two channels.  A step is affine in the state, so a wave's tokens are one
// factor and one addend; waves meet in LDS, tiles through memory: a tile publishes its factor and
// addend, then waits for the state before it, which it takes from the nearest of the eight tiles
// before that has published its own, folded with the factors and addends in between, one after
// the other, as those tiles do it themselves.  So the same bits come out whoever was first, and a chain of
// tiles moves on by up to eight a round trip through memory.  The backward does the same from the
// other end, with the states before the tiles as a forward left them.
//
// Nobody waits for a tile that has not begun: tiles are taken by a counter, in the order of the
// chain, and a tile's predecessors have smaller numbers.  A published value is a whole word that is
// not all ones (a NaN of that pattern is replaced), read and written past the caches of one die, so
// that it needs no other ordering.  Sequences start and end anywhere in a tile: their rows are known
// by three masks that every lane of a wave shares, and a state is chosen, never multiplied by zero,
// where one starts, so that NaN does not cross.

#include "gdr2_gatedrec.hpp"
#include "gdr2_bf16.hpp"

namespace gdr2 {

namespace {

constexpr int kBack = 8;  // tiles before that are looked at
constexpr uint32_t kNone = 0xffffffffu;

// ---- CPL neighbouring channels of a lane, on their way from memory --------------------------
template <typename T, int CPL>
struct RecRaw;
template <>
struct RecRaw<float, 1> {
  float x;
  __device__ __forceinline__ void load(const float* p) { x = *p; }
  __device__ __forceinline__ float get(int) const { return x; }
};
template <>
struct RecRaw<float, 2> {
  float2 x;
  __device__ __forceinline__ void load(const float* p) { x = *reinterpret_cast<const float2*>(p); }
  __device__ __forceinline__ float get(int j) const { return j == 0 ? x.x : x.y; }
};
template <>
struct RecRaw<bf16_t, 1> {
  uint16_t x;
  __device__ __forceinline__ void load(const bf16_t* p) { x = p->x; }
  __device__ __forceinline__ float get(int) const { return __uint_as_float((uint32_t)x << 16); }
};
template <>
struct RecRaw<bf16_t, 2> {
  uint32_t x;
  __device__ __forceinline__ void load(const bf16_t* p) { x = *reinterpret_cast<const uint32_t*>(p); }
  __device__ __forceinline__ float get(int j) const { return __uint_as_float(j == 0 ? x << 16 : x & 0xffff0000u); }
};
__device__ __forceinline__ void rec_put(float* p, const float (&x)[1]) { *p = x[0]; }
__device__ __forceinline__ void rec_put(float* p, const float (&x)[2]) { *reinterpret_cast<float2*>(p) = float2{x[0], x[1]}; }
__device__ __forceinline__ void rec_put(bf16_t* p, const float (&x)[1]) { *reinterpret_cast<__bf16*>(p) = (__bf16)x[0]; }
__device__ __forceinline__ void rec_put(bf16_t* p, const float (&x)[2]) {
  typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
  *reinterpret_cast<bf2*>(p) = bf2{(__bf16)x[0], (__bf16)x[1]};
}

// a = exp(g), and m = sqrt(1 - a^2) by -expm1(2 g), from its series where 1 - a^2 would cancel:
// nine terms, (3/4)^9 / 10! < 2^-25 of the first
template <bool NORM>
__device__ __forceinline__ void rec_factors(float g, float& a, float& m) {
  a = expf(g);
  m = 1.f;
  if constexpr (NORM) {
    const float y = 2.f * g;
    float s = 1.f + y * (1.f / 9.f);
#pragma unroll
    for (int k = 8; k >= 2; --k) s = fmaf(y * s, 1.f / (float)k, 1.f);
    m = __builtin_amdgcn_sqrtf(y > -0.75f ? -y * s : fmaf(-a, a, 1.f));
  }
}

// ---- which rows start, end or belong to a sequence ------------------------------------------
// Rows t0 .. t0 + R of the flattened tokens; every value the same in all lanes of a wave.
struct RecRows {
  uint32_t start, end, valid;
  int first, last;  // sequences of the first and the last row (packed: -1 before the first, nseq behind the last)
};
// the last sequence whose offset is at most t; in [-1, nseq] whatever the offsets hold
__device__ __forceinline__ int rec_find(const int32_t* cu, int nseq, int t) {
  int lo = -1, hi = nseq + 1;  // cu[lo] <= t < cu[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid] <= t)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}
template <int R>
__device__ __forceinline__ RecRows rec_rows(const int32_t* cu, int nseq, int len, int rows, int t0) {
  RecRows w{0, 0, 0, 0, 0};
  const int n = min(R, rows - t0);  // may be below 1
  if (cu == nullptr) {
    int s = t0 / len, pos = t0 - s * len;
    w.first = s;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r < n) {
        w.valid |= 1u << r;
        if (pos == 0) w.start |= 1u << r;
        if (pos == len - 1) w.end |= 1u << r;
        w.last = s;
        if (++pos == len) pos = 0, ++s;
      }
    }
  } else {
    int s = rec_find(cu, nseq, t0);
    w.first = s;
    int from = s >= 0 ? cu[s] : -1, to = s < nseq ? cu[s + 1] : rows;  // the sequence's rows, or those of none
    for (int r = 0; r < n; ++r) {
      const int t = t0 + r;
      while (s < nseq && t >= to) {
        ++s;
        from = to;
        to = s < nseq ? cu[s + 1] : rows;
      }
      if (s >= 0 && s < nseq) {
        w.valid |= 1u << r;
        if (t == from) w.start |= 1u << r;
        if (t == to - 1) w.end |= 1u << r;
      }
    }
    w.last = s;
  }
  return w;
}
__device__ __forceinline__ bool rec_bit(uint32_t m, int r) { return (m >> r & 1u) != 0; }
// the sequence of row t, from that of an earlier (a later) row
__device__ __forceinline__ int rec_later(const int32_t* cu, int nseq, int len, int s, int t) {
  if (cu == nullptr) return t / len;
  while (s + 1 < nseq && (s < 0 || cu[s + 1] <= t)) ++s;
  return s;
}
__device__ __forceinline__ int rec_earlier(const int32_t* cu, int nseq, int len, int s, int t) {
  if (cu == nullptr) return t / len;
  s = min(s, nseq - 1);
  while (s > 0 && cu[s] > t) --s;
  return max(s, 0);
}

// ---- the chain of tiles ----------------------------------------------------------------------
__device__ __forceinline__ uint32_t rec_word(float x) {
  const uint32_t w = __float_as_uint(x);
  return w == kNone ? 0x7fc00000u : w;
}
template <int CPL>
__device__ __forceinline__ void rec_publish(float* pref, const float (&x)[CPL]) {
#pragma unroll
  for (int j = 0; j < CPL; ++j)
    __hip_atomic_store(reinterpret_cast<uint32_t*>(pref) + j, rec_word(x[j]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// One wave's part of the chain, for its lanes' channels c .. c + CPL (on: they exist): tile k takes the
// state through h -> A h + U.  wait: the state before the tile is asked for, and returned in h;
// cut: the state behind it does not depend on the one before.
template <int CPL>
__device__ __forceinline__ void rec_chain(const RecChain& ch, int D, int k, int c, bool on, bool wait, bool cut,
                                          const float (&A)[CPL], const float (&U)[CPL], float (&h)[CPL]) {
  const size_t at = (size_t)k * D + c;
  wait = wait && k > 0;  // (offsets that describe no sequences may ask for a state before the first row)
  if (on) {
    if (cut || !wait) {
      rec_publish<CPL>(ch.pref + at, U);
    } else {
#pragma unroll
      for (int j = 0; j < CPL; ++j)
        __hip_atomic_store(reinterpret_cast<uint64_t*>(ch.agg) + at + j, (uint64_t)rec_word(U[j]) << 32 | rec_word(A[j]),
                           __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
#pragma unroll
  for (int j = 0; j < CPL; ++j) h[j] = 0.f;
  if (!wait) return;
  for (bool have = false; !have;) {
    uint32_t p[kBack][CPL];
    uint64_t f[kBack][CPL];
#pragma unroll
    for (int d = 0; d < kBack; ++d)
#pragma unroll
      for (int j = 0; j < CPL; ++j) {
        const size_t from = (size_t)(k - 1 - d) * D + c + j;
        p[d][j] = kNone;
        f[d][j] = ~0ull;
        if (on && d < k) {
          p[d][j] = __hip_atomic_load(reinterpret_cast<const uint32_t*>(ch.pref) + from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          if (d < kBack - 1)
            f[d][j] = __hip_atomic_load(reinterpret_cast<const uint64_t*>(ch.agg) + from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
      }
#pragma unroll
    for (int d = kBack - 1; d >= 0; --d) {
      bool there = true, folds = true;
#pragma unroll
      for (int j = 0; j < CPL; ++j) {
        there = there && p[d][j] != kNone;
        folds = folds && (uint32_t)f[d][j] != kNone && (uint32_t)(f[d][j] >> 32) != kNone;
      }
      if (d < k && __all(there || !on)) {
        have = true;
#pragma unroll
        for (int j = 0; j < CPL; ++j) h[j] = __uint_as_float(p[d][j]);
      } else if (have && __all(folds || !on)) {
#pragma unroll
        for (int j = 0; j < CPL; ++j) h[j] = fmaf(__uint_as_float((uint32_t)f[d][j]), h[j], __uint_as_float((uint32_t)(f[d][j] >> 32)));
      } else {
        have = false;
      }
    }
    if (!have) __builtin_amdgcn_s_sleep(2);
  }
  if (on && !cut) {
    float e[CPL];
#pragma unroll
    for (int j = 0; j < CPL; ++j) e[j] = fmaf(A[j], h[j], U[j]);
    rec_publish<CPL>(ch.pref + at, e);
  }
}

// the workgroup's number in the chain's order (every lane gets it)
__device__ __forceinline__ int rec_ticket(uint32_t* counter, bool chained) {
  if (!chained) return blockIdx.x;
  __shared__ uint32_t n;
  if (threadIdx.x == 0) n = atomicAdd(counter, 1u);
  __syncthreads();
  return __builtin_amdgcn_readfirstlane((int)n);
}

}  // namespace

// R tokens a wave, kRecTile / R waves
template <typename T, int CPL, int R, bool GATED, bool NORM>
__global__ __launch_bounds__(64 * kRecTile / R) void rec_fwd_kernel(RecArgs<T> a) {
  constexpr int NW = kRecTile / R;
  __shared__ float2 agg[NW][64 * CPL];   // a wave's factor and addend
  __shared__ float before[NW][64 * CPL]; // the state before a wave's tokens
  __shared__ uint32_t cuts[NW];          // whether a sequence starts in them
  const int D = a.D, ncg = (D + 64 * CPL - 1) / (64 * CPL), tiles = (a.rows + kRecTile - 1) / kRecTile;
  const int n = rec_ticket(a.chain.ticket, tiles > 1), tile = n / ncg;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = CPL * lane, c = (n - tile * ncg) * 64 * CPL + col;
  const bool on = c < D;
  const int t0 = tile * kRecTile + wave * R, cs = on ? c : 0;

  RecRaw<T, CPL> rx[R], ri[R];
  RecRaw<float, CPL> rg[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const size_t at = (size_t)min(t0 + r, a.rows - 1) * D + cs;
    rg[r].load(a.g + at);
    rx[r].load(a.x + at);
    if constexpr (GATED) ri[r].load(a.i + at);
  }
  const RecRows w = rec_rows<R>(a.cu, a.nseq, a.len, a.rows, t0);
  float al[R][CPL], u[R][CPL], A[CPL], U[CPL];
#pragma unroll
  for (int j = 0; j < CPL; ++j) A[j] = 1.f, U[j] = 0.f;
  int s = w.first;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool valid = rec_bit(w.valid, r), start = rec_bit(w.start, r);
#pragma unroll
    for (int j = 0; j < CPL; ++j) {
      float m;
      rec_factors<NORM>(rg[r].get(j), al[r][j], m);
      u[r][j] = (GATED ? m * ri[r].get(j) : m) * rx[r].get(j);
      if (!valid) al[r][j] = 1.f, u[r][j] = 0.f;
    }
    if (start && a.h0) {
      s = rec_later(a.cu, a.nseq, a.len, s, t0 + r);
      RecRaw<float, CPL> h0;
      h0.load(a.h0 + (size_t)s * D + cs);
#pragma unroll
      for (int j = 0; j < CPL; ++j) u[r][j] = fmaf(al[r][j], h0.get(j), u[r][j]);
    }
#pragma unroll
    for (int j = 0; j < CPL; ++j) {
      U[j] = start ? u[r][j] : fmaf(al[r][j], U[j], u[r][j]);
      A[j] *= al[r][j];
    }
  }
#pragma unroll
  for (int j = 0; j < CPL; ++j) agg[wave][col + j] = float2{A[j], U[j]};
  if (lane == 0) cuts[wave] = w.start;
  __syncthreads();
  if (wave == 0) {
    float At[CPL], Ut[CPL], h[CPL];
    bool cut = false;
#pragma unroll
    for (int j = 0; j < CPL; ++j) At[j] = 1.f, Ut[j] = 0.f;
    for (int v = 0; v < NW; ++v) {
      const bool here = __builtin_amdgcn_readfirstlane(cuts[v]) != 0;
      cut = cut || here;
#pragma unroll
      for (int j = 0; j < CPL; ++j) {
        const float2 x = agg[v][col + j];
        Ut[j] = here ? x.y : fmaf(x.x, Ut[j], x.y);
        At[j] *= x.x;
      }
    }
#pragma unroll
    for (int j = 0; j < CPL; ++j) h[j] = 0.f;
    if (tiles > 1) rec_chain<CPL>(a.chain, D, tile, c, on, rec_bit(w.valid & ~w.start, 0), cut, At, Ut, h);
    for (int v = 0; v < NW; ++v) {
      const bool here = __builtin_amdgcn_readfirstlane(cuts[v]) != 0;
#pragma unroll
      for (int j = 0; j < CPL; ++j) {
        const float2 x = agg[v][col + j];
        before[v][col + j] = h[j];
        h[j] = here ? x.y : fmaf(x.x, h[j], x.y);
      }
    }
  }
  if (a.o == nullptr) return;
  __syncthreads();
  float h[CPL];
#pragma unroll
  for (int j = 0; j < CPL; ++j) h[j] = before[wave][col + j];
  s = w.first;
#pragma unroll
  for (int r = 0; r < R; ++r) {
#pragma unroll
    for (int j = 0; j < CPL; ++j) h[j] = rec_bit(w.start, r) ? u[r][j] : fmaf(al[r][j], h[j], u[r][j]);
    if (rec_bit(w.valid, r) && on) rec_put(a.o + (size_t)(t0 + r) * D + c, h);
    if (rec_bit(w.end, r) && a.hT) {
      s = rec_later(a.cu, a.nseq, a.len, s, t0 + r);
      if (on) rec_put(a.hT + (size_t)s * D + c, h);
    }
  }
  if (a.cu && a.hT)  // empty sequences, shared out over the tiles' waves
    for (int q = tile * NW + wave; q < a.nseq; q += tiles * NW)
      if (a.cu[q + 1] <= a.cu[q] && on) {
        float h0[CPL];
#pragma unroll
        for (int j = 0; j < CPL; ++j) h0[j] = a.h0 ? a.h0[(size_t)q * D + c + j] : 0.f;
        rec_put(a.hT + (size_t)q * D + c, h0);
      }
}

template <typename T, int CPL, int R, bool GATED, bool NORM>
__global__ __launch_bounds__(64 * kRecTile / R) void rec_bwd_kernel(RecBwdArgs<T> a) {
  constexpr int NW = kRecTile / R;
  __shared__ float2 agg[NW][64 * CPL];   // forward
  __shared__ float radd[NW][64 * CPL];   // backward: the addend (the factor is the same)
  __shared__ float before[NW][64 * CPL], behind[NW][64 * CPL];
  __shared__ uint32_t cuts[NW], rcuts[NW];
  const int D = a.D, ncg = (D + 64 * CPL - 1) / (64 * CPL), tiles = (a.rows + kRecTile - 1) / kRecTile;
  const int n = rec_ticket(a.chain.ticket, tiles > 1), k = n / ncg, tile = tiles - 1 - k;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = CPL * lane, c = (n - k * ncg) * 64 * CPL + col;
  const bool on = c < D;
  const int t0 = tile * kRecTile + wave * R, cs = on ? c : 0;

  RecRaw<T, CPL> rx[R], ri[R], rd[R];
  RecRaw<float, CPL> rg[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const size_t at = (size_t)min(t0 + r, a.rows - 1) * D + cs;
    rg[r].load(a.g + at);
    rx[r].load(a.x + at);
    if constexpr (GATED) ri[r].load(a.i + at);
    rd[r].load(a.dout + at);
  }
  const RecRows w = rec_rows<R>(a.cu, a.nseq, a.len, a.rows, t0);
  float al[R][CPL], m[R][CPL], A[CPL], U[CPL];
  // the state before a sequence's first row and its gradient behind its last one
  const auto state_of = [&](const float* p, int s, float (&h)[CPL]) {
    RecRaw<float, CPL> v;
    if (p) v.load(p + (size_t)s * D + cs);
#pragma unroll
    for (int j = 0; j < CPL; ++j) h[j] = p ? v.get(j) : 0.f;
  };
  const auto input = [&](int r, int j) { return (GATED ? m[r][j] * ri[r].get(j) : m[r][j]) * rx[r].get(j); };
#pragma unroll
  for (int j = 0; j < CPL; ++j) A[j] = 1.f, U[j] = 0.f;
  int s = w.first;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool valid = rec_bit(w.valid, r);
    if (rec_bit(w.start, r)) {
      s = rec_later(a.cu, a.nseq, a.len, s, t0 + r);
      state_of(a.h0, s, U);
    }
#pragma unroll
    for (int j = 0; j < CPL; ++j) {
      rec_factors<NORM>(rg[r].get(j), al[r][j], m[r][j]);
      if (!valid) al[r][j] = 1.f;
      U[j] = fmaf(al[r][j], U[j], valid ? input(r, j) : 0.f);
      A[j] *= al[r][j];
    }
  }
#pragma unroll
  for (int j = 0; j < CPL; ++j) agg[wave][col + j] = float2{A[j], U[j]}, U[j] = 0.f;
  s = w.last;
#pragma unroll
  for (int r = R - 1; r >= 0; --r) {
    if (rec_bit(w.end, r)) {
      s = rec_earlier(a.cu, a.nseq, a.len, s, t0 + r);
      state_of(a.dhT, s, U);
    }
#pragma unroll
    for (int j = 0; j < CPL; ++j) U[j] = al[r][j] * (U[j] + (rec_bit(w.valid, r) ? rd[r].get(j) : 0.f));
  }
#pragma unroll
  for (int j = 0; j < CPL; ++j) radd[wave][col + j] = U[j];
  if (lane == 0) cuts[wave] = w.start, rcuts[wave] = w.end;
  __syncthreads();
  if (wave == 1 % NW) {  // the states before the waves' rows
    float h[CPL];
#pragma unroll
    for (int j = 0; j < CPL; ++j) h[j] = tile > 0 && on ? a.states[(size_t)(tile - 1) * D + c + j] : 0.f;
    for (int v = 0; v < NW; ++v) {
      const bool here = __builtin_amdgcn_readfirstlane(cuts[v]) != 0;
#pragma unroll
      for (int j = 0; j < CPL; ++j) {
        const float2 x = agg[v][col + j];
        before[v][col + j] = h[j];
        h[j] = here ? x.y : fmaf(x.x, h[j], x.y);
      }
    }
  }
  if (wave == NW - 1) {  // the gradients behind them; this wave's last row is the tile's
    float At[CPL], Ut[CPL], h[CPL];
    bool cut = false;
#pragma unroll
    for (int j = 0; j < CPL; ++j) At[j] = 1.f, Ut[j] = 0.f;
    for (int v = NW - 1; v >= 0; --v) {
      const bool here = __builtin_amdgcn_readfirstlane(rcuts[v]) != 0;
      cut = cut || here;
#pragma unroll
      for (int j = 0; j < CPL; ++j) {
        const float f = agg[v][col + j].x, b = radd[v][col + j];
        Ut[j] = here ? b : fmaf(f, Ut[j], b);
        At[j] *= f;
      }
    }
#pragma unroll
    for (int j = 0; j < CPL; ++j) h[j] = 0.f;
    if (tiles > 1) rec_chain<CPL>(a.chain, D, k, c, on, rec_bit(w.valid & ~w.end, R - 1), cut, At, Ut, h);
    for (int v = NW - 1; v >= 0; --v) {
      const bool here = __builtin_amdgcn_readfirstlane(rcuts[v]) != 0;
#pragma unroll
      for (int j = 0; j < CPL; ++j) {
        const float f = agg[v][col + j].x, b = radd[v][col + j];
        behind[v][col + j] = h[j];
        h[j] = here ? b : fmaf(f, h[j], b);
      }
    }
  }
  __syncthreads();
  float h[CPL], hb[R][CPL];
#pragma unroll
  for (int j = 0; j < CPL; ++j) h[j] = before[wave][col + j];
  s = w.first;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (rec_bit(w.start, r)) {
      s = rec_later(a.cu, a.nseq, a.len, s, t0 + r);
      state_of(a.h0, s, h);
    }
#pragma unroll
    for (int j = 0; j < CPL; ++j) {
      hb[r][j] = h[j];
      h[j] = fmaf(al[r][j], h[j], input(r, j));
    }
  }
#pragma unroll
  for (int j = 0; j < CPL; ++j) h[j] = behind[wave][col + j];
  s = w.last;
#pragma unroll
  for (int r = R - 1; r >= 0; --r) {
    if (!rec_bit(w.valid, r)) continue;
    if (rec_bit(w.end, r)) {
      s = rec_earlier(a.cu, a.nseq, a.len, s, t0 + r);
      state_of(a.dhT, s, h);
    }
    float dx[CPL], di[CPL], dg[CPL];
#pragma unroll
    for (int j = 0; j < CPL; ++j) {
      const float dh = rd[r].get(j) + h[j], i = GATED ? ri[r].get(j) : 1.f, x = rx[r].get(j);
      h[j] = al[r][j] * dh;
      const float md = m[r][j] * dh;
      dx[j] = GATED ? md * i : md;
      di[j] = md * x;
      dg[j] = h[j] * hb[r][j];
      if constexpr (NORM) {
        const float slope = m[r][j] > 0.f ? al[r][j] * al[r][j] / m[r][j] : 0.f;
        dg[j] -= slope * i * x * dh;
      }
    }
    if (on) {
      const size_t at = (size_t)(t0 + r) * D + c;
      rec_put(a.dx + at, dx);
      if constexpr (GATED) rec_put(a.di + at, di);
      rec_put(a.dg + at, dg);
    }
    if (rec_bit(w.start, r) && a.dh0) {
      const int q = rec_earlier(a.cu, a.nseq, a.len, s, t0 + r);
      if (on) rec_put(a.dh0 + (size_t)q * D + c, h);
    }
  }
  if (a.cu && a.dh0)  // empty sequences
    for (int q = tile * NW + wave; q < a.nseq; q += tiles * NW)
      if (a.cu[q + 1] <= a.cu[q] && on) {
        state_of(a.dhT, q, h);
        rec_put(a.dh0 + (size_t)q * D + c, h);
      }
}

// Token by token: a lane for each (sequence, channel)
template <typename T>
__global__ __launch_bounds__(256) void rec_step_kernel(RecStepArgs<T> a) {
  const int nc = (a.D + 255) / 256, s = blockIdx.x / nc, c = (blockIdx.x % nc) * 256 + threadIdx.x;
  if (c >= a.D) return;
  int t0 = 0, n = a.len;  // packed offsets are kept in range whatever they are
  size_t row0 = (size_t)s * a.len;
  if (a.cu) {
    t0 = min(max(a.cu[s], 0), a.len);
    n = min(max(a.cu[s + 1], t0), a.len) - t0;
    row0 = t0;
  }
  if (n == 0) return;
  float h = a.h[(size_t)s * a.D + c];
  for (int t = 0; t < n; ++t) {
    const size_t at = (row0 + t) * a.D + c;
    RecRaw<T, 1> x, i;
    x.load(a.x + at);
    float al, m = 1.f;
    if (a.normalize)
      rec_factors<true>(a.g[at], al, m);
    else
      rec_factors<false>(a.g[at], al, m);
    if (a.i) {
      i.load(a.i + at);
      m *= i.get(0);
    }
    h = fmaf(al, h, m * x.get(0));
    const float o[1] = {h};
    rec_put(a.o + at, o);
  }
  a.h[(size_t)s * a.D + c] = h;
}

__global__ __launch_bounds__(256) void rec_clear_kernel(u4v* p, size_t words) {
  u4v* chain = p + blockIdx.y * words;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < words; i += (size_t)gridDim.x * 256) {
    const uint32_t v = i < 16 ? 0u : kNone;
    chain[i] = u4v{v, v, v, v};
  }
}

hipError_t launch_rec_clear(void* p, size_t words, int chains, hipStream_t st) {
  const size_t blocks = (words + 255) / 256;
  hipLaunchKernelGGL(rec_clear_kernel, dim3((unsigned)(blocks < 2048 ? blocks : 2048), chains), dim3(256), 0, st,
                     static_cast<u4v*>(p), words);
  return hipGetLastError();
}

namespace {
// f(gated, normalized) with the two as types
template <class F>
hipError_t rec_options(bool gated, bool norm, F&& f) {
  if (gated) return norm ? f(std::true_type{}, std::true_type{}) : f(std::true_type{}, std::false_type{});
  return norm ? f(std::false_type{}, std::true_type{}) : f(std::false_type{}, std::false_type{});
}
template <int CPL>
unsigned rec_blocks(int rows, int D) {
  return (unsigned)((rows + kRecTile - 1) / kRecTile) * (unsigned)((D + 64 * CPL - 1) / (64 * CPL));
}
}  // namespace

template <typename T>
hipError_t launch_rec_fwd(const RecArgs<T>& a, hipStream_t st) {
  constexpr int R = 16;
  return rec_options(a.i != nullptr, a.normalize != 0, [&](auto gated, auto norm) {
    if (a.D % 2 == 0 && a.D > 64)
      hipLaunchKernelGGL((rec_fwd_kernel<T, 2, R, decltype(gated)::value, decltype(norm)::value>), dim3(rec_blocks<2>(a.rows, a.D)),
                         dim3(64 * kRecTile / R), 0, st, a);
    else
      hipLaunchKernelGGL((rec_fwd_kernel<T, 1, R, decltype(gated)::value, decltype(norm)::value>), dim3(rec_blocks<1>(a.rows, a.D)),
                         dim3(64 * kRecTile / R), 0, st, a);
    return hipGetLastError();
  });
}
template <typename T>
hipError_t launch_rec_bwd(const RecBwdArgs<T>& a, hipStream_t st) {
  constexpr int R = 8;
  return rec_options(a.i != nullptr, a.normalize != 0, [&](auto gated, auto norm) {
    if (a.D % 2 == 0 && a.D > 64)
      hipLaunchKernelGGL((rec_bwd_kernel<T, 2, R, decltype(gated)::value, decltype(norm)::value>), dim3(rec_blocks<2>(a.rows, a.D)),
                         dim3(64 * kRecTile / R), 0, st, a);
    else
      hipLaunchKernelGGL((rec_bwd_kernel<T, 1, R, decltype(gated)::value, decltype(norm)::value>), dim3(rec_blocks<1>(a.rows, a.D)),
                         dim3(64 * kRecTile / R), 0, st, a);
    return hipGetLastError();
  });
}
template <typename T>
hipError_t launch_rec_step(const RecStepArgs<T>& a, hipStream_t st) {
  hipLaunchKernelGGL(rec_step_kernel<T>, dim3((unsigned)((size_t)a.nseq * ((a.D + 255) / 256))), dim3(256), 0, st, a);
  return hipGetLastError();
}

#define GDR2_REC(T)                                              \
  template hipError_t launch_rec_fwd<T>(const RecArgs<T>&, hipStream_t);     \
  template hipError_t launch_rec_bwd<T>(const RecBwdArgs<T>&, hipStream_t);  \
  template hipError_t launch_rec_step<T>(const RecStepArgs<T>&, hipStream_t);
GDR2_REC(float)
GDR2_REC(bf16_t)

}  // namespace gdr2

// Gated linear recurrence (include/gdr2_gatedrec.h), one pass over the tokens each way:
//     h = a h + m i x;   dh = do + a_next dh_next,  dx = m i dh,  di = m x dh,
//     dg = a h_before dh - (a^2 / m) i x dh
// bound by memory: the forward reads x, i and g and writes o, 10 bytes an element in bf16, the
// backward reads do besides and writes three gradients, 18.
//
// A workgroup takes a tile of 128 or 64 tokens (the backward: 64) and 64 or 128 channels, each wave R of the
// tokens in registers, a lane one or two channels.  A step is affine in the state, so a wave's tokens are one
// factor and one addend; waves meet in LDS, tiles through memory: a tile publishes its factor and
// addend, then waits for the state before it, which it takes from the nearest of the eight tiles
// before (each wave looks at one; on long chains up to 128 of them) that has published its own, folded with
// the factors and addends in between, one after the other, as those tiles do it themselves.  So the same
// bits come out whoever was first, and a chain of tiles moves on by up to eight (128) a round trip through
// memory, about 1.5 us.  The backward does the same from the other end, with the states before the
// tiles as a forward left them.
//
// Measured (normalized, input gate, bf16; medians of ten traced calls): 8 x 4096 tokens of 2048 channels forward
// 161 us (671 MB, 4.2 TB/s), backward 283 us (1.2 GB, 4.3 TB/s); 65536 tokens of 2048 without gate and norm 245
// and 461 us (1.07 GB, 4.4 TB/s, and 1.88 GB, 4.1 TB/s).  Below that: 1000 tokens of 2048 channels 15 and 20 us, the latency of a tile's life.
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

constexpr uint32_t kNone = 0xffffffffu;
constexpr uint32_t kCut = 1, kWait = 2;
// Looks of 1 to 2 us before a tile gives up: seconds, where a wait takes some of them.  Only calls that overlap on
// one workspace, which is not allowed, get there.  They end, and no more than that is ensured: a tile that gives up
// takes NaN, one whose ticket is out of range writes nothing, and one may fold in what the other call published.
constexpr int kPatience = 1 << 22;

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

// a = exp(g): 2^(k + f) with g log2(e) = k + f, f good to 2^-30; and m = sqrt(1 - a^2) by -expm1(2 g), from its
// series where 1 - a^2 would cancel: nine terms, (3/4)^9 / 10! < 2^-25 of the first
template <bool NORM>
__device__ __forceinline__ void rec_factors(float g, float& a, float& m) {
  constexpr float kHigh = 1.44269504f, kLow = 1.92596299e-8f;  // log2(e)
  const float x = g < -200.f ? -200.f : g;  // (-inf too; exp(-200) is 0 in fp32.  NaN stays.)
  const float k = rintf(x * kHigh), f = fmaf(x, kLow, fmaf(x, kHigh, -k));
  a = ldexpf(__builtin_amdgcn_exp2f(f), (int)k);
  m = 1.f;
  if constexpr (NORM) {
    const float y = 2.f * g;
    float s = 1.f / 362880.f;
    s = fmaf(s, y, 1.f / 40320.f);
    s = fmaf(s, y, 1.f / 5040.f);
    s = fmaf(s, y, 1.f / 720.f);
    s = fmaf(s, y, 1.f / 120.f);
    s = fmaf(s, y, 1.f / 24.f);
    s = fmaf(s, y, 1.f / 6.f);
    s = fmaf(s, y, 0.5f);
    s = fmaf(s, y, 1.f);
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

// What a tile's waves see of the tiles before it: NW at a time, one each (two or four each took 3 to 10 %
// longer), and BACK times as many before they wait for a state among the last of them.
template <int CPL, int NW, int BACK>
struct RecLook {
  float2 step[BACK * NW][64 * CPL];
  float state[NW][64 * CPL];
  float before[64 * CPL];  // what comes of it: the state before the tile
  int found[NW];           // 2: the state is there; 1: factor and addend; 0: neither
};

// Tile k's word to the tiles behind it, from its lanes with channels c .. c + CPL: the state behind it
// where that does not depend on the one before (final), else factor and addend.
template <int CPL>
__device__ __forceinline__ void rec_announce(const RecChain& ch, int D, int k, int c, bool final, const float (&A)[CPL],
                                             const float (&U)[CPL]) {
  const size_t at = (size_t)k * D + c;
  if (final) {
    rec_publish<CPL>(ch.pref + at, U);
  } else {
#pragma unroll
    for (int j = 0; j < CPL; ++j)
      __hip_atomic_store(reinterpret_cast<uint64_t*>(ch.agg) + at + j, (uint64_t)rec_word(U[j]) << 32 | rec_word(A[j]),
                         __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

__device__ __forceinline__ uint32_t rec_peek(const float* pref) {
  return __hip_atomic_load(reinterpret_cast<const uint32_t*>(pref), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t rec_peek2(const float* agg) {
  return __hip_atomic_load(reinterpret_cast<const uint64_t*>(agg), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ bool rec_whole(uint64_t f) { return (uint32_t)f != kNone && (uint32_t)(f >> 32) != kNone; }

// The state before tile k > 0, waited for by the whole workgroup; the first wave gets it, for the others
// it is in look.before behind the next barrier.
template <int CPL, int NW, int BACK>
__device__ __forceinline__ void rec_await(const RecChain& ch, int D, int k, int c, int col, bool on, int wave,
                                          RecLook<CPL, NW, BACK>& look, float (&h)[CPL]) {
  const int lane = threadIdx.x & 63;
  int seen = 0, from = -1, far = 0;
  for (int looks = 0; looks < kPatience; ++looks) {
    const int d = far * NW + wave;
    if (d < k && seen < 2) {
      const size_t at = (size_t)(k - 1 - d) * D + c;
      bool there = true, steps = true;
      if (on) {
        uint32_t p[CPL];
        uint64_t f[CPL];
#pragma unroll
        for (int j = 0; j < CPL; ++j) {
          p[j] = rec_peek(ch.pref + at + j);
          if (seen < 1) f[j] = rec_peek2(ch.agg + 2 * (at + j));
        }
#pragma unroll
        for (int j = 0; j < CPL; ++j) {
          there = there && p[j] != kNone;
          look.state[wave][col + j] = __uint_as_float(p[j]);
          if (seen < 1) {
            steps = steps && rec_whole(f[j]);
            look.step[d][col + j] = float2{__uint_as_float((uint32_t)f[j]), __uint_as_float((uint32_t)(f[j] >> 32))};
          }
        }
      }
      seen = __all(there) ? 2 : seen == 1 || __all(steps) ? 1 : 0;
    }
    if (lane == 0) look.found[wave] = seen;
    __syncthreads();
    int v = 0, f = 1;
    for (; v < NW; ++v) {
      f = __builtin_amdgcn_readfirstlane(look.found[v]);
      if (f != 1) break;
    }
    if (f == 2) {
      from = v;
      break;
    }
    if (f == 1 && far + 1 < BACK) {
      ++far;
      seen = 0;
    } else {
      __builtin_amdgcn_s_sleep(1);
    }
    __syncthreads();  // everyone has read what is written again
  }
  if (wave == 0) {
#pragma unroll
    for (int j = 0; j < CPL; ++j) h[j] = from < 0 ? __uint_as_float(0x7fc00000u) : look.state[from][col + j];
    for (int v = from < 0 ? -1 : far * NW + from - 1; v >= 0; --v)
#pragma unroll
      for (int j = 0; j < CPL; ++j) {
        const float2 f = look.step[v][col + j];
        h[j] = fmaf(f.x, h[j], f.y);
      }
#pragma unroll
    for (int j = 0; j < CPL; ++j) look.before[col + j] = h[j];
  }
}

// The workgroup's tile, in the chain's order (every lane gets it), and its group of channels.  A counter
// for each group, a line apart: one counter for all handed out a tile every 20 ns at best.
__device__ __forceinline__ int rec_ticket(uint32_t* counters, int groups, int tiles, int& group) {
  group = (blockIdx.x + blockIdx.x / groups) % groups;
  if (tiles == 1) return 0;
  __shared__ uint32_t n;
  if (threadIdx.x == 0) n = atomicAdd(counters + 16 * group, 1u);
  __syncthreads();
  return __builtin_amdgcn_readfirstlane((int)n);
}

}  // namespace

// R tokens a wave
template <typename T, int CPL, int R, int BACK, bool GATED, bool NORM>
__global__ __launch_bounds__(64 * kRecWaves, 4) void rec_fwd_kernel(RecArgs<T> a) {
  constexpr int NW = kRecWaves, TILE = R * NW;
  static_assert(kRecBlock % R == 0, "states at waves' ends");
  __shared__ float2 agg[NW][64 * CPL];  // a wave's factor and addend
  __shared__ uint32_t cuts[NW];         // whether a sequence starts in its tokens; the first one asks for a state
  __shared__ RecLook<CPL, NW, BACK> look;
  const int D = a.D, ncg = (D + 64 * CPL - 1) / (64 * CPL), tiles = (a.rows + TILE - 1) / TILE;
  int group;
  const int tile = rec_ticket(a.chain.ticket, ncg, tiles, group);
  if ((uint32_t)tile >= (uint32_t)tiles) return;  // (a counter that another call's launch shares)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = CPL * lane, c = group * 64 * CPL + col;
  const bool on = c < D;
  const int t0 = tile * TILE + wave * R, cs = on ? c : 0;

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
  if (lane == 0) cuts[wave] = (w.start != 0 ? kCut : 0) | (rec_bit(w.valid & ~w.start, 0) ? kWait : 0);
  __syncthreads();
  const bool wait = tile > 0 && (cuts[0] & kWait) != 0;
  float At[CPL], Ut[CPL], h[CPL];
  bool cut = false;
  if (wave == 0 && tiles > 1) {
#pragma unroll
    for (int j = 0; j < CPL; ++j) At[j] = 1.f, Ut[j] = 0.f;
    for (int v = 0; v < NW; ++v) {
      const bool here = (cuts[v] & kCut) != 0;
      cut = cut || here;
#pragma unroll
      for (int j = 0; j < CPL; ++j) {
        const float2 x = agg[v][col + j];
        Ut[j] = here ? x.y : fmaf(x.x, Ut[j], x.y);
        At[j] *= x.x;
      }
    }
    if (on) rec_announce<CPL>(a.chain, D, tile, c, cut || !wait, At, Ut);
  }
#pragma unroll
  for (int j = 0; j < CPL; ++j) h[j] = 0.f;
  if (wait) {
    rec_await<CPL, NW, BACK>(a.chain, D, tile, c, col, on, wave, look, h);
    if (wave == 0 && on && !cut) {
      float e[CPL];
#pragma unroll
      for (int j = 0; j < CPL; ++j) e[j] = fmaf(At[j], h[j], Ut[j]);
      rec_publish<CPL>(a.chain.pref + (size_t)tile * D + c, e);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < CPL; ++j) h[j] = look.before[col + j];
  }
  for (int v = 0; v < wave; ++v) {
    const bool here = (cuts[v] & kCut) != 0;
#pragma unroll
    for (int j = 0; j < CPL; ++j) {
      const float2 x = agg[v][col + j];
      h[j] = here ? x.y : fmaf(x.x, h[j], x.y);
    }
  }
  s = w.first;
#pragma unroll
  for (int r = 0; r < R; ++r) {
#pragma unroll
    for (int j = 0; j < CPL; ++j) h[j] = rec_bit(w.start, r) ? u[r][j] : fmaf(al[r][j], h[j], u[r][j]);
    if (a.o && rec_bit(w.valid, r) && on) rec_put(a.o + (size_t)(t0 + r) * D + c, h);
    if (rec_bit(w.end, r) && a.hT) {
      s = rec_later(a.cu, a.nseq, a.len, s, t0 + r);
      if (on) rec_put(a.hT + (size_t)s * D + c, h);
    }
  }
  if (a.states && (t0 + R) % kRecBlock == 0 && t0 < a.rows && on) rec_put(a.states + (size_t)(t0 / kRecBlock) * D + c, h);
  if (a.cu && a.hT)  // empty sequences, shared out over the tiles' waves
    for (int q = tile * NW + wave; q < a.nseq; q += tiles * NW)
      if (a.cu[q + 1] <= a.cu[q] && on) {
        float h0[CPL];
#pragma unroll
        for (int j = 0; j < CPL; ++j) h0[j] = a.h0 ? a.h0[(size_t)q * D + c + j] : 0.f;
        rec_put(a.hT + (size_t)q * D + c, h0);
      }
}

template <typename T, int CPL, int R, int BACK, bool GATED, bool NORM>
__global__ __launch_bounds__(64 * kRecWaves, 4) void rec_bwd_kernel(RecBwdArgs<T> a) {
  constexpr int NW = kRecWaves, TILE = R * NW;
  static_assert(TILE == kRecBlock, "a tile starts at a stored state");
  __shared__ float2 agg[NW][64 * CPL];   // forward
  __shared__ float radd[NW][64 * CPL];   // backward: the addend (the factor is the same)
  __shared__ uint32_t cuts[NW], rcuts[NW];
  __shared__ RecLook<CPL, NW, BACK> look;
  const int D = a.D, ncg = (D + 64 * CPL - 1) / (64 * CPL), tiles = (a.rows + TILE - 1) / TILE;
  int group;
  const int k = rec_ticket(a.chain.ticket, ncg, tiles, group), tile = tiles - 1 - k;
  if ((uint32_t)k >= (uint32_t)tiles) return;  // (a counter that another call's launch shares)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = CPL * lane, c = group * 64 * CPL + col;
  const bool on = c < D;
  const int t0 = tile * TILE + wave * R, cs = on ? c : 0;

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
  if (lane == 0) {
    cuts[wave] = w.start != 0 ? kCut : 0;
    rcuts[wave] = (w.end != 0 ? kCut : 0) | (rec_bit(w.valid & ~w.end, R - 1) ? kWait : 0);
  }
  float h[CPL];  // the state before the tile
#pragma unroll
  for (int j = 0; j < CPL; ++j) h[j] = tile > 0 && on ? a.states[(size_t)(tile - 1) * D + c + j] : 0.f;
  __syncthreads();
  // the gradient behind the tile's last row, from the other end
  const bool wait = k > 0 && (rcuts[NW - 1] & kWait) != 0;
  float At[CPL], Ut[CPL], back[CPL];
  bool cut = false;
  if (wave == 0 && tiles > 1) {
#pragma unroll
    for (int j = 0; j < CPL; ++j) At[j] = 1.f, Ut[j] = 0.f;
    for (int v = NW - 1; v >= 0; --v) {
      const bool here = (rcuts[v] & kCut) != 0;
      cut = cut || here;
#pragma unroll
      for (int j = 0; j < CPL; ++j) {
        const float f = agg[v][col + j].x, b = radd[v][col + j];
        Ut[j] = here ? b : fmaf(f, Ut[j], b);
        At[j] *= f;
      }
    }
    if (on) rec_announce<CPL>(a.chain, D, k, c, cut || !wait, At, Ut);
  }
#pragma unroll
  for (int j = 0; j < CPL; ++j) back[j] = 0.f;
  if (wait) {
    rec_await<CPL, NW, BACK>(a.chain, D, k, c, col, on, wave, look, back);
    if (wave == 0 && on && !cut) {
      float e[CPL];
#pragma unroll
      for (int j = 0; j < CPL; ++j) e[j] = fmaf(At[j], back[j], Ut[j]);
      rec_publish<CPL>(a.chain.pref + (size_t)k * D + c, e);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < CPL; ++j) back[j] = look.before[col + j];
  }
  for (int v = NW - 1; v > wave; --v) {
    const bool here = (rcuts[v] & kCut) != 0;
#pragma unroll
    for (int j = 0; j < CPL; ++j) {
      const float b = radd[v][col + j];
      back[j] = here ? b : fmaf(agg[v][col + j].x, back[j], b);
    }
  }
  float hb[R][CPL];
  for (int v = 0; v < wave; ++v) {
    const bool here = (cuts[v] & kCut) != 0;
#pragma unroll
    for (int j = 0; j < CPL; ++j) {
      const float2 x = agg[v][col + j];
      h[j] = here ? x.y : fmaf(x.x, h[j], x.y);
    }
  }
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
  for (int j = 0; j < CPL; ++j) h[j] = back[j];
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
        const float slope = m[r][j] > 0.f ? al[r][j] * al[r][j] * __builtin_amdgcn_rcpf(m[r][j]) : 0.f;
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

__global__ __launch_bounds__(256) void rec_clear_kernel(RecClear x, RecClear y) {
  const RecClear& c = blockIdx.y == 0 ? x : y;
  u4v* p = static_cast<u4v*>(c.p);
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < c.words; i += (size_t)gridDim.x * 256) {
    const uint32_t v = i < c.zeros ? 0u : kNone;
    p[i] = u4v{v, v, v, v};
  }
}

hipError_t launch_rec_clear(const RecClear& x, const RecClear& y, hipStream_t st) {
  const size_t words = x.words > y.words ? x.words : y.words, blocks = (words + 255) / 256;
  if (words == 0) return hipSuccess;
  hipLaunchKernelGGL(rec_clear_kernel, dim3((unsigned)(blocks < 2048 ? blocks : 2048), y.words > 0 ? 2 : 1), dim3(256), 0, st, x, y);
  return hipGetLastError();
}

namespace {
// f(gated, normalized) with the two as types
template <class F>
hipError_t rec_options(bool gated, bool norm, F&& f) {
  if (gated) return norm ? f(std::true_type{}, std::true_type{}) : f(std::true_type{}, std::false_type{});
  return norm ? f(std::false_type{}, std::true_type{}) : f(std::false_type{}, std::false_type{});
}
dim3 rec_grid(int rows, int tile, int D) { return dim3((unsigned)((rows + tile - 1) / tile) * (unsigned)rec_groups(D)); }
}  // namespace

template <typename T>
hipError_t launch_rec_fwd(const RecArgs<T>& a, hipStream_t st) {
  const int len = a.cu ? a.len / a.nseq : a.len, tile = rec_tile(len, a.rows, a.D);
  const dim3 grid = rec_grid(a.rows, tile, a.D), block(64 * kRecWaves);
  const bool far = rec_far(len, a.rows, a.D);
  return rec_options(a.i != nullptr, a.normalize != 0, [&](auto gated, auto norm) {
    constexpr bool G = decltype(gated)::value, N = decltype(norm)::value;
    constexpr int R = kRecTile / kRecWaves;
    const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, a); };
    // (a far look goes with tiles of kRecTile)
    if (rec_channels(a.D) == 128) {
      if (far)
        go(rec_fwd_kernel<T, 2, R, kRecFar / 2, G, N>);
      else
        tile == kRecTile ? go(rec_fwd_kernel<T, 2, R, 1, G, N>) : go(rec_fwd_kernel<T, 2, R / 2, 1, G, N>);
    } else {
      if (far)
        go(rec_fwd_kernel<T, 1, R, kRecFar, G, N>);
      else
        tile == kRecTile ? go(rec_fwd_kernel<T, 1, R, 1, G, N>) : go(rec_fwd_kernel<T, 1, R / 2, 1, G, N>);
    }
    return hipGetLastError();
  });
}
template <typename T>
hipError_t launch_rec_bwd(const RecBwdArgs<T>& a, hipStream_t st) {
  const dim3 grid = rec_grid(a.rows, kRecBlock, a.D), block(64 * kRecWaves);
  const bool far = rec_far(a.cu ? a.len / a.nseq : a.len, a.rows, a.D);
  return rec_options(a.i != nullptr, a.normalize != 0, [&](auto gated, auto norm) {
    constexpr bool G = decltype(gated)::value, N = decltype(norm)::value;
    constexpr int R = kRecBlock / kRecWaves;
    const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, a); };
    if (rec_channels(a.D) == 128)
      far ? go(rec_bwd_kernel<T, 2, R, kRecFar / 2, G, N>) : go(rec_bwd_kernel<T, 2, R, 1, G, N>);
    else
      far ? go(rec_bwd_kernel<T, 1, R, kRecFar, G, N>) : go(rec_bwd_kernel<T, 1, R, 1, G, N>);
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

// Gated feed-forward block (include/gdr2_gatedff.h): one product kernel for its products,
//     g = x Wg^T, u = x Wu^T, y = h Wd^T;  dh = dy Wd, dx = dg Wg + du Wu, dWg = dg^T x, dWu = du^T x, dWd = dy^T h
//
// A workgroup takes a tile of C, 256 x 256 in eight waves or 128 x 128 or 64 x 64 in four, through K in
// steps of 128 bytes (64 bf16, 32 fp32): the next step's tiles of A and B come straight into LDS while the
// matrix cores work on this one's.  bf16 products are v_mfma_f32_16x16x32_bf16, fp32 ones
// v_mfma_f32_16x16x4_f32; the operands change places, so that a lane has four neighbouring columns of
// C.  Operands with their sum along the rows are read as 16-byte fragments, the others (bf16) through
// the transposing load; both are stored with their 16-byte pieces exchanged within a row so that
// neither way of reading meets a bank twice.
//
// Tiles that are left over when every CU has had the same number are cut along K so that all CUs have a
// part of them; parts meet in a second launch, in order.  Values past a matrix's end come as zeros
// from the buffer loads' range check, and pieces past the end of the sum are sent out of range.
//
// C leaves through LDS, 16 rows of a wave at a time, so that memory sees whole rows of a tile;
// the activation and its gradient are formed on that way, from fp32.  In bf16 h, dg and du are rounded there, for
// the bf16 products that read them: an output's error is 2.35e-3 of its norm, 1.66e-3 with those in 32 bits; two
// bf16 parts of each would double the products of y, dx and the weights.
//
// Measured, 32768 rows, 2048 -> 5504, us: g, u, h with g and u kept 1550 (0.95 PFLOP/s), y 655 (1.13), dg and du
// 1000 (0.74, beside 1.4 GB of g, u, dg, du), dx 1230 and the weights' gradients 1840 (1.20).  The way from beyond
// L2 and the matrix cores are each near 85 % of y's time: 562 with all its steps in L2, 584 without the
// products.  A library's large bf16 product reaches 1.43 PFLOP/s on this card, and 1.26, 1.29 and 0.78 on the three
// forms at this size.

#include "gdr2_gatedff.hpp"
#include "gdr2_bf16.hpp"

namespace gdr2 {

namespace {

// 16 bytes of an operand: a bf16 fragment, or four fp32 ones
template <typename T>
struct FfType;
template <>
struct FfType<bf16_t> {
  static constexpr int E = 2;
  using Frag = bf8;
  static __device__ __forceinline__ f4 mma(const Frag& a, const Frag& b, f4 c) { return gdr2::mma(a, b, c); }
};
template <>
struct FfType<float> {
  static constexpr int E = 4;
  using Frag = f4;
  static __device__ __forceinline__ f4 mma(const Frag& a, const Frag& b, f4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = mfma_f32(a[i], b[i], c);  // k = 4 (lane / 16) + i in both
    return c;
  }
};

// ---- tiles in LDS -----------------------------------------------------------------------------
// Rows: ROWS rows of 128 bytes, piece p of row r at place p ^ ff_row_swz(r).  16-byte reads serve 16 lanes
// at a time: quads of rows {0-3, 8-11} or {4-7, 12-15}, two neighbouring pieces.
__device__ __forceinline__ int ff_row_swz(int r) { return (r & 2) | ((r & 8) >> 1); }
// Columns: kFfStep / E rows of ROWS elements.  bf16: the transposing load serves 32 lanes at a time, 32 bytes
// of rows {0-3, 8-11} (+ 4); fp32: four rows, four apart, of 64 bytes.
template <typename T, int RB>  // bytes of a row
__device__ __forceinline__ int ff_col_swz(int k) {
  if (sizeof(T) == 4) return (k >> 2 & 3) << 2;
  return RB == 128 ? ((k & 2) | (k & 8) >> 1) : ((k & 3) | ((k & 8) >> 1)) << 1;
}

// One operand's way into LDS: ROWS x 128 bytes by NW waves, 1 KB an instruction.
template <typename T, bool COL, int ROWS, int NW>
struct FfLoad {
  static constexpr int NI = ROWS * kFfStep / 1024 / NW;             // instructions a wave
  static constexpr int RB = COL ? ROWS * (int)sizeof(T) : kFfStep;  // bytes of an LDS row
  static constexpr int RI = 1024 / RB;                           // LDS rows an instruction
  // the exchange is the same in every instruction but for bit 3 of the row in fp32 columns
  static constexpr int FLIP = COL && sizeof(T) == 4 ? (NW * RI & 8) : 0;
  static_assert(NW * RI % 16 == 0 || FLIP != 0, "");
  unsigned row;  // offset of the lane's row in the first instruction
  int piece;     // and the lane's piece there
  __device__ __forceinline__ FfLoad(unsigned ld, int lane, int wave) {  // ld: bytes from row to row
    const int r = wave * RI + lane / (RB / 16);
    piece = (lane % (RB / 16)) ^ (COL ? ff_col_swz<T, RB>(r) : ff_row_swz(r));
    row = r * ld;
  }
  __device__ __forceinline__ unsigned at(int i, unsigned ld) const {
    return row + i * (NW * RI) * ld + ((piece ^ (i & 1 ? FLIP : 0)) << 4);
  }
};

// Written out, and waited for by ff_landed: as builtins, the compiler would hold every LDS read
// behind them.
__device__ __forceinline__ void ff_to_lds(unsigned to, unsigned from, u4v buf) {
  // m0, the place in LDS, has to be written a wait state before the load reads it
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(from), "s"(buf)
               : "memory", "m0");
}
__device__ __forceinline__ void ff_landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ u4v ff_buffer(const void* p, int64_t left) {
  const uint64_t at = (uint64_t)(uintptr_t)p;
  const unsigned n = left <= 0 ? 0u : left > 0x7fffffff ? 0x7fffffffu : (unsigned)left;
  return u4v{(unsigned)at, (unsigned)(at >> 32) & 0xffffu, n, 0x00020000u};
}
constexpr unsigned kOutside = 0x80000000u;  // an offset past every buffer

}  // namespace

template <typename T, int FORM, int END, int BM, int BN>
struct FfTile {
  static constexpr int E = sizeof(T);
  static constexpr int NWM = ff_waves_m(BM), NWN = 2, NW = NWM * NWN, WM = BM / NWM;  // waves of WM x WN
  static constexpr int WN = BN / NWN, MT = WM / 16, NT = WN / 16;
  static constexpr int BK = kFfStep / E;
  static constexpr bool ACOL = FORM == FF_COLUMNS, BCOL = FORM != FF_ROWS;
  static constexpr int BUF = (BM + BN) * kFfStep;
  static constexpr int SLD = WN + 4;                            // floats from row to row where C passes through LDS
  static constexpr int BNC = END == FF_GATE ? BN / 2 : BN;      // columns of N that a tile takes
};

// A wave's strip of C: 16 rows x WN columns, COLS of N; through LDS a lane has CW neighbouring columns, 16
// bytes of T, of IT rows, RI apart.
template <typename T, int FORM, int END, int BM, int BN>
struct FfStrip : FfTile<T, FORM, END, BM, BN> {
  using Z = FfTile<T, FORM, END, BM, BN>;
  static constexpr int CW = 16 / (int)sizeof(T), COLS = END == FF_GATE ? Z::WN / 2 : Z::WN;
  static constexpr int LR = COLS / CW, RI = 64 / LR, IT = 16 / RI;
  static constexpr bool HALVES = END == FF_GATE && sizeof(T) == 2;
  static constexpr int NB = Z::WN / kFfBlock;                  // blocks of a row of the strip with a power of their own
  static_assert(!HALVES || COLS % kFfBlock == 0, "whole blocks");
  static constexpr int BYTES = 16 * (Z::SLD + (HALVES ? NB : 0)) * 4;  // LDS of a wave
  int64_t m, n;  // the strip's first row and column
  int r, c;      // the lane's first row and its columns, within the strip
  __device__ __forceinline__ FfStrip(int64_t m, int64_t n, int lane) : m(m), n(n), r(lane / LR), c(CW * (lane % LR)) {}
  // the lane's rows that there are, RI apart
  __device__ __forceinline__ int rows(const FfArgs<T>& p) const {
    const int left = (int)min((int64_t)16, p.M - m) - r;
    return n + c < p.N && left > 0 ? (left + RI - 1) / RI : 0;
  }
};

// The stored g and u of a strip, loaded ahead
template <typename T, class S>
struct FfPast {
  f4 g[S::IT], u[S::IT];
  __device__ __forceinline__ void load(const FfArgs<T>& p, const S& s) {
    const int rows = s.rows(p);
    const int64_t at = (s.m + s.r) * p.N + s.n + s.c;
    const float *gp = static_cast<const float*>(p.hid.g) + at, *up = static_cast<const float*>(p.hid.u) + at;
#pragma unroll
    for (int it = 0; it < S::IT; ++it, gp += S::RI * p.N, up += S::RI * p.N)
      if (it < rows) {
        g[it] = *reinterpret_cast<const f4*>(gp);
        u[it] = *reinterpret_cast<const f4*>(up);
      }
  }
  __device__ __forceinline__ void get(int it, float (&gx)[4], float (&ux)[4]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) gx[i] = g[it][i], ux[i] = u[it][i];
  }
};
template <class S>
struct FfPast<bf16_t, S> {
  f16x8 g[S::IT], u[S::IT];
  int8_t ge[S::IT], ue[S::IT];
  __device__ __forceinline__ void load(const FfArgs<bf16_t>& p, const S& s) {
    const int rows = s.rows(p);
    const int64_t nb = (p.N + kFfBlock - 1) / kFfBlock, at = (s.m + s.r) * p.N + s.n + s.c;
    const _Float16 *gp = static_cast<const _Float16*>(p.hid.g) + at, *up = static_cast<const _Float16*>(p.hid.u) + at;
    int64_t b = (s.m + s.r) * nb + (s.n + s.c) / kFfBlock;
#pragma unroll
    for (int it = 0; it < S::IT; ++it, gp += S::RI * p.N, up += S::RI * p.N, b += S::RI * nb)
      if (it < rows) {
        g[it] = *reinterpret_cast<const f16x8*>(gp);
        u[it] = *reinterpret_cast<const f16x8*>(up);
        ge[it] = p.hid.ge[b];
        ue[it] = p.hid.ue[b];
      }
  }
  __device__ __forceinline__ void get(int it, float (&gx)[8], float (&ux)[8]) const {
    const float a = ldexpf(1.f, -ge[it]), b = ldexpf(1.f, -ue[it]);
#pragma unroll
    for (int i = 0; i < 8; ++i) gx[i] = (float)g[it][i] * a, ux[i] = (float)u[it][i] * b;
  }
};

__device__ __forceinline__ void ff_put(float* to, const float (&x)[4]) { *reinterpret_cast<f4*>(to) = f4{x[0], x[1], x[2], x[3]}; }
__device__ __forceinline__ void ff_put(bf16_t* to, const float (&x)[8]) { st8(reinterpret_cast<__bf16*>(to), round8(x)); }
__device__ __forceinline__ void ff_keep(float* to, const float (&x)[4], float) { ff_put(to, x); }
__device__ __forceinline__ void ff_keep(_Float16* to, const float (&x)[8], float f) {
  f16x8 h;
#pragma unroll
  for (int i = 0; i < 8; ++i) h[i] = (_Float16)(x[i] * f);
  *reinterpret_cast<f16x8*>(to) = h;
}
template <int N>
__device__ __forceinline__ void ff_take(const float* from, float (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const f4 v = *reinterpret_cast<const f4*>(from + i);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[i + j] = v[j];
  }
}

// act(g) and, where wanted, its slope
template <bool SLOPE>
__device__ __forceinline__ void ff_act(int act, float g, float& a, float& slope) {
  slope = 0.f;
  if (act == 0) {  // SiLU; the logistic function by 2^x and the reciprocal, an ulp each
    const float s = __builtin_amdgcn_rcpf(1.f + ex2(g * -kLog2e));
    a = g * s;
    if constexpr (SLOPE) slope = s * (1.f + g * (1.f - s));
  } else {  // GELU
    const float s = 0.5f * (1.f + erff(g * 0.70710678118654752f));
    a = g * s;
    if constexpr (SLOPE) slope = s + g * expf(-0.5f * g * g) * 0.39894228040143268f;
  }
}

// What lanes of a wave leave for each other in LDS: it serves a wave's instructions in order.
__device__ __forceinline__ void ff_wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A strip's products x, in the lanes' layout, through the wave's place in LDS (lds, BYTES of it).
template <typename T, int END, class S>
__device__ __forceinline__ void ff_leave(const FfArgs<T>& p, const f4* x, float* lds, const S& s, const FfPast<T, S>* past,
                                         int lane) {
  float* power = lds + 16 * S::SLD;  // of the row's blocks: g's, then u's
  ff_wave_order();
#pragma unroll
  for (int j = 0; j < S::NT; ++j) *reinterpret_cast<f4*>(lds + (lane & 15) * S::SLD + 16 * j + 4 * (lane >> 4)) = x[j];
  if constexpr (S::HALVES) {
    if (p.hid.g) {
      const int64_t nb = (p.N + kFfBlock - 1) / kFfBlock, row = s.m + (lane & 15);
#pragma unroll
      for (int b = 0; b < S::NB; ++b) {
        float most = 0.f;
#pragma unroll
        for (int j = 2 * b; j < 2 * b + 2; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float v = fabsf(x[j][i]);
            most = v <= 3.0e38f ? fmaxf(most, v) : most;
          }
        most = fmaxf(most, row_partner16(most, (lane & 16) != 0));
        most = fmaxf(most, row_partner32(most, lane >= 32));
        const int sh = state_shift(most);
        const int64_t col = s.n + kFfBlock * (b % (S::NB / 2));
        if (lane < 16) {
          power[lane * S::NB + b] = ldexpf(1.f, sh);
          if (row < p.M && col < p.N) (b < S::NB / 2 ? p.hid.ge : p.hid.ue)[row * nb + col / kFfBlock] = (int8_t)sh;
        }
      }
    }
  }
  ff_wave_order();
  const int rows = s.rows(p);
  const int64_t row0 = s.m + s.r, col = s.n + s.c;
  int64_t at = row0 * p.N + col;
#pragma unroll
  for (int it = 0; it < S::IT; ++it, at += S::RI * p.N) {
    if (it >= rows) continue;
    const int r = s.r + S::RI * it;
    float v[S::CW];
    ff_take(lds + r * S::SLD + s.c, v);
    if constexpr (END == FF_STORE) {
      ff_put((s.m + r < p.cut ? p.c[0] : p.c[1] - p.cut * p.N) + at, v);
    } else if constexpr (END == FF_GATE) {
      using H = typename std::conditional<sizeof(T) == 2, _Float16, float>::type;
      float u[S::CW];
      ff_take(lds + r * S::SLD + S::COLS + s.c, u);
      if (p.hid.g) {
        const float* f = power + r * S::NB + s.c / kFfBlock;
        ff_keep(static_cast<H*>(p.hid.g) + at, v, S::HALVES ? f[0] : 1.f);
        ff_keep(static_cast<H*>(p.hid.u) + at, u, S::HALVES ? f[S::NB / 2] : 1.f);
      }
      if (p.h) {
#pragma unroll
        for (int i = 0; i < S::CW; ++i) {
          float a, slope;
          ff_act<false>(p.act, v[i], a, slope);
          v[i] = a * u[i];
        }
        ff_put(p.h + at, v);
      }
    } else {
      float g[S::CW], u[S::CW];
      past->get(it, g, u);
#pragma unroll
      for (int i = 0; i < S::CW; ++i) {
        float a, slope;
        ff_act<true>(p.act, g[i], a, slope);
        g[i] = v[i] * u[i] * slope;
        u[i] = v[i] * a;
      }
      T* to = p.dgu + 2 * at - col;
      ff_put(to, g);
      ff_put(to + p.N, u);
    }
  }
}

// The tile of a workgroup: XCDs take blocks in turn, so that a run of neighbouring tiles, eight of M by
// as many of N, is on one and shares its L2.
// FF_COLUMNS: from tile tm tn on those of the second product, which p then becomes.
template <typename T, int FORM>
__device__ __forceinline__ void ff_place(FfArgs<T>& p, int t, int& im, int& in) {
  const int per = p.tiles / 8, rest = p.tiles % 8, x = t % 8;
  t = x * per + min(x, rest) + t / 8;
  if constexpr (FORM == FF_COLUMNS)
    if (t >= p.tm * p.tn) {
      t -= p.tm * p.tn;
      static_cast<FfProduct<T>&>(p) = p.also;
    }
  constexpr int GM = 8;
  const int group = t / (GM * p.tn), first = group * GM, rows = min(GM, p.tm - first), k = t - group * GM * p.tn;
  im = first + k % rows;
  in = k / rows;
}

template <typename T, int FORM, int END, int BM, int BN>
__global__ __launch_bounds__(ff_threads(BM), 2) void ff_kernel(FfArgs<T> p) {
  using Z = FfTile<T, FORM, END, BM, BN>;
  using F = FfType<T>;
  using Frag = typename F::Frag;
  constexpr int E = Z::E, MT = Z::MT, NT = Z::NT;
  __shared__ __align__(1024) unsigned char smem[2 * Z::BUF];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / Z::NWN, wn = wave % Z::NWN, r16 = lane & 15, grp = lane >> 4;
  // whole tiles first; then parts of the others, a tile's parts apart
  int t = blockIdx.x, part = 0, im, in;
  if (t >= p.full) {
    const int left = p.tiles - p.full;
    part = (t - p.full) / left;
    t = p.full + (t - p.full) % left;
  }
  const bool whole = t < p.full;
  const int cut = t - p.full;  // its number among those that are cut
  ff_place<T, FORM>(p, t, im, in);
  const int64_t m0 = (int64_t)im * BM, n0 = (int64_t)in * Z::BNC;
  const int per = (int)((p.K + Z::BK - 1) / Z::BK), steps = per * p.pairs;  // steps of one product, of all
  const int s0 = whole ? 0 : (int)((int64_t)steps * part / p.split);
  const int s1 = whole ? steps : (int)((int64_t)steps * (part + 1) / p.split);

  const unsigned la = (unsigned)(p.lda * E), lb = (unsigned)(p.ldb * E);
  using LA = FfLoad<T, Z::ACOL, BM, Z::NW>;
  using LB = FfLoad<T, Z::BCOL, BN, Z::NW>;
  const LA fa(la, lane, wave);
  const LB fb(lb, lane, wave);
  const unsigned lds = (unsigned)(uintptr_t)(const __attribute__((address_space(3))) void*)smem;
  const auto fetch = [&](int s) {
    const int pair = s >= per ? 1 : 0, k = s - pair * per;
    const int64_t k0 = (int64_t)k * Z::BK;
    const bool last = k == per - 1;
    unsigned to = lds + (s & 1) * Z::BUF;
    asm("" : "+s"(to));
    {
      const T* base = p.a + (pair ? p.a2 : 0);
      const u4v buf = Z::ACOL ? ff_buffer(base + k0 * p.lda + m0, ((p.K - k0 - 1) * p.lda + p.M - m0) * E)
                              : ff_buffer(base + m0 * p.lda + k0, ((min((int64_t)BM, p.M - m0) - 1) * p.lda + p.K - k0) * E);
      const bool past = !Z::ACOL && last && k0 + fa.piece * (16 / E) >= p.K;
#pragma unroll
      for (int i = 0; i < LA::NI; ++i) ff_to_lds(to + (wave + i * Z::NW) * 1024, past ? kOutside : fa.at(i, la), buf);
    }
    {
      const bool past = !Z::BCOL && last && k0 + fb.piece * (16 / E) >= p.K;
      to += BM * kFfStep;
      if constexpr (END == FF_GATE) {
        // the tile's rows: for each wave column half of them Wg's, half Wu's, of the same channels
        constexpr int HALF = Z::WN / 2;
        const int64_t left = ((min((int64_t)Z::BNC, p.N - n0) - 1) * p.ldb + p.K - k0) * E;
        const u4v b0 = ff_buffer(p.b[0] + n0 * p.ldb + k0, left), b1 = ff_buffer(p.b[1] + n0 * p.ldb + k0, left);
#pragma unroll
        for (int i = 0; i < LB::NI; ++i) {
          const int row = (wave + i * Z::NW) * LB::RI, w = row % Z::WN, f = row / Z::WN * HALF + w % HALF;  // the instruction's first row
          const unsigned at = past ? kOutside : (f + lane / 8) * lb + fb.piece * 16;
          if (w < HALF)
            ff_to_lds(to + (wave + i * Z::NW) * 1024, at, b0);
          else
            ff_to_lds(to + (wave + i * Z::NW) * 1024, at, b1);
        }
      } else {
        const T* base = p.b[pair];
        const u4v buf = Z::BCOL ? ff_buffer(base + k0 * p.ldb + n0, ((p.K - k0 - 1) * p.ldb + p.N - n0) * E)
                                : ff_buffer(base + n0 * p.ldb + k0, ((min((int64_t)BN, p.N - n0) - 1) * p.ldb + p.K - k0) * E);
#pragma unroll
        for (int i = 0; i < LB::NI; ++i) ff_to_lds(to + (wave + i * Z::NW) * 1024, past ? kOutside : fb.at(i, lb), buf);
      }
    }
  };
  // fragment of 16 rows (of M or N) from r0, half ks of the step
  const auto rows_frag = [&](const unsigned char* s, int r0, int ks) {
    return *reinterpret_cast<const Frag*>(s + (r0 + r16) * kFfStep + (((4 * ks + grp) ^ ff_row_swz(r16)) << 4));
  };
  const auto cols_frag = [&](const unsigned char* s, auto row_bytes, int r0, int ks) {
    constexpr int RB = decltype(row_bytes)::value;
    Frag x;
    if constexpr (E == 2) {
      const int k = 32 * ks + 8 * grp + (r16 >> 2);
      const unsigned char* q = s + k * RB + (((2 * (r0 / 16)) ^ ff_col_swz<T, RB>(k)) << 4) + 8 * (r16 & 3);
      x = ld_tr8p(reinterpret_cast<const __bf16*>(q), reinterpret_cast<const __bf16*>(q + 4 * RB));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int k = 16 * ks + 4 * grp + i;
        x[i] = *reinterpret_cast<const float*>(s + k * RB + (((r0 / 4) ^ ff_col_swz<T, RB>(k)) << 4) + 4 * r16);
      }
    }
    return x;
  };
  f4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f4zero();
  if (s0 < s1) fetch(s0);
  for (int s = s0; s < s1; ++s) {
    ff_landed();
    __syncthreads();
    if (s + 1 < s1) fetch(s + 1);
    const unsigned char *sa = smem + (s & 1) * Z::BUF, *sb = sa + BM * kFfStep;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      Frag a[MT], b[NT];
#pragma unroll
      for (int i = 0; i < MT; ++i)
        a[i] = Z::ACOL ? cols_frag(sa, std::integral_constant<int, BM * E>{}, Z::WM * wm + 16 * i, ks) : rows_frag(sa, Z::WM * wm + 16 * i, ks);
#pragma unroll
      for (int j = 0; j < NT; ++j)
        b[j] = Z::BCOL ? cols_frag(sb, std::integral_constant<int, BN * E>{}, Z::WN * wn + 16 * j, ks) : rows_frag(sb, Z::WN * wn + 16 * j, ks);
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = F::mma(b[j], a[i], acc[i][j]);
    }
  }
  if (!whole) {  // the lanes' registers as they are: 16 bytes a lane and instruction
    const int64_t slot = (int64_t)cut * p.split + part;
    float* to = p.part + slot * (BM * BN) + wave * (Z::WM * Z::WN) + 4 * lane;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) *reinterpret_cast<f4*>(to + (i * NT + j) * 256) = acc[i][j];
    return;
  }
  ff_landed();  // (nothing is under way; said where a path from a load to the barrier is looked for)
  __syncthreads();
  using S = FfStrip<T, FORM, END, BM, BN>;
  static_assert(Z::NW * S::BYTES <= 2 * Z::BUF, "strips in the tiles' place");
  float* stage = reinterpret_cast<float*>(smem + wave * S::BYTES);
  const int64_t n = n0 + S::COLS * wn;
  const auto strip = [&](int i) { return S(m0 + Z::WM * wm + 16 * i, n, lane); };
  if constexpr (END == FF_GRAD) {  // a strip's g and u on their way while the strip before it leaves
    FfPast<T, S> past[2];
    past[0].load(p, strip(0));
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      if (i + 1 < MT) past[(i + 1) & 1].load(p, strip(i + 1));
      ff_leave<T, END, S>(p, acc[i], stage, strip(i), &past[i & 1], lane);
    }
  } else {
#pragma unroll
    for (int i = 0; i < MT; ++i) ff_leave<T, END, S>(p, acc[i], stage, strip(i), nullptr, lane);
  }
}

// The parts of the tiles that were cut, a strip a wave
template <typename T, int FORM, int END, int BM, int BN>
__global__ __launch_bounds__(256) void ff_join_kernel(FfArgs<T> p) {
  using Z = FfTile<T, FORM, END, BM, BN>;
  using S = FfStrip<T, FORM, END, BM, BN>;
  constexpr int STRIPS = Z::NW * Z::MT;
  __shared__ __align__(16) unsigned char stage[4][S::BYTES];
  const int lane = threadIdx.x & 63, w4 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int id = blockIdx.x * 4 + w4, tile = id / STRIPS, strip = id % STRIPS, wave = strip / Z::MT, i = strip % Z::MT;
  int im, in;
  ff_place<T, FORM>(p, p.full + tile, im, in);
  f4 x[Z::NT];
  const float* from = p.part + (int64_t)tile * p.split * (BM * BN) + wave * (Z::WM * Z::WN) + i * Z::NT * 256 + 4 * lane;
#pragma unroll
  for (int j = 0; j < Z::NT; ++j) x[j] = *reinterpret_cast<const f4*>(from + j * 256);
  for (int q = 1; q < p.split; ++q) {
    from += BM * BN;
#pragma unroll
    for (int j = 0; j < Z::NT; ++j) x[j] += *reinterpret_cast<const f4*>(from + j * 256);
  }
  const S s((int64_t)im * BM + Z::WM * (wave / Z::NWN) + 16 * i, (int64_t)in * Z::BNC + S::COLS * (wave % Z::NWN), lane);
  FfPast<T, S> past;
  if constexpr (END == FF_GRAD) past.load(p, s);
  ff_leave<T, END, S>(p, x, reinterpret_cast<float*>(stage[w4]), s, &past, lane);
}

// Few rows of A (up to 16 MT): the weights' way through memory is all there is.  A workgroup takes 16 rows of
// B (FF_GATE: of each of the pair), its eight waves a part of the sum each, AHEAD steps of 64 bytes a row
// on their way at a time.  Loads have four lanes a row (16 address cycles; a row a lane, as the fragments
// have it, takes 64, and took 13.4 us where this takes 11.4:
// one token, F = 5504 pairs of 2048, 4.0 TB/s) and pass through the wave's own place in
// LDS; the waves' sums meet there too, in order.
template <typename T, int END, int MT>
__global__ __launch_bounds__(512) void ff_thin_kernel(FfArgs<T> p) {
  using F = FfType<T>;
  using Frag = typename F::Frag;
  constexpr int P = END == FF_GATE ? 2 : 1, KF = 16 / (int)sizeof(T), KS = 4 * KF;  // elements of a piece, of a step
  // FF_GATE: two workgroups a CU; else it has a workgroup a CU or less
  constexpr int AHEAD = P == 2 ? (MT == 1 ? 3 : MT == 2 ? 2 : 1) : (MT == 1 ? 8 : MT == 2 ? 5 : 3);
  constexpr int NW = 8, OWN = AHEAD * (P + MT) * 1024, ALL = NW * (OWN > P * MT * 1024 ? OWN : P * MT * 1024);
  __shared__ __align__(16) unsigned char smem[ALL];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane >> 2, lq = lane & 3;  // the row and the piece that the lane loads
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int steps = (int)((p.K + KS - 1) / KS), s0 = (int)((int64_t)steps * wave / NW), s1 = (int)((int64_t)steps * (wave + 1) / NW);
  const T *b[P], *a[MT];
#pragma unroll
  for (int q = 0; q < P; ++q) b[q] = p.b[q] + min(n0 + lr, p.N - 1) * p.ldb + KF * lq;
#pragma unroll
  for (int i = 0; i < MT; ++i) a[i] = p.a + min((int64_t)(16 * i + lr), p.M - 1) * p.lda + KF * lq;
  f4 acc[P][MT];
#pragma unroll
  for (int q = 0; q < P; ++q)
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[q][i] = f4zero();
  const u4v zero = {0, 0, 0, 0};
  const auto piece = [&](const T* x, int s) {  // what lies past the sum's end is zero
    const int64_t k = (int64_t)s * KS;
    return s < s1 && k + KF * lq < p.K ? ldg16(x + k) : zero;
  };
  // 16 rows of 64 bytes, pieces exchanged between rows below and from 8: 16 lanes are read at a time, of
  // rows {0-3, 8-11} or {4-7, 12-15} and two neighbouring pieces
  unsigned char* own = smem + wave * OWN;
  const int put = 64 * lr + ((lq ^ (lr >> 3 << 1)) << 4);
  const int get = 64 * (lane & 15) + (((lane >> 4) ^ ((lane >> 3 & 1) << 1)) << 4);
  for (int s = s0; s < s1; s += AHEAD) {
    u4v w[AHEAD][P], x[AHEAD][MT];
#pragma unroll
    for (int v = 0; v < AHEAD; ++v) {
#pragma unroll
      for (int q = 0; q < P; ++q) w[v][q] = piece(b[q], s + v);
#pragma unroll
      for (int i = 0; i < MT; ++i) x[v][i] = piece(a[i], s + v);
    }
    ff_wave_order();
#pragma unroll
    for (int v = 0; v < AHEAD; ++v) {
#pragma unroll
      for (int q = 0; q < P; ++q) sts16(own + (v * (P + MT) + q) * 1024 + put, w[v][q]);
#pragma unroll
      for (int i = 0; i < MT; ++i) sts16(own + (v * (P + MT) + P + i) * 1024 + put, x[v][i]);
    }
    ff_wave_order();
#pragma unroll
    for (int v = 0; v < AHEAD; ++v) {
      const auto frag = [&](int k) { return *reinterpret_cast<const Frag*>(own + (v * (P + MT) + k) * 1024 + get); };
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const Frag f = frag(P + i);
#pragma unroll
        for (int q = 0; q < P; ++q) acc[q][i] = F::mma(frag(q), f, acc[q][i]);
      }
    }
  }
  __syncthreads();
  float(*sum)[P * MT][256] = reinterpret_cast<float(*)[P * MT][256]>(smem);
#pragma unroll
  for (int q = 0; q < P; ++q)
#pragma unroll
    for (int i = 0; i < MT; ++i) *reinterpret_cast<f4*>(&sum[wave][q * MT + i][4 * lane]) = acc[q][i];
  __syncthreads();
  // neighbouring threads, neighbouring columns of C
  for (int e = tid; e < 256 * MT; e += 64 * NW) {
    const int c = e & 15, m = e >> 4, at = 4 * (16 * (c >> 2) + (m & 15)) + (c & 3);
    if (m >= p.M || n0 + c >= p.N) continue;
    float v[P];
#pragma unroll
    for (int q = 0; q < P; ++q) {
      v[q] = sum[0][q * MT + (m >> 4)][at];
      for (int w = 1; w < NW; ++w) v[q] += sum[w][q * MT + (m >> 4)][at];
    }
    T* to = (END == FF_GATE ? p.h : p.c[0]) + (int64_t)m * p.N + n0 + c;
    if constexpr (END == FF_GATE) {
      float act, slope;
      ff_act<false>(p.act, v[0], act, slope);
      v[0] = act * v[1];
    }
    if constexpr (sizeof(T) == 2)
      *reinterpret_cast<__bf16*>(to) = (__bf16)v[0];
    else
      *to = v[0];
  }
}

namespace {

template <typename T>
FfSize ff_size(const FfArgs<T>& a) {
  return {{a.M, a.also.M}, {a.N, a.also.N}, a.K, a.pairs};
}

template <typename T, int FORM, int END, int BM, int BN>
hipError_t ff_go(const FfArgs<T>& a, hipStream_t st) {
  using Z = FfTile<T, FORM, END, BM, BN>;
  const int left = a.tiles - a.full;
  hipLaunchKernelGGL((ff_kernel<T, FORM, END, BM, BN>), dim3((unsigned)(a.full + left * a.split)), dim3(ff_threads(BM)), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && left > 0) {
    hipLaunchKernelGGL((ff_join_kernel<T, FORM, END, BM, BN>), dim3((unsigned)(left * (Z::NW * Z::MT / 4))), dim3(256), 0, st, a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

namespace {
template <typename T, int END, int MT>
hipError_t ff_thin(const FfArgs<T>& a, hipStream_t st) {
  hipLaunchKernelGGL((ff_thin_kernel<T, END, MT>), dim3((unsigned)((a.N + 15) / 16)), dim3(512), 0, st, a);
  return hipGetLastError();
}
}  // namespace

template <typename T, int FORM, int END>
size_t ff_part_bytes(const FfArgs<T>& a) {
  return ff_part_bytes(ff_choose(END, ff_size(a), sizeof(T)));
}

template <typename T, int FORM, int END>
hipError_t launch_ff(FfArgs<T> a, hipStream_t st) {
  if constexpr (FORM == FF_ROWS && END != FF_GRAD)
    if (ff_thin_rows(a.M, a.N, a.K, sizeof(T)) && !a.hid.g) {
      if (a.M <= 16) return ff_thin<T, END, 1>(a, st);
      if (a.M <= 32) return ff_thin<T, END, 2>(a, st);
      return ff_thin<T, END, 4>(a, st);
    }
  const FfPlan q = ff_choose(END, ff_size(a), sizeof(T));
  a.tm = q.tm[0];
  a.tn = q.tn[0];
  a.also.tm = q.tm[1];
  a.also.tn = q.tn[1];
  a.tiles = q.tiles;
  a.full = q.full;
  a.split = q.split;
  if constexpr (sizeof(T) == 2)
    if (q.bm == 256) return ff_go<T, FORM, END, 256, 256>(a, st);
  if (q.bm == 128) return ff_go<T, FORM, END, 128, 128>(a, st);
  return ff_go<T, FORM, END, 64, sizeof(T) == 2 && END == FF_GATE ? 128 : 64>(a, st);
}

#define GDR2_FF_ONE(T, FORM, END)                               \
  template size_t ff_part_bytes<T, FORM, END>(const FfArgs<T>&); \
  template hipError_t launch_ff<T, FORM, END>(FfArgs<T>, hipStream_t);
#define GDR2_FF(T)                  \
  GDR2_FF_ONE(T, FF_ROWS, FF_STORE)  \
  GDR2_FF_ONE(T, FF_ROWS, FF_GATE)   \
  GDR2_FF_ONE(T, FF_MIXED, FF_STORE) \
  GDR2_FF_ONE(T, FF_MIXED, FF_GRAD)  \
  GDR2_FF_ONE(T, FF_COLUMNS, FF_STORE)
GDR2_FF(float)
GDR2_FF(bf16_t)

}  // namespace gdr2

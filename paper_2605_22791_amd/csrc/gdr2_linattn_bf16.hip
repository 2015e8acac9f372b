// Linear attention with a decay for each head, bf16 problems: scans over the chunks of a
// segment with the state in registers.
//
// Forward and backward are one form.  With X, Y (rows of length A) and Z (rows of length
// B) among q, k, v, dout, and a state St (A x B), a chunk gives
//     out_i = f_i X_i St + sum_j P_ij Z_j,     P_ij = D (X_i . Y_j)
//     St   <- exp(G_C) St + sum_j Y_j^T (w_j Z_j)
//   o :  X q, Y k,  Z v;   St = S,     f = exp(G_r), w = exp(G_C - G_s), j <= i, first chunk to last
//   dq:  X do, Y v, Z k;   St = S^T,   as above
//   dv:  X k, Y q,  Z do;  St = dS,    f = exp(G_C - G_s), w = scale exp(G_r), j >= i, last chunk to first
//   dk:  X v, Y do, Z q;   St = dS^T,  as dv
//
// A wave owns 16 columns of B over all of A: its state tiles are the accumulators of the
// update, and split to bf16 they are the A operand of X St as they lie (the K order of that
// product is permuted to the accumulators' rows), so the state never leaves its registers.
// The tiles X, Y, Z go through LDS; the scores of a chunk are shared out over the waves,
// pass through LDS split into two bf16 parts, and meet the same Z fragments that the update
// uses (scaled).
//
// Precision: inputs are exact bf16 operands.  fp32 operands are split: scores and the state
// in products that only feed bf16 outputs into two parts (16 bits, against the outputs' 8);
// the decayed Z of the update, and the state where the decay gradient's sums read the
// product, into three (24 bits).

#include "gdr2_linattn.hpp"
#include "gdr2_bf16.hpp"

namespace gdr2 {

namespace {

struct LaUnit {
  size_t row0;
  int len, seq, slot;
  bool first, last;
};

// Segment `slot`; false past the last one in use (uniform).  Table entries are kept in range
// whatever a workspace holds.
__device__ __forceinline__ bool la_unit(const LaSegs& s, int T, int slot, LaUnit& u) {
  u.slot = slot;
  if (s.off == nullptr) {
    if (slot >= s.nslot) return false;
    const int i = slot % s.nseg;
    u.seq = slot / s.nseg;
    u.row0 = (size_t)u.seq * T + (size_t)i * s.seg_tokens;
    u.len = min(s.seg_tokens, T - i * s.seg_tokens);
    u.first = i == 0;
    u.last = i + 1 == s.nseg;
    return true;
  }
  if (slot >= min(s.nslot, ld_table(s.off, s.nseq))) return false;
  u.seq = (int)min((unsigned)ld_table(s.seq, slot), (unsigned)s.nseq - 1);
  const int t0 = (int)min((unsigned)ld_table(s.t0, slot), (unsigned)T);
  u.row0 = (size_t)t0;
  u.len = max(0, min(ld_table(s.len, slot), min(s.seg_tokens, T - t0)));
  u.first = slot == ld_table(s.off, u.seq);
  u.last = slot + 1 == ld_table(s.off, u.seq + 1);
  return true;
}

// Workgroup b of a grid of (unit, slice): the NS slices of a unit run on one XCD (blocks go to
// the eight XCDs in turn) and share its L2; unit < n.
template <int NS>
__device__ __forceinline__ bool la_slot(int b, int n, int& unit, int& slice) {
  unit = b / (8 * NS) * 8 + b % 8;
  slice = b / 8 % NS;
  return unit < n;
}
template <int NS>
unsigned la_grid(int n) { return (unsigned)((n + 7) / 8 * 8) * NS; }

// ---- decays of a chunk -----------------------------------------------------
// Sums are taken within the blocks of 16 rows in 64 bits, p_r up to and including r, so that
// no factor is a difference of long sums.  Between blocks j < i, D_rs = L_r R_is with
// L_r = exp(p_r) and R_is the rest of the way from s to block i; both are at most 1.
struct alignas(16) LaTab {
  double p[CH];
  float L[CH], R[3][CH], E[CH], T[CH];  // R[i - 1][s]; E: exp(G_r), T: exp(G_C - G_s)
  float eC, pad[3];
};

template <int CTRL>
__device__ __forceinline__ double la_dpp(double x) {
  const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(x), CTRL, 0xF, 0xF, true);
  const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(x), CTRL, 0xF, 0xF, true);
  return __hiloint2double(hi, lo);
}
__device__ __forceinline__ double la_lane(double x, int lane) {
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(x), lane),
                          __builtin_amdgcn_readlane(__double2loint(x), lane));
}
__device__ __forceinline__ float la_ex(double x) { return ex2((float)x * kLog2e); }

// One wave, a row a lane: g the row's log-decay (0 past the chunk's end).
__device__ __forceinline__ void la_tables(float g, LaTab& t, int lane) {
  double p = (double)g;
  p += la_dpp<0x111>(p);  // row_shr 1, 2, 4, 8
  p += la_dpp<0x112>(p);
  p += la_dpp<0x114>(p);
  p += la_dpp<0x118>(p);
  const double b0 = la_lane(p, 15), b1 = la_lane(p, 31), b2 = la_lane(p, 47), b3 = la_lane(p, 63);
  const int i = lane >> 4;
  const double before = i == 0 ? 0.0 : i == 1 ? b0 : i == 2 ? b0 + b1 : b0 + b1 + b2;
  const double after = i == 3 ? 0.0 : i == 2 ? b3 : i == 1 ? b2 + b3 : b1 + b2 + b3;
  const double rest = (i == 0 ? b0 : i == 1 ? b1 : i == 2 ? b2 : b3) - p;
  t.p[lane] = p;
  t.L[lane] = la_ex(p);
  t.E[lane] = la_ex(before + p);
  t.T[lane] = la_ex(rest + after);
  t.R[0][lane] = la_ex(rest);                                     // read for rows of block 0
  t.R[1][lane] = la_ex(rest + (i == 0 ? b1 : 0.0));               // of blocks 0, 1
  t.R[2][lane] = la_ex(rest + (i == 0 ? b1 + b2 : i == 1 ? b2 : 0.0));
  if (lane == 0) t.eC = la_ex(b0 + b1 + b2 + b3);
}

// ---- tiles -----------------------------------------------------------------
// COLS columns of 64 rows, LDS row stride COLS + 8: the 16 rows that a fragment read touches
// start in different banks.
template <int COLS, int NTHR>
struct LaTile {
  static constexpr int LD = COLS + 8, BYTES = CH * LD * 2;
  static constexpr int PR = COLS / 8;                           // 16-byte pieces a row
  static constexpr int NP = (CH * PR + NTHR - 1) / NTHR;        // pieces a thread
  u4v x[NP];
  __device__ __forceinline__ void load(const bf16_t* src, size_t stride, int len, int tid) {
#pragma unroll
    for (int m = 0; m < NP; ++m) {
      const int e = tid + m * NTHR, r = min(e / PR, len - 1);
      if (CH * PR % NTHR == 0 || e < CH * PR) x[m] = ldg16(src + (size_t)r * stride + 8 * (e % PR));
    }
  }
  // rows >= len become zero
  __device__ __forceinline__ void store(__bf16* dst, int len, int tid) const {
#pragma unroll
    for (int m = 0; m < NP; ++m) {
      const int e = tid + m * NTHR, r = e / PR;
      if (CH * PR % NTHR == 0 || e < CH * PR) sts16(dst + r * LD + 8 * (e % PR), r < len ? x[m] : u4v{0, 0, 0, 0});
    }
  }
};

struct Fr3 {
  bf8 hi, mid, lo;
};
__device__ __forceinline__ Fr3 split8x3(const float (&x)[8]) {
  Fr3 f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const __bf16 h = (__bf16)x[e];
    const float r = x[e] - (float)h;
    const __bf16 m = (__bf16)r;
    f.hi[e] = h;
    f.mid[e] = m;
    f.lo[e] = (__bf16)(r - (float)m);
  }
  return f;
}

// X[r][..] fragment in the accumulators' row order: columns k0 + 4 g + (0..3), k0 + 16 + 4 g + (0..3)
__device__ __forceinline__ bf8 ld_rows8(const __bf16* row, int k0, int g) {
  const bf4 a = *reinterpret_cast<const bf4*>(row + k0 + 4 * g), b = *reinterpret_cast<const bf4*>(row + k0 + 16 + 4 * g);
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

constexpr int LS = CH + 8;  // row stride of the score tiles (bf16)

// ---- a wave's state: 16 columns over A rows --------------------------------
template <int A>
struct LaState {
  f4 s[A / 16];  // lane (g, c): rows 16 t + 4 g + u, column c

  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int t = 0; t < A / 16; ++t) s[t] = f4zero();
  }
  // row-major (A, ld), the wave's columns from c0 on; or its transpose, row-major (., A)
  __device__ __forceinline__ void load(const float* src, int ld, int c0, int lane) {
    const int g = lane >> 4, c = lane & 15;
#pragma unroll
    for (int t = 0; t < A / 16; ++t)
#pragma unroll
      for (int u = 0; u < 4; ++u) s[t][u] = src[(size_t)(16 * t + 4 * g + u) * ld + c0 + c];
  }
  __device__ __forceinline__ void load_t(const float* src, int c0, int lane) {
    const int g = lane >> 4, c = lane & 15;
#pragma unroll
    for (int t = 0; t < A / 16; ++t) s[t] = *reinterpret_cast<const f4*>(src + (size_t)(c0 + c) * A + 16 * t + 4 * g);
  }
  __device__ __forceinline__ void store(float* dst, int ld, int c0, int lane) const {
    const int g = lane >> 4, c = lane & 15;
#pragma unroll
    for (int t = 0; t < A / 16; ++t)
#pragma unroll
      for (int u = 0; u < 4; ++u) dst[(size_t)(16 * t + 4 * g + u) * ld + c0 + c] = s[t][u];
  }
  __device__ __forceinline__ void store_t(float* dst, int c0, int lane) const {
    const int g = lane >> 4, c = lane & 15;
#pragma unroll
    for (int t = 0; t < A / 16; ++t) *reinterpret_cast<f4*>(dst + (size_t)(c0 + c) * A + 16 * t + 4 * g) = s[t];
  }

  // acc[i] (columns c0 + 4 g + u of row 16 i + c) = X St, the state split into PARTS
  template <int PARTS>
  __device__ __forceinline__ void read(const __bf16* X, f4 (&acc)[4], int lane) const {
    const int g = lane >> 4, c = lane & 15;
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = f4zero();
#pragma unroll
    for (int p = 0; p < A / 32; ++p) {
      const float x[8] = {s[2 * p][0],     s[2 * p][1],     s[2 * p][2],     s[2 * p][3],
                          s[2 * p + 1][0], s[2 * p + 1][1], s[2 * p + 1][2], s[2 * p + 1][3]};
      bf8 b[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) b[i] = ld_rows8(X + (16 * i + c) * (A + 8), 32 * p, g);
      if constexpr (PARTS == 3) {
        const Fr3 f = split8x3(x);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = mma(f.lo, b[i], acc[i]);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = mma(f.mid, b[i], acc[i]);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = mma(f.hi, b[i], acc[i]);
      } else {
        const Fr f = split8(x);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = mma(f.lo, b[i], acc[i]);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = mma(f.hi, b[i], acc[i]);
      }
    }
  }

  // St <- eC St + Y^T (w Z): z[kb] the wave's Z columns, rows 32 kb + 8 g + e
  __device__ __forceinline__ void update(const __bf16* Y, const bf8 (&z)[2], const float* w, float f, float eC, int lane) {
    const int g = lane >> 4;
    Fr3 d[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      float x[8], wv[8];
      unpack8(z[kb], x);
      ldf8(w + 32 * kb + 8 * g, wv);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= wv[e] * f;
      d[kb] = split8x3(x);
    }
#pragma unroll
    for (int t = 0; t < A / 16; ++t) s[t] *= eC;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int t = 0; t < A / 16; ++t) {
        const bf8 y = ld_tr8(Y, A + 8, 32 * kb, 16 * t, lane);
        s[t] = mma(y, d[kb].lo, s[t]);
        s[t] = mma(y, d[kb].mid, s[t]);
        s[t] = mma(y, d[kb].hi, s[t]);
      }
  }
};

// ---- scores ----------------------------------------------------------------
// One 16 x 16 tile of  sum_a Am[m][a] Bn[n][a]; lane (g, c): rows 4 g + u of Am, row c of Bn
template <int A>
__device__ __forceinline__ f4 la_score(const __bf16* Am, const __bf16* Bn, int m0, int n0, int lane) {
  const int g = lane >> 4, c = lane & 15;
  f4 acc = f4zero();
#pragma unroll
  for (int p = 0; p < A / 32; ++p)
    acc = mma(ld8(Am + (m0 + c) * (A + 8) + 32 * p + 8 * g), ld8(Bn + (n0 + c) * (A + 8) + 32 * p + 8 * g), acc);
  return acc;
}

// Factors D_rs of a tile: ROWS of the lane's four values are s (r = r0 + c, one a lane), or r
// (s = s0 + c).  i, j: the blocks of r and s.
template <bool ROWS_S>
__device__ __forceinline__ f4 la_decay_tile(const LaTab& t, int i, int j, int lane) {
  const int g = lane >> 4, c = lane & 15;
  f4 d;
  if (i != j) {
    if constexpr (ROWS_S) {
      const float l = t.L[16 * i + c];
      d = *reinterpret_cast<const f4*>(&t.R[i - 1][16 * j + 4 * g]) * l;
    } else {
      const float r = t.R[i - 1][16 * j + c];
      d = *reinterpret_cast<const f4*>(&t.L[16 * i + 4 * g]) * r;
    }
  } else {
    const double pc = t.p[16 * i + c];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const double pu = t.p[16 * i + 4 * g + u];
      const bool in = ROWS_S ? 4 * g + u <= c : c <= 4 * g + u;
      d[u] = in ? la_ex(ROWS_S ? pc - pu : pu - pc) : 0.f;
    }
  }
  return d;
}

__device__ __forceinline__ void la_zero_tile(__bf16* P, int r0, int s0, int lane) {
  *reinterpret_cast<bf4*>(P + (r0 + (lane & 15)) * LS + s0 + 4 * (lane >> 4)) = bf4{};
}

// Lower tiles (i, j <= i) in the order in which the waves take them: long rows first.
__device__ __forceinline__ void la_tile_of(int n, int& i, int& j) {
  // 0..9: (3,0) (3,1) (3,2) (3,3) (2,0) (2,1) (2,2) (1,0) (1,1) (0,0)
  i = n < 4 ? 3 : n < 7 ? 2 : n < 9 ? 1 : 0;
  j = n < 4 ? n : n < 7 ? n - 4 : n < 9 ? n - 7 : 0;
}

// out[r][c0 + 4 g + u] of the rows 16 i + c < len
template <class Put>
__device__ __forceinline__ void la_rows_out(const f4 (&acc)[4], int len, int lane, Put&& put) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 16 * i + (lane & 15);
    if (r < len) put(r, acc[i]);
  }
}

}  // namespace

// ---- a segment's own contribution to the state -----------------------------
// N = sum of Y^T (w Z) over the segment, from zero: S (k, v; first chunk to last) or, REV, dS
// (q, dout; last to first).  Not needed of the segment that ends its chain.
template <int DK, int DV, bool REV>
__global__ __launch_bounds__(256) void la_segstate_kernel(LaScanArgs a) {
  constexpr int NS = DV / 64, NTHR = 256;
  using TY = LaTile<DK, NTHR>;
  using TZ = LaTile<64, NTHR>;
  __shared__ __align__(16) unsigned char smem[TY::BYTES + TZ::BYTES];
  __shared__ LaTab tab[2];
  __bf16 *sY = reinterpret_cast<__bf16*>(smem), *sZ = reinterpret_cast<__bf16*>(smem + TY::BYTES);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int H = a.geo.H, HK = H / a.geo.G;
  int unit, slice;
  if (!la_slot<NS>(blockIdx.x, a.segs.nslot * H, unit, slice)) return;
  LaUnit un;
  if (!la_unit(a.segs, a.geo.T, unit / H, un)) return;
  const int h = unit % H, hk = h / a.geo.G;
  const int nc = (un.len + CH - 1) / CH;
  double gs = 0.0;
  LaState<DK> st;
  st.zero();
  const bf16_t* Y = (REV ? a.q : a.k) + (un.row0 * HK + hk) * DK;
  const bf16_t* Z = (REV ? a.dout : a.v) + (un.row0 * H + h) * DV + 64 * slice;
  const auto at = [&](int n) { return REV ? nc - 1 - n : n; };
  const auto rows = [&](int n) { return min(CH, un.len - CH * at(n)); };
  const auto decay = [&](int n) {
    return lane < rows(n) ? la_decay_at(a.geo, un.row0 + CH * at(n) + lane, h) : 0.f;
  };
  if (REV ? un.first : un.last) return;
  TY ty;
  TZ tz;
  const auto fetch = [&](int n) {
    ty.load(Y + (size_t)(CH * at(n)) * HK * DK, (size_t)HK * DK, rows(n), tid);
    tz.load(Z + (size_t)(CH * at(n)) * H * DV, (size_t)H * DV, rows(n), tid);
  };
  float g = 0.f;
  if (nc > 0) {
    fetch(0);
    if (wave == 0) {
      g = decay(0);
      la_tables(g, tab[0], lane);
      gs += (double)g;
    }
    ty.store(sY, rows(0), tid);
    tz.store(sZ, rows(0), tid);
  }
  for (int n = 0; n < nc; ++n) {
    __syncthreads();
    const bool more = n + 1 < nc;
    if (more) {
      fetch(n + 1);
      if (wave == 0) g = decay(n + 1);
    }
    const LaTab& t = tab[n & 1];
    const bf8 z[2] = {ld_tr8(sZ, TZ::LD, 0, 16 * wave, lane), ld_tr8(sZ, TZ::LD, 32, 16 * wave, lane)};
    st.update(sY, z, REV ? t.E : t.T, REV ? a.geo.scale : 1.f, t.eC, lane);
    if (more && wave == 0) {
      la_tables(g, tab[(n + 1) & 1], lane);
      gs += (double)g;
    }
    __syncthreads();
    if (more) {
      ty.store(sY, rows(n + 1), tid);
      tz.store(sZ, rows(n + 1), tid);
    }
  }
  float* N = (REV ? a.dS : a.S) + (size_t)unit * (DK * DV);
  st.store(N, DV, 64 * slice + 16 * wave, lane);
  if (slice == 0 && wave == 0) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) gs += __shfl_xor(gs, o);
    if (lane == 0) a.dec[unit] = la_ex(gs);
  }
}

// The states behind the segments (rev: the gradients before them), in the place of their
// contributions: what the chain's next segment starts from.
__global__ __launch_bounds__(256) void la_segcombine_kernel(LaScanArgs a, int size, int rev) {
  constexpr int AHEAD = 4;
  const int H = a.geo.H, per = size / 1024;
  const int q = blockIdx.x / per, e = ((blockIdx.x % per) * 256 + threadIdx.x) * 4, s = q / H, h = q % H;
  int c0 = s * a.segs.nseg, c1 = c0 + a.segs.nseg;
  if (a.segs.off) {
    c0 = min(max(ld_table(a.segs.off, s), 0), a.segs.nslot);
    c1 = min(max(ld_table(a.segs.off, s + 1), c0), a.segs.nslot);
  }
  const int n = c1 - c0 - 1;  // steps of the chain
  float* N = rev ? a.dS : a.S;
  const float* init = rev ? a.dST : a.S0;
  f4 S = f4zero();
  if (init) S = *reinterpret_cast<const f4*>(init + (size_t)q * size + e);
  for (int i0 = 0; i0 < n; i0 += AHEAD) {
    f4 x[AHEAD];
    float d[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int i = min(i0 + j, n - 1);
      const size_t u = (size_t)(rev ? c1 - 1 - i : c0 + i) * H + h;
      x[j] = *reinterpret_cast<const f4*>(N + u * size + e);
      d[j] = a.dec[u];
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if (i0 + j < n) {
        const size_t u = (size_t)(rev ? c1 - 1 - (i0 + j) : c0 + i0 + j) * H + h;
        S = S * d[j] + x[j];
        *reinterpret_cast<f4*>(N + u * size + e) = S;
      }
    }
  }
}

// ---- o, and dq -------------------------------------------------------------
// DQ false: o from q, k, v.  DQ true: dq from dout, v, k, with a_r and S at the anchors.
template <int DK, int DV, bool DQ>
struct LaFwdCfg {
  static constexpr int A = DQ ? DV : DK, B = DQ ? DK : DV, NS = B / 64, NTHR = 256;
  using TX = LaTile<A, NTHR>;
  using TZ = LaTile<64, NTHR>;
  static constexpr int OFF_Y = TX::BYTES, OFF_Z = 2 * TX::BYTES, OFF_P = OFF_Z + TZ::BYTES;
  static constexpr int OFF_T = OFF_P + 2 * CH * LS * 2, OFF_A = OFF_T + 2 * (int)sizeof(LaTab);
  static constexpr int LDS = OFF_A + 4 * CH * 4;
};

template <int DK, int DV, bool DQ>
__device__ void la_forward(const LaScanArgs& a, int block, unsigned char* smem) {
  using C = LaFwdCfg<DK, DV, DQ>;
  constexpr int A = C::A, B = C::B;
  __bf16 *sX = reinterpret_cast<__bf16*>(smem), *sY = reinterpret_cast<__bf16*>(smem + C::OFF_Y);
  __bf16 *sZ = reinterpret_cast<__bf16*>(smem + C::OFF_Z), *sPh = reinterpret_cast<__bf16*>(smem + C::OFF_P);
  __bf16* sPl = sPh + CH * LS;
  LaTab* tab = reinterpret_cast<LaTab*>(smem + C::OFF_T);
  float* sA = reinterpret_cast<float*>(smem + C::OFF_A);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, c = lane & 15;
  const int H = a.geo.H, HK = H / a.geo.G;
  int unit, slice;
  if (!la_slot<C::NS>(block, a.segs.nslot * H, unit, slice)) return;
  LaUnit un;
  if (!la_unit(a.segs, a.geo.T, unit / H, un)) return;
  const int h = unit % H, hk = h / a.geo.G, nc = (un.len + CH - 1) / CH;
  const int b0 = 64 * slice + 16 * wave;  // the wave's columns
  const size_t sk = (size_t)HK * DK, sv = (size_t)H * DV;
  const bf16_t *k0 = a.k + (un.row0 * HK + hk) * DK, *v0 = a.v + (un.row0 * H + h) * DV;
  const bf16_t* q0 = a.q + (un.row0 * HK + hk) * DK;
  const bf16_t *X = DQ ? a.dout + (un.row0 * H + h) * DV : q0, *Y = DQ ? v0 : k0, *Z = (DQ ? k0 : v0) + 64 * slice;
  const size_t sx = DQ ? sv : sk, sy = sx, sz = DQ ? sk : sv;
  const auto rows = [&](int n) { return min(CH, un.len - CH * n); };
  const auto decay = [&](int n) { return lane < rows(n) ? la_decay_at(a.geo, un.row0 + CH * n + lane, h) : 0.f; };

  LaState<A> st;
  {
    const float* init = un.first ? (a.S0 ? a.S0 + ((size_t)un.seq * H + h) * (DK * DV) : nullptr)
                                 : a.S + ((size_t)unit - H) * (DK * DV);
    if (init == nullptr)
      st.zero();
    else if (DQ)
      st.load_t(init, b0, lane);
    else
      st.load(init, DV, b0, lane);
  }
  typename C::TX tx, ty;
  typename C::TZ tz;
  const auto fetch = [&](int n) {
    tx.load(X + (size_t)(CH * n) * sx, sx, rows(n), tid);
    ty.load(Y + (size_t)(CH * n) * sy, sy, rows(n), tid);
    tz.load(Z + (size_t)(CH * n) * sz, sz, rows(n), tid);
  };
  const auto settle = [&](int n) {
    tx.store(sX, rows(n), tid);
    ty.store(sY, rows(n), tid);
    tz.store(sZ, rows(n), tid);
  };
  float gd = 0.f;
  if (nc > 0) {
    fetch(0);
    if (wave == 0) la_tables(decay(0), tab[0], lane);
    if (wave == 1) {  // the tiles above the diagonal that a product of 32 rows meets
      la_zero_tile(sPh, 0, 16, lane);
      la_zero_tile(sPl, 0, 16, lane);
      la_zero_tile(sPh, 32, 48, lane);
      la_zero_tile(sPl, 32, 48, lane);
    }
    settle(0);
  }
  for (int n = 0; n < nc; ++n) {
    __syncthreads();
    const bool more = n + 1 < nc;
    const LaTab& t = tab[n & 1];
    const int len = rows(n);
    if (more) {
      fetch(n + 1);
      if (wave == 0) gd = decay(n + 1);
    }
    // scores, P[r][s], four s a lane
    for (int m = wave; m < 10; m += 4) {
      int i, j;
      la_tile_of(m, i, j);
      f4 x = la_score<A>(sY, sX, 16 * j, 16 * i, lane);
      x *= la_decay_tile<true>(t, i, j, lane);
      const int at = (16 * i + c) * LS + 16 * j + 4 * g;
      st4split(sPh + at, sPl + at, x);
    }
    bf4 qv[4];
    if constexpr (DQ) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        qv[i] = *reinterpret_cast<const bf4*>(q0 + (size_t)(CH * n + min(16 * i + c, len - 1)) * sk + b0 + 4 * g);
    }
    __syncthreads();
    f4 acc[4];
    st.template read<DQ ? 3 : 2>(sX, acc, lane);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] *= t.E[16 * i + c];
    if constexpr (DQ) {
      // a_r over the wave's columns
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float x = 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u) x += acc[i][u] * (float)qv[i][u];
        x += row_partner16(x, (lane & 16) != 0);
        x += row_partner32(x, lane >= 32);
        if (g == 0) sA[wave * CH + 16 * i + c] = x;
      }
    }
    const bf8 z[2] = {ld_tr8(sZ, C::TZ::LD, 0, 16 * wave, lane), ld_tr8(sZ, C::TZ::LD, 32, 16 * wave, lane)};
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 2 * kb; i < 4; ++i) {
        acc[i] = mma(z[kb], ld8(sPl + (16 * i + c) * LS + 32 * kb + 8 * g), acc[i]);
        acc[i] = mma(z[kb], ld8(sPh + (16 * i + c) * LS + 32 * kb + 8 * g), acc[i]);
      }
    st.update(sY, z, t.T, 1.f, t.eC, lane);
    const float sc = a.geo.scale;
    const size_t row = un.row0 + CH * n;
    la_rows_out(acc, len, lane, [&](int r, const f4& x) {
      if constexpr (!DQ) {
        st4(reinterpret_cast<__bf16*>(a.o) + (row + r) * sv + (size_t)h * DV + b0 + 4 * g, sc * x[0], sc * x[1], sc * x[2],
            sc * x[3]);
      } else if (a.Pq) {
        *reinterpret_cast<f4*>(a.Pq + ((row + r) * H + h) * DK + b0 + 4 * g) = x * sc;
      } else {
        st4(reinterpret_cast<__bf16*>(a.dq) + (row + r) * sk + (size_t)hk * DK + b0 + 4 * g, sc * x[0], sc * x[1],
            sc * x[2], sc * x[3]);
      }
    });
    if constexpr (DQ) {
      if ((n + 1) % kLaAnchor == 0 || !more)
        st.store_t(a.aS + ((size_t)unit * a.anchors + n / kLaAnchor) * (DK * DV), b0, lane);
    }
    if (more && wave == 0) la_tables(gd, tab[(n + 1) & 1], lane);
    __syncthreads();
    if constexpr (DQ) {
      if (tid < len)
        a.pa[((size_t)slice * a.geo.B * a.geo.T + row + tid) * H + h] =
            sc * ((sA[tid] + sA[CH + tid]) + (sA[2 * CH + tid] + sA[3 * CH + tid]));
    }
    if (more) settle(n + 1);
  }
  if constexpr (!DQ) {
    if (un.last && a.ST) st.store(a.ST + ((size_t)un.seq * H + h) * (DK * DV), DV, b0, lane);
  }
}

template <int DK, int DV>
__global__ __launch_bounds__(256) void la_scan_fwd_kernel(LaScanArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  la_forward<DK, DV, false>(a, blockIdx.x, smem);
}
template <int DK, int DV>
__global__ __launch_bounds__(256) void la_scan_dq_kernel(LaScanArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  la_forward<DK, DV, true>(a, blockIdx.x, smem);
}

// ---- dk and dv -------------------------------------------------------------
// A workgroup takes a slice of dv's columns (its first NWV waves) and one of dk's; both read
// the same four tiles.
template <int DK, int DV>
struct LaRevCfg {
  static constexpr int NS = (DK > DV ? DK : DV) / 64;
  static constexpr int BV = DV / NS, BK = DK / NS, NWV = BV / 16, NWK = BK / 16, NW = NWV + NWK, NTHR = 64 * NW;
  using TK = LaTile<DK, NTHR>;
  using TV = LaTile<DV, NTHR>;
  static constexpr int OFF_K = TK::BYTES, OFF_V = 2 * TK::BYTES, OFF_D = OFF_V + TV::BYTES, OFF_P = OFF_D + TV::BYTES;
  static constexpr int PB = CH * LS * 2;  // one plane of scores
  static constexpr int OFF_T = OFF_P + 4 * PB, OFF_W = OFF_T + 2 * (int)sizeof(LaTab);
  static constexpr int LDS = OFF_W + (4 + 4 + 4) * CH * 4;
};

template <int DK, int DV>
__global__ __launch_bounds__((LaRevCfg<DK, DV>::NTHR)) void la_scan_dkv_kernel(LaScanArgs a) {
  using C = LaRevCfg<DK, DV>;
  extern __shared__ __align__(16) unsigned char smem[];
  __bf16 *sQ = reinterpret_cast<__bf16*>(smem), *sK = reinterpret_cast<__bf16*>(smem + C::OFF_K);
  __bf16 *sV = reinterpret_cast<__bf16*>(smem + C::OFF_V), *sD = reinterpret_cast<__bf16*>(smem + C::OFF_D);
  __bf16* sP = reinterpret_cast<__bf16*>(smem + C::OFF_P);  // planes: q k hi, lo; do v hi, lo
  LaTab* tab = reinterpret_cast<LaTab*>(smem + C::OFF_T);
  float* sRow = reinterpret_cast<float*>(smem + C::OFF_W);  // [j][r], [i][s], [wave][s]
  float *sCol = sRow + 4 * CH, *sB = sCol + 4 * CH;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, c = lane & 15;
  const int H = a.geo.H, HK = H / a.geo.G;
  int unit, slice;
  if (!la_slot<C::NS>(blockIdx.x, a.segs.nslot * H, unit, slice)) return;
  LaUnit un;
  if (!la_unit(a.segs, a.geo.T, unit / H, un)) return;
  const int h = unit % H, hk = h / a.geo.G, nc = (un.len + CH - 1) / CH;
  const size_t sk = (size_t)HK * DK, sv = (size_t)H * DV;
  const bf16_t *q0 = a.q + (un.row0 * HK + hk) * DK, *k0 = a.k + (un.row0 * HK + hk) * DK;
  const bf16_t *v0 = a.v + (un.row0 * H + h) * DV, *d0 = a.dout + (un.row0 * H + h) * DV;
  const float scale = a.geo.scale;
  const auto at = [&](int n) { return nc - 1 - n; };
  const auto rows = [&](int n) { return min(CH, un.len - CH * at(n)); };
  const auto decay = [&](int n) {
    return lane < rows(n) ? la_decay_at(a.geo, un.row0 + CH * at(n) + lane, h) : 0.f;
  };
  const bool isv = wave < C::NWV;
  const int b0 = isv ? C::BV * slice + 16 * wave : C::BK * slice + 16 * (wave - C::NWV);

  const float* init = un.last ? (a.dST ? a.dST + ((size_t)un.seq * H + h) * (DK * DV) : nullptr)
                              : a.dS + ((size_t)unit + H) * (DK * DV);
  LaState<DK> sdv;  // dS, columns of Dv (waves of dv)
  LaState<DV> sdk;  // dS^T, columns of Dk (waves of dk)
  if (isv) {
    if (init) sdv.load(init, DV, b0, lane); else sdv.zero();
  } else {
    if (init) sdk.load_t(init, b0, lane); else sdk.zero();
  }
  typename C::TK tq, tk;
  typename C::TV tv, td;
  const auto fetch = [&](int n) {
    const size_t r = CH * at(n);
    tq.load(q0 + r * sk, sk, rows(n), tid);
    tk.load(k0 + r * sk, sk, rows(n), tid);
    tv.load(v0 + r * sv, sv, rows(n), tid);
    td.load(d0 + r * sv, sv, rows(n), tid);
  };
  const auto settle = [&](int n) {
    tq.store(sQ, rows(n), tid);
    tk.store(sK, rows(n), tid);
    tv.store(sV, rows(n), tid);
    td.store(sD, rows(n), tid);
  };
  float gd = 0.f;
  if (nc > 0) {
    fetch(0);
    if (wave == 0) la_tables(decay(0), tab[0], lane);
    if (wave == 1) {
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        la_zero_tile(sP + m * (CH * LS), 16, 0, lane);
        la_zero_tile(sP + m * (CH * LS), 48, 32, lane);
      }
    }
    settle(0);
  }
  for (int n = 0; n < nc; ++n) {
    __syncthreads();
    const bool more = n + 1 < nc;
    const LaTab& t = tab[n & 1];
    const int len = rows(n), cn = at(n);
    const size_t row = un.row0 + CH * cn;
    if (more) {
      fetch(n + 1);
      if (wave == 0) gd = decay(n + 1);
    }
    if ((cn + 1) % kLaAnchor == 0 || n == 0) {  // dS behind this chunk
      if (isv) sdv.store(a.aD + ((size_t)unit * a.anchors + cn / kLaAnchor) * (DK * DV), DV, b0, lane);
    }
    // scores, P[s][r], four r a lane, and the sums of W
    for (int m = wave; m < 10; m += C::NW) {
      int i, j;
      la_tile_of(m, i, j);
      const f4 d = la_decay_tile<false>(t, i, j, lane) * scale;
      const f4 x = la_score<DK>(sQ, sK, 16 * i, 16 * j, lane) * d;
      const f4 y = la_score<DV>(sD, sV, 16 * i, 16 * j, lane);
      const int p = (16 * j + c) * LS + 16 * i + 4 * g;
      st4split(sP + p, sP + CH * LS + p, x);
      st4split(sP + 2 * CH * LS + p, sP + 3 * CH * LS + p, y * d);
      f4 w = x * y;
      if (i == j) {
#pragma unroll
        for (int u = 0; u < 4; ++u) w[u] = c < 4 * g + u ? w[u] : 0.f;
      }
      float col = (w[0] + w[1]) + (w[2] + w[3]);
      col += row_partner16(col, (lane & 16) != 0);
      col += row_partner32(col, lane >= 32);
      if (g == 0) sCol[i * CH + 16 * j + c] = col;
#pragma unroll
      for (int u = 0; u < 4; ++u) w[u] = row_sum(w[u]);
      if (c == 0) *reinterpret_cast<f4*>(&sRow[j * CH + 16 * i + 4 * g]) = w;
    }
    __syncthreads();
    f4 acc[4];
    const __bf16* Ph = sP + (isv ? 0 : 2 * CH * LS);
    const __bf16 *Z = isv ? sD : sQ, *Pl = Ph + CH * LS;
    if (isv)
      sdv.template read<3>(sK, acc, lane);
    else
      sdk.template read<2>(sV, acc, lane);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] *= t.T[16 * i + c];
    if (isv) {
      // b_s over the wave's columns
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bf4 vv = *reinterpret_cast<const bf4*>(sV + (16 * i + c) * C::TV::LD + b0 + 4 * g);
        float x = 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u) x += acc[i][u] * (float)vv[u];
        x += row_partner16(x, (lane & 16) != 0);
        x += row_partner32(x, lane >= 32);
        if (g == 0) sB[wave * CH + 16 * i + c] = x;
      }
    }
    const int ldz = isv ? C::TV::LD : C::TK::LD;
    const bf8 z[2] = {ld_tr8(Z, ldz, 0, b0, lane), ld_tr8(Z, ldz, 32, b0, lane)};
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 2 + 2 * kb; ++i) {
        acc[i] = mma(z[kb], ld8(Pl + (16 * i + c) * LS + 32 * kb + 8 * g), acc[i]);
        acc[i] = mma(z[kb], ld8(Ph + (16 * i + c) * LS + 32 * kb + 8 * g), acc[i]);
      }
    if (isv)
      sdv.update(sQ, z, t.E, scale, t.eC, lane);
    else
      sdk.update(sD, z, t.E, scale, t.eC, lane);
    la_rows_out(acc, len, lane, [&](int r, const f4& x) {
      if (isv)
        st4(reinterpret_cast<__bf16*>(a.dv) + (row + r) * sv + (size_t)h * DV + b0 + 4 * g, x[0], x[1], x[2], x[3]);
      else if (a.Pk)
        *reinterpret_cast<f4*>(a.Pk + ((row + r) * H + h) * DK + b0 + 4 * g) = x;
      else
        st4(reinterpret_cast<__bf16*>(a.dk) + (row + r) * sk + (size_t)hk * DK + b0 + 4 * g, x[0], x[1], x[2], x[3]);
    });
    if (more && wave == 0) la_tables(gd, tab[(n + 1) & 1], lane);
    __syncthreads();
    if (tid < len) {
      float x = 0.f;
#pragma unroll
      for (int w = 0; w < C::NWV; ++w) x += sB[w * CH + tid];
      a.pb[((size_t)slice * a.geo.B * a.geo.T + row + tid) * H + h] = x;
      if (slice == 0) {
        const int blk = tid >> 4;
        float rs = 0.f, cs = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          rs += j <= blk ? sRow[j * CH + tid] : 0.f;
          cs += j >= blk ? sCol[j * CH + tid] : 0.f;
        }
        a.prc[(row + tid) * H + h] = rs - cs;
      }
    }
    if (more) settle(n + 1);
  }
  if (un.first && a.dS0 && isv) sdv.store(a.dS0 + ((size_t)un.seq * H + h) * (DK * DV), DV, b0, lane);
}

// ---- the decays' gradient --------------------------------------------------
// dg_t = <S, dS> behind the last token of the stretch + sum over t' >= t of a + row - b - col,
// in 64 bits; a stretch of up to kLaAnchor chunks a workgroup, a token a thread.
template <int DK, int DV>
__global__ __launch_bounds__(kLaAnchor * CH) void la_dg_kernel(LaScanArgs a) {
  constexpr int NTHR = kLaAnchor * CH, NA = DK / 64, NB = LaRevCfg<DK, DV>::NS;
  __shared__ double part[NTHR / 64], phi[NTHR / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int H = a.geo.H, unit = blockIdx.x / a.anchors, k = blockIdx.x % a.anchors, h = unit % H;
  LaUnit un;
  if (!la_unit(a.segs, a.geo.T, unit / H, un)) return;
  const int t0 = k * NTHR, len = min(NTHR, un.len - t0);
  if (len <= 0) return;
  double x = 0.0;
  const size_t row = un.row0 + t0 + tid, rows = (size_t)a.geo.B * a.geo.T;
  if (tid < len) {
    float pa = 0.f, pb = 0.f;
#pragma unroll
    for (int s = 0; s < NA; ++s) pa += a.pa[(s * rows + row) * H + h];
#pragma unroll
    for (int s = 0; s < NB; ++s) pb += a.pb[(s * rows + row) * H + h];
    x = (double)pa + a.prc[row * H + h] - pb;
  }
  double f = 0.0;
  if (!(un.last && t0 + len == un.len && a.dST == nullptr)) {
    const float *S = a.aS + (size_t)blockIdx.x * (DK * DV), *D = a.aD + (size_t)blockIdx.x * (DK * DV);
    for (int e = 4 * tid; e < DK * DV; e += 4 * NTHR) {
      const float4 p = ld4(S + e), q = ld4(D + e);
      f += (double)(p.x * q.x + p.y * q.y) + (double)(p.z * q.z + p.w * q.w);
    }
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double y = __shfl_down(x, o);
    if (lane + o < 64) x += y;
    f += __shfl_xor(f, o);
  }
  if (lane == 0) {
    part[wave] = x;
    phi[wave] = f;
  }
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int w = 0; w < NTHR / 64; ++w) s += phi[w] + (w > wave ? part[w] : 0.0);
  if (tid < len) a.dg[row * H + h] = (float)(s + x);
}

// ---- segment table of a packed batch ---------------------------------------
// One workgroup, 1024 sequences at a time: a scan of their segment counts, then every
// sequence writes its segments.
__global__ __launch_bounds__(1024) void la_segtable_kernel(const int* cu, LaSegs s, int T, int* t0, int* len, int* seq,
                                                           int* off) {
  __shared__ int wt[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int carry = 0;
  for (int base = 0; base < s.nseq; base += 1024) {
    const int q = base + tid;
    int a = 0, b = 0, n = 0;
    if (q < s.nseq) {
      a = min(max(cu[q], 0), T);
      b = min(max(cu[q + 1], a), T);
      n = max(1, (b - a + s.seg_tokens - 1) / s.seg_tokens);
    }
    int x = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(x, o);
      if (lane >= o) x += y;
    }
    if (lane == 63) wt[wave] = x;
    __syncthreads();
    int before = carry, all = carry;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      before += w < wave ? wt[w] : 0;
      all += wt[w];
    }
    const int at = before + x - n;
    if (q < s.nseq) {
      off[q] = min(at, s.nslot);
      for (int i = 0; i < n && at + i < s.nslot; ++i) {
        t0[at + i] = a + i * s.seg_tokens;
        len[at + i] = min(s.seg_tokens, b - a - i * s.seg_tokens);
        seq[at + i] = q;
      }
    }
    carry = all;
    __syncthreads();
  }
  if (tid == 0) off[s.nseq] = min(carry, s.nslot);
}

// ---- launches --------------------------------------------------------------
namespace {
template <class K>
hipError_t la_launch(K kernel, unsigned grid, unsigned threads, size_t lds, const LaScanArgs& a, hipStream_t st) {
  hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(threads), lds, st, a);
  return hipGetLastError();
}
}  // namespace

template <int DK, int DV>
hipError_t launch_la_segstate(const LaScanArgs& a, bool rev, hipStream_t st) {
  const unsigned grid = la_grid<DV / 64>(a.segs.nslot * a.geo.H);
  if (rev)
    hipLaunchKernelGGL((la_segstate_kernel<DK, DV, true>), dim3(grid), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((la_segstate_kernel<DK, DV, false>), dim3(grid), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_la_segcombine(const LaScanArgs& a, int size, bool rev, hipStream_t st) {
  hipLaunchKernelGGL(la_segcombine_kernel, dim3((unsigned)(a.segs.nseq * a.geo.H * (size / 1024))), dim3(256), 0, st, a, size,
                     rev ? 1 : 0);
  return hipGetLastError();
}

template <int DK, int DV>
hipError_t launch_la_scan_fwd(const LaScanArgs& a, hipStream_t st) {
  using C = LaFwdCfg<DK, DV, false>;
  return la_launch(la_scan_fwd_kernel<DK, DV>, la_grid<C::NS>(a.segs.nslot * a.geo.H), 256, C::LDS, a, st);
}

template <int DK, int DV>
hipError_t launch_la_scan_bwd(const LaScanArgs& a, hipStream_t st) {
  using CQ = LaFwdCfg<DK, DV, true>;
  using CR = LaRevCfg<DK, DV>;
  const int units = a.segs.nslot * a.geo.H;
  hipError_t e = la_launch(la_scan_dq_kernel<DK, DV>, la_grid<CQ::NS>(units), 256, CQ::LDS, a, st);
  if (e == hipSuccess) e = la_launch(la_scan_dkv_kernel<DK, DV>, la_grid<CR::NS>(units), CR::NTHR, CR::LDS, a, st);
  if (e == hipSuccess) {
    hipLaunchKernelGGL((la_dg_kernel<DK, DV>), dim3((unsigned)(units * a.anchors)), dim3(kLaAnchor * CH), 0, st, a);
    e = hipGetLastError();
  }
  return e;
}

hipError_t launch_la_segtable(const int* cu, const LaSegs& s, int T, int* t0, int* len, int* seq, int* off, hipStream_t st) {
  hipLaunchKernelGGL(la_segtable_kernel, dim3(1), dim3(1024), 0, st, cu, s, T, t0, len, seq, off);
  return hipGetLastError();
}

#define GDR2_LA_SCAN(DK, DV)                                                          \
  template hipError_t launch_la_segstate<DK, DV>(const LaScanArgs&, bool, hipStream_t); \
  template hipError_t launch_la_scan_fwd<DK, DV>(const LaScanArgs&, hipStream_t);       \
  template hipError_t launch_la_scan_bwd<DK, DV>(const LaScanArgs&, hipStream_t);
GDR2_LA_SCAN(64, 64)
GDR2_LA_SCAN(64, 128)
GDR2_LA_SCAN(128, 64)
GDR2_LA_SCAN(128, 128)

}  // namespace gdr2

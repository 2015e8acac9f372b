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
  float L[CH], R[3][CH], E[CH], T[CH];  // R[i - 1][s]; E: exp(G_r) (scale exp(G_r) in the reverse scans), T: exp(G_C - G_s)
  float eC, pad[3];
};

template <int CTRL>
__device__ __forceinline__ double la_dpp(double x) {
  const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(x), CTRL, 0xF, 0xF, true);
  const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(x), CTRL, 0xF, 0xF, true);
  return __hiloint2double(hi, lo);
}
__device__ __forceinline__ float la_lanef(float x, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane));
}
__device__ __forceinline__ float la_ex(float x) { return ex2(x * kLog2e); }

// One wave, a row a lane: g the row's raw log-decay; rows past the chunk's end do not decay.
// E is multiplied by scale.  Returns the row's log-decay.
__device__ __forceinline__ float la_tables(float g, int rows, LaTab& t, int lane, float scale) {
  const float g0 = lane < rows ? (g < kLaForget ? kLaForget : g) : 0.f;
  double p = (double)g0;
  p += la_dpp<0x111>(p);  // row_shr 1, 2, 4, 8
  p += la_dpp<0x112>(p);
  p += la_dpp<0x114>(p);
  p += la_dpp<0x118>(p);
  const double all = la_dpp<0x15F>(p);  // the block's last row
  const float pf = (float)p, rest = (float)(all - p), b = (float)all;
  const float b0 = la_lanef(b, 0), b1 = la_lanef(b, 16), b2 = la_lanef(b, 32), b3 = la_lanef(b, 48);
  const int i = lane >> 4;
  const float before = (i > 0 ? b0 : 0.f) + (i > 1 ? b1 : 0.f) + (i > 2 ? b2 : 0.f);
  const float m1 = i < 1 ? b1 : 0.f, m2 = i < 2 ? b2 : 0.f, m3 = i < 3 ? b3 : 0.f;
  const float r1 = rest, r2 = r1 + m1, r3 = r2 + m2;  // from the row to the blocks behind its own
  t.p[lane] = p;
  t.L[lane] = la_ex(pf);
  t.E[lane] = scale * la_ex(before + pf);
  t.T[lane] = la_ex(r3 + m3);
  t.R[0][lane] = la_ex(r1);  // to block 1: read for rows of block 0
  t.R[1][lane] = la_ex(r2);  // to block 2: of blocks 0, 1
  t.R[2][lane] = la_ex(r3);
  if (lane == 0) t.eC = la_ex((b0 + b1) + (b2 + b3));
  return g0;
}

// ---- memory ----------------------------------------------------------------
// The rows of a chunk as a buffer: a load past its last row gives zero, a store there is
// dropped, and a lane's offsets are the same for every chunk (the base moves in scalar
// registers).
typedef unsigned u2v __attribute__((ext_vector_type(2)));
__device__ __forceinline__ __amdgpu_buffer_rsrc_t la_buf(const void* p, size_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)(unsigned)bytes, 0x00020000);
}
// byte offset of (row, byte b) under a row stride; one past 32 bits stays out of range
__device__ __forceinline__ unsigned la_off(int row, size_t stride, int b) {
  const size_t x = (size_t)row * stride + b;
  return x < 0xfffffff0u ? (unsigned)x : 0xfffffff0u;
}
__device__ __forceinline__ void la_put4(__amdgpu_buffer_rsrc_t buf, unsigned at, const f4& x) {
  bf4 v;
  v[0] = (__bf16)x[0], v[1] = (__bf16)x[1], v[2] = (__bf16)x[2], v[3] = (__bf16)x[3];
  __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u2v, v), buf, at, 0, 0);
}
__device__ __forceinline__ void la_putf(__amdgpu_buffer_rsrc_t buf, unsigned at, const f4& x) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4v, x), buf, at, 0, 0);
}

// The log-decay of row `lane` of a chunk as it lies in memory: loaded a step before it is
// needed, and looked at only there.
struct LaDecays {
  const char* base;
  size_t stride;  // bytes a row; 0: one for every token
  unsigned off;
  __device__ __forceinline__ LaDecays(const LaGeo& a, size_t row0, int h, int lane) {
    base = reinterpret_cast<const char*>(a.per_head ? a.g + h : a.g + row0 * a.H + h);
    stride = a.per_head ? 0 : (size_t)a.H * 4;
    off = la_off(lane, stride, 0);
  }
  __device__ __forceinline__ float load(int chunk, int rows) const {
    const auto buf = la_buf(base + (size_t)chunk * CH * stride, (size_t)(rows - 1) * stride + 4);
    return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(buf, off, 0, 0));
  }
};

// ---- tiles -----------------------------------------------------------------
// COLS columns of 64 rows.  LDS row stride COLS + 8: the 16 rows that a fragment read touches
// start in different banks; + 16 where the transposed reads are the most (four rows of 32
// bytes at a time: 4 banks apart they would overlap).
template <int COLS, int NTHR, int PAD = 8>
struct LaTile {
  static constexpr int LD = COLS + PAD, BYTES = CH * LD * 2;
  static constexpr int PR = COLS / 8;                           // 16-byte pieces a row
  static constexpr int NP = (CH * PR + NTHR - 1) / NTHR;        // pieces a thread
  u4v x[NP];
  struct Off {  // a thread's pieces in memory
    unsigned at[NP];
    __device__ __forceinline__ Off(size_t stride, int tid) {  // stride: bytes a row
#pragma unroll
      for (int m = 0; m < NP; ++m) {
        const int e = tid + m * NTHR;
        at[m] = e < CH * PR ? la_off(e / PR, stride, 16 * (e % PR)) : 0xfffffff0u;
      }
    }
  };
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t buf, const Off& off) {
#pragma unroll
    for (int m = 0; m < NP; ++m) x[m] = __builtin_amdgcn_raw_buffer_load_b128(buf, off.at[m], 0, 0);
  }
  __device__ __forceinline__ void store(__bf16* dst, int tid) const {
#pragma unroll
    for (int m = 0; m < NP; ++m) {
      const int e = tid + m * NTHR;
      if (CH * PR % NTHR == 0 || e < CH * PR) sts16(dst + e / PR * LD + 8 * (e % PR), x[m]);
    }
  }
};

// ---- splits ----------------------------------------------------------------
// x = hi + lo (+ lower), bf16 parts of two values at a time.  What a part leaves is
// x - hi, exact in fp32, and one v_dot2_f32_bf16 of the packed parts with (-1, 0) or
// (0, -1) forms it from the pair (unpacking first takes two instructions; a scan's vector
// instructions are what bounds it).
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ bf2 la_pick(unsigned bits) {
  // in a register: as an immediate, -1.0 would be the fp32 constant, whose low half is 0
  asm("" : "+s"(bits));
  return __builtin_bit_cast(bf2, bits);
}
__device__ __forceinline__ bf2 la_part(float a, float b) {
  bf2 h;
  h[0] = (__bf16)a;
  h[1] = (__bf16)b;
  return h;
}
__device__ __forceinline__ void la_left(bf2 h, float& a, float& b) {
  a = __builtin_amdgcn_fdot2_f32_bf16(h, la_pick(0x0000bf80u), a, false);
  b = __builtin_amdgcn_fdot2_f32_bf16(h, la_pick(0xbf800000u), b, false);
}
template <int PARTS>
struct LaFr {
  bf8 p[PARTS];  // largest first
};
template <int PARTS>
__device__ __forceinline__ LaFr<PARTS> la_split8(const float (&x)[8]) {
  LaFr<PARTS> f;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    float a = x[e], b = x[e + 1];
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
      const bf2 h = la_part(a, b);
      f.p[k][e] = h[0];
      f.p[k][e + 1] = h[1];
      if (k + 1 < PARTS) la_left(h, a, b);
    }
  }
  return f;
}
__device__ __forceinline__ void la_split4(__bf16* hi, __bf16* lo, const f4& x) {
  float r[4] = {x[0], x[1], x[2], x[3]};
  const bf2 h0 = la_part(r[0], r[1]), h1 = la_part(r[2], r[3]);
  la_left(h0, r[0], r[1]);
  la_left(h1, r[2], r[3]);
  const bf2 l0 = la_part(r[0], r[1]), l1 = la_part(r[2], r[3]);
  *reinterpret_cast<bf4*>(hi) = bf4{h0[0], h0[1], h1[0], h1[1]};
  *reinterpret_cast<bf4*>(lo) = bf4{l0[0], l0[1], l1[0], l1[1]};
}

// X[r][..] fragment in the accumulators' row order: columns k0 + 4 g + (0..3), k0 + 16 + 4 g + (0..3)
__device__ __forceinline__ bf8 ld_rows8(const __bf16* row, int k0, int g) {
  const bf4 a = *reinterpret_cast<const bf4*>(row + k0 + 4 * g), b = *reinterpret_cast<const bf4*>(row + k0 + 16 + 4 * g);
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

constexpr int LS = CH + 8;  // row stride of the score tiles (bf16)

// ---- a wave's state: 16 columns over half of the A rows ---------------------
// The two waves of a column group take the rows a0 .. a0 + A / 2 each: two waves a SIMD, which
// hide each other's latencies (a wave with all of A: 325 us for the forward of B = 8, T = 4096,
// 16 heads of 128 x 128, 10.8 thousand cycles a chunk of which 2.5 thousand issue).
template <int A>
struct LaState {
  static constexpr int AH = A / 2;
  f4 s[AH / 16];  // lane (g, c): rows a0 + 16 t + 4 g + u, column c
  int a0;

  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int t = 0; t < AH / 16; ++t) s[t] = f4zero();
  }
  // row-major (A, ld), the wave's columns from c0 on; or its transpose, row-major (., A)
  __device__ __forceinline__ void load(const float* src, int ld, int c0, int lane) {
    const int g = lane >> 4, c = lane & 15;
#pragma unroll
    for (int t = 0; t < AH / 16; ++t)
#pragma unroll
      for (int u = 0; u < 4; ++u) s[t][u] = src[(size_t)(a0 + 16 * t + 4 * g + u) * ld + c0 + c];
  }
  __device__ __forceinline__ void load_t(const float* src, int c0, int lane) {
    const int g = lane >> 4, c = lane & 15;
#pragma unroll
    for (int t = 0; t < AH / 16; ++t)
      s[t] = *reinterpret_cast<const f4*>(src + (size_t)(c0 + c) * A + a0 + 16 * t + 4 * g);
  }
  __device__ __forceinline__ void store(float* dst, int ld, int c0, int lane) const {
    const int g = lane >> 4, c = lane & 15;
#pragma unroll
    for (int t = 0; t < AH / 16; ++t)
#pragma unroll
      for (int u = 0; u < 4; ++u) dst[(size_t)(a0 + 16 * t + 4 * g + u) * ld + c0 + c] = s[t][u];
  }
  __device__ __forceinline__ void store_t(float* dst, int c0, int lane) const {
    const int g = lane >> 4, c = lane & 15;
#pragma unroll
    for (int t = 0; t < AH / 16; ++t)
      *reinterpret_cast<f4*>(dst + (size_t)(c0 + c) * A + a0 + 16 * t + 4 * g) = s[t];
  }

  // acc[i] (columns c0 + 4 g + u of row 16 i + c) = X St over the wave's rows, the state split into PARTS
  template <int PARTS>
  __device__ __forceinline__ void read(const __bf16* X, int ld, f4 (&acc)[4], int lane) const {
    const int g = lane >> 4, c = lane & 15;
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = f4zero();
#pragma unroll
    for (int p = 0; p < AH / 32; ++p) {
      const float x[8] = {s[2 * p][0],     s[2 * p][1],     s[2 * p][2],     s[2 * p][3],
                          s[2 * p + 1][0], s[2 * p + 1][1], s[2 * p + 1][2], s[2 * p + 1][3]};
      bf8 b[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) b[i] = ld_rows8(X + (16 * i + c) * ld + a0, 32 * p, g);
      const LaFr<PARTS> f = la_split8<PARTS>(x);
#pragma unroll
      for (int k = PARTS - 1; k >= 0; --k)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = mma(f.p[k], b[i], acc[i]);
    }
  }

  // St <- eC St + Y^T (w Z): z[kb] the wave's Z columns, rows 32 kb + 8 g + e
  __device__ __forceinline__ void update(const __bf16* Y, int ld, const bf8 (&z)[2], const float* w, float eC, int lane) {
    const int g = lane >> 4;
    LaFr<3> d[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      float x[8], wv[8];
      unpack8(z[kb], x);
      ldf8(w + 32 * kb + 8 * g, wv);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= wv[e];
      d[kb] = la_split8<3>(x);
    }
#pragma unroll
    for (int t = 0; t < AH / 16; ++t) s[t] *= eC;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      bf8 y[AH / 16];
#pragma unroll
      for (int t = 0; t < AH / 16; ++t) y[t] = ld_tr8(Y, ld, 32 * kb, a0 + 16 * t, lane);
#pragma unroll
      for (int k = 2; k >= 0; --k)
#pragma unroll
        for (int t = 0; t < AH / 16; ++t) s[t] = mma(y[t], d[kb].p[k], s[t]);
    }
  }
};

// The two halves' X St meet in LDS: of the four row tiles the wave of half 0 keeps 0 and 3, the
// other 1 and 2 (the same number of score tiles each way), and hands over the rest; 512 floats a wave.
__device__ __forceinline__ void la_hand(const f4 (&acc)[4], bool hf, float* mine, int lane) {
  *reinterpret_cast<f4*>(mine + 4 * lane) = hf ? acc[0] : acc[1];
  *reinterpret_cast<f4*>(mine + 256 + 4 * lane) = hf ? acc[3] : acc[2];
}
__device__ __forceinline__ void la_take(const f4 (&acc)[4], bool hf, const float* other, f4 (&own)[2], int lane) {
  own[0] = (hf ? acc[1] : acc[0]) + *reinterpret_cast<const f4*>(other + 4 * lane);
  own[1] = (hf ? acc[2] : acc[3]) + *reinterpret_cast<const f4*>(other + 256 + 4 * lane);
}

// ---- scores ----------------------------------------------------------------
// One 16 x 16 tile of  sum_a Am[m][a] Bn[n][a]; lane (g, c): rows 4 g + u of Am, row c of Bn
template <int A, int LDA, int LDB>
__device__ __forceinline__ f4 la_score(const __bf16* Am, const __bf16* Bn, int m0, int n0, int lane) {
  const int g = lane >> 4, c = lane & 15;
  f4 x = f4zero();
#pragma unroll
  for (int p = 0; p < A / 32; ++p)
    x = mma(ld8(Am + (m0 + c) * LDA + 32 * p + 8 * g), ld8(Bn + (n0 + c) * LDB + 32 * p + 8 * g), x);
  return x;
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
      const float e = la_ex((float)(ROWS_S ? pc - pu : pu - pc));
      d[u] = (ROWS_S ? 4 * g + u <= c : c <= 4 * g + u) ? e : 0.f;
    }
  }
  return d;
}

__device__ __forceinline__ void la_zero_tile(__bf16* P, int r0, int s0, int lane) {
  *reinterpret_cast<bf4*>(P + (r0 + (lane & 15)) * LS + s0 + 4 * (lane >> 4)) = bf4{};
}

// The lower tiles (i, j <= i) of a chunk's scores over the waves.  Eight waves: four take one on
// the diagonal (dearer), three two off it, the last one the decays of the next chunk.  Twelve or
// sixteen: one each, and the last wave the decays.
template <int NW>
__device__ __forceinline__ int la_tiles(int wave) {
  return NW == 8 ? (wave < 4 ? 1 : wave < 7 ? 2 : 0) : (wave < 10 ? 1 : 0);
}
template <int NW>
__device__ __forceinline__ void la_tile_of(int wave, int m, int& i, int& j) {
  // (0,0) (1,1) (2,2) (3,3) (3,0) (3,1) (3,2) (2,0) (2,1) (1,0)
  const int n = NW == 8 && wave >= 4 ? 2 * wave - 4 + m : wave;
  i = n < 4 ? n : n < 7 ? 3 : n < 9 ? 2 : 1;
  j = n < 4 ? n : n < 7 ? n - 4 : n < 9 ? n - 7 : 0;
}

}  // namespace

// ---- a segment's own contribution to the state -----------------------------
// N = sum of Y^T (w Z) over the segment, from zero: S (k, v; first chunk to last) or, REV, dS
// (q, dout; last to first).  Not needed of the segment that ends its chain.
template <int DK, int DV, bool REV>
__global__ __launch_bounds__(512) void la_segstate_kernel(LaScanArgs a) {
  constexpr int NS = DV / 64, NTHR = 512, TW = 7;
  using TY = LaTile<DK, NTHR, 16>;
  using TZ = LaTile<64, NTHR>;
  constexpr int BUF = TY::BYTES + TZ::BYTES;
  __shared__ __align__(16) unsigned char smem[2 * BUF];
  __shared__ LaTab tab[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int H = a.geo.H, HK = H / a.geo.G;
  int unit, slice;
  if (!la_slot<NS>(blockIdx.x, a.segs.nslot * H, unit, slice)) return;
  LaUnit un;
  if (!la_unit(a.segs, a.geo.T, unit / H, un)) return;
  if (REV ? un.first : un.last) return;
  const int h = unit % H, hk = h / a.geo.G;
  const int nc = (un.len + CH - 1) / CH;
  const size_t sy = (size_t)HK * DK * 2, sz = (size_t)H * DV * 2;  // bytes a row
  const bf16_t* Y = (REV ? a.q : a.k) + (un.row0 * HK + hk) * DK;
  const bf16_t* Z = (REV ? a.dout : a.v) + (un.row0 * H + h) * DV + 64 * slice;
  const float scale = REV ? a.geo.scale : 1.f;
  const auto at = [&](int n) { return REV ? nc - 1 - n : n; };
  const auto rows = [&](int n) { return min(CH, un.len - CH * at(n)); };
  const LaDecays decays(a.geo, un.row0, h, lane);
  const auto decay = [&](int n) { return decays.load(at(n), rows(n)); };
  const auto sYb = [&](int n) { return reinterpret_cast<__bf16*>(smem + (n & 1) * BUF); };
  const auto sZb = [&](int n) { return reinterpret_cast<__bf16*>(smem + (n & 1) * BUF + TY::BYTES); };
  double gs = 0.0;
  LaState<DK> st;
  st.a0 = wave >= 4 ? DK / 2 : 0;
  st.zero();
  TY ty;
  TZ tz;
  const typename TY::Off oy(sy, tid);
  const typename TZ::Off oz(sz, tid);
  const auto fetch = [&](int n) {
    ty.load(la_buf(reinterpret_cast<const char*>(Y) + (size_t)(CH * at(n)) * sy, (rows(n) - 1) * sy + 2 * DK), oy);
    tz.load(la_buf(reinterpret_cast<const char*>(Z) + (size_t)(CH * at(n)) * sz, (rows(n) - 1) * sz + 128), oz);
  };
  float graw = 0.f;
  if (nc > 0) {
    fetch(0);
    if (wave == TW) {
      gs += (double)la_tables(decay(0), rows(0), tab[0], lane, scale);
      if (nc > 1) graw = decay(1);
    }
    ty.store(sYb(0), tid);
    tz.store(sZb(0), tid);
  }
  for (int n = 0; n < nc; ++n) {
    __syncthreads();
    const bool more = n + 1 < nc;
    if (more) {
      fetch(n + 1);
      if (wave == TW) {
        gs += (double)la_tables(graw, rows(n + 1), tab[(n + 1) & 1], lane, scale);
        if (n + 2 < nc) graw = decay(n + 2);
      }
    }
    const LaTab& t = tab[n & 1];
    const __bf16* sZ = sZb(n);
    const int c0 = 16 * (wave & 3);
    const bf8 z[2] = {ld_tr8(sZ, TZ::LD, 0, c0, lane), ld_tr8(sZ, TZ::LD, 32, c0, lane)};
    st.update(sYb(n), TY::LD, z, REV ? t.E : t.T, t.eC, lane);
    if (more) {
      ty.store(sYb(n + 1), tid);
      tz.store(sZb(n + 1), tid);
    }
  }
  float* N = (REV ? a.dS : a.S) + (size_t)unit * (DK * DV);
  st.store(N, DV, 64 * slice + 16 * (wave & 3), lane);
  if (slice == 0 && wave == TW) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) gs += __shfl_xor(gs, o);
    if (lane == 0) a.dec[unit] = la_ex((float)gs);
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
// Two barriers a chunk: the tiles of the next one go to LDS beside this one's.
template <int DK, int DV, bool DQ>
struct LaFwdCfg {
  static constexpr int A = DQ ? DV : DK, B = DQ ? DK : DV, NS = B / 64, NTHR = 512;
  using TX = LaTile<A, NTHR>;
  using TY = LaTile<A, NTHR, 16>;
  using TZ = LaTile<64, NTHR>;
  static constexpr int OFF_Y = TX::BYTES, OFF_Z = OFF_Y + TY::BYTES, BUF = OFF_Z + TZ::BYTES;
  static constexpr int OFF_P = 2 * BUF, OFF_T = OFF_P + 2 * CH * LS * 2, OFF_X = OFF_T + 2 * (int)sizeof(LaTab);
  static constexpr int OFF_A = OFF_X + 8 * 512 * 4;
  static constexpr int LDS = OFF_A + (DQ ? 8 * CH * 4 : 0);
  static_assert(LDS <= 160 * 1024, "LDS budget");
};

template <int DK, int DV, bool DQ>
__device__ __forceinline__ void la_forward(const LaScanArgs& a, int block, unsigned char* smem) {
  using C = LaFwdCfg<DK, DV, DQ>;
  constexpr int A = C::A, B = C::B, TW = 7;
  __bf16 *sPh = reinterpret_cast<__bf16*>(smem + C::OFF_P), *sPl = sPh + CH * LS;
  LaTab* tab = reinterpret_cast<LaTab*>(smem + C::OFF_T);
  float *sEx = reinterpret_cast<float*>(smem + C::OFF_X), *sA = reinterpret_cast<float*>(smem + C::OFF_A);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, c = lane & 15;
  const bool hf = wave >= 4;
  const int H = a.geo.H, HK = H / a.geo.G;
  int unit, slice;
  if (!la_slot<C::NS>(block, a.segs.nslot * H, unit, slice)) return;
  LaUnit un;
  if (!la_unit(a.segs, a.geo.T, unit / H, un)) return;
  const int h = unit % H, hk = h / a.geo.G, nc = (un.len + CH - 1) / CH;
  const int b0 = 64 * slice + 16 * (wave & 3);                     // the wave's columns
  const size_t sk = (size_t)HK * DK * 2, sv = (size_t)H * DV * 2;  // bytes a row
  const bf16_t *k0 = a.k + (un.row0 * HK + hk) * DK, *v0 = a.v + (un.row0 * H + h) * DV;
  const bf16_t* q0 = a.q + (un.row0 * HK + hk) * DK;
  const bf16_t *X = DQ ? a.dout + (un.row0 * H + h) * DV : q0, *Y = DQ ? v0 : k0, *Z = (DQ ? k0 : v0) + 64 * slice;
  const size_t sx = DQ ? sv : sk, sz = DQ ? sk : sv;
  const auto chunk = [](const void* p, size_t stride, int n, int rows, int width) {
    return la_buf(static_cast<const char*>(p) + (size_t)(CH * n) * stride, (size_t)(rows - 1) * stride + width);
  };
  const auto rows = [&](int n) { return min(CH, un.len - CH * n); };
  const LaDecays decays(a.geo, un.row0, h, lane);
  const auto decay = [&](int n) { return decays.load(n, rows(n)); };

  LaState<A> st;
  st.a0 = hf ? A / 2 : 0;
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
  typename C::TX tx;
  typename C::TY ty;
  typename C::TZ tz;
  const typename C::TX::Off ox(sx, tid);
  const typename C::TY::Off oy(sx, tid);
  const typename C::TZ::Off oz(sz, tid);
  const auto fetch = [&](int n) {
    tx.load(chunk(X, sx, n, rows(n), 2 * A), ox);
    ty.load(chunk(Y, sx, n, rows(n), 2 * A), oy);
    tz.load(chunk(Z, sz, n, rows(n), 128), oz);
  };
  const auto settle = [&](int buf) {
    tx.store(reinterpret_cast<__bf16*>(smem + buf * C::BUF), tid);
    ty.store(reinterpret_cast<__bf16*>(smem + buf * C::BUF + C::OFF_Y), tid);
    tz.store(reinterpret_cast<__bf16*>(smem + buf * C::BUF + C::OFF_Z), tid);
  };
  // output rows 16 i + c, columns b0 + 4 g: a row each of o, dq or the group's part
  const int i0 = hf ? 1 : 0, i1 = hf ? 2 : 3;  // the wave's row tiles
  const bool part = DQ && a.Pq != nullptr;
  const size_t so = DQ ? (part ? (size_t)H * DK * 4 : sk) : sv;
  char* O = DQ ? (part ? reinterpret_cast<char*>(a.Pq + (un.row0 * H + h) * DK)
                       : reinterpret_cast<char*>(a.dq + (un.row0 * HK + hk) * DK))
               : reinterpret_cast<char*>(a.o + (un.row0 * H + h) * DV);
  const unsigned oo[2] = {la_off(16 * i0 + c, so, (part ? 4 : 2) * (b0 + 4 * g)),
                          la_off(16 * i1 + c, so, (part ? 4 : 2) * (b0 + 4 * g))};
  unsigned oq[4];
  if constexpr (DQ) {
#pragma unroll
    for (int i = 0; i < 4; ++i) oq[i] = la_off(16 * i + c, sk, 2 * (b0 + 4 * g));
  }
  float graw = 0.f;
  if (nc > 0) {
    fetch(0);
    if (wave == TW) {
      la_tables(decay(0), rows(0), tab[0], lane, 1.f);
      if (nc > 1) graw = decay(1);
    }
    if (wave == 1) {  // the tiles above the diagonal that a product of 32 rows meets
      la_zero_tile(sPh, 0, 16, lane);
      la_zero_tile(sPl, 0, 16, lane);
      la_zero_tile(sPh, 32, 48, lane);
      la_zero_tile(sPl, 32, 48, lane);
    }
    settle(0);
  }
  const auto step = [&](int n, auto buf) {  // buf: n's parity
    constexpr int BUF = decltype(buf)::value;
    __syncthreads();
    const bool more = n + 1 < nc;
    const LaTab& t = tab[BUF];
    const int len = rows(n);
    const __bf16* sX = reinterpret_cast<const __bf16*>(smem + BUF * C::BUF);
    const __bf16* sY = reinterpret_cast<const __bf16*>(smem + BUF * C::BUF + C::OFF_Y);
    const __bf16* sZ = reinterpret_cast<const __bf16*>(smem + BUF * C::BUF + C::OFF_Z);
    bf4 qv[4];
    if constexpr (DQ) {
      const auto buf = chunk(q0, sk, n, len, 2 * DK);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        qv[i] = __builtin_bit_cast(bf4, __builtin_amdgcn_raw_buffer_load_b64(buf, oq[i], 0, 0));
    }
    if (more) fetch(n + 1);
    // scores, P[r][s], four s a lane
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      if (m < la_tiles<8>(wave)) {
        int i, j;
        la_tile_of<8>(wave, m, i, j);
        f4 x = la_score<A, C::TY::LD, C::TX::LD>(sY, sX, 16 * j, 16 * i, lane);
        x *= la_decay_tile<true>(t, i, j, lane);
        const int at = (16 * i + c) * LS + 16 * j + 4 * g;
        la_split4(sPh + at, sPl + at, x);
      }
    }
    if (more && wave == TW) {
      la_tables(graw, rows(n + 1), tab[BUF ^ 1], lane, 1.f);
      if (n + 2 < nc) graw = decay(n + 2);
    }
    f4 acc[4];
    st.template read<DQ ? 3 : 2>(sX, C::TX::LD, acc, lane);
    if constexpr (DQ) {
      // a_r over the wave's columns and its half of the state
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
    la_hand(acc, hf, sEx + wave * 512, lane);
    __syncthreads();
    f4 own[2];
    la_take(acc, hf, sEx + (wave ^ 4) * 512, own, lane);
    own[0] *= t.E[16 * i0 + c];
    own[1] *= t.E[16 * i1 + c];
    const int c0 = 16 * (wave & 3);
    const bf8 z[2] = {ld_tr8(sZ, C::TZ::LD, 0, c0, lane), ld_tr8(sZ, C::TZ::LD, 32, c0, lane)};
    const __bf16 *p0 = sPh + (16 * i0 + c) * LS + 8 * g, *p1 = sPh + (16 * i1 + c) * LS + 8 * g;
    constexpr int PL = CH * LS;  // from the high plane to the low
    own[0] = mma(z[0], ld8(p0 + PL), own[0]);
    own[1] = mma(z[0], ld8(p1 + PL), own[1]);
    own[0] = mma(z[0], ld8(p0), own[0]);
    own[1] = mma(z[1], ld8(p1 + PL + 32), own[1]);
    own[1] = mma(z[0], ld8(p1), own[1]);
    own[1] = mma(z[1], ld8(p1 + 32), own[1]);
    st.update(sY, C::TY::LD, z, t.T, t.eC, lane);
    const float sc = a.geo.scale;
    const size_t row = un.row0 + CH * n;
    const auto out = chunk(O, so, n, len, (part ? 4 : 2) * B);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (part)
        la_putf(out, oo[i], own[i] * sc);
      else
        la_put4(out, oo[i], own[i] * sc);
    }
    if constexpr (DQ) {
      if ((n + 1) % kLaAnchor == 0 || !more)
        st.store_t(a.aS + ((size_t)unit * a.anchors + n / kLaAnchor) * (DK * DV), b0, lane);
      if (wave == 0 && lane < len) {
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) x += sA[w * CH + lane];
        a.pa[((size_t)slice * a.geo.B * a.geo.T + row + lane) * H + h] = sc * x * t.E[lane];
      }
    }
    if (more) settle(BUF ^ 1);
  };
  for (int n = 0; n < nc; n += 2) {
    step(n, std::integral_constant<int, 0>{});
    if (n + 1 < nc) step(n + 1, std::integral_constant<int, 1>{});
  }
  if constexpr (!DQ) {
    if (un.last && a.ST) st.store(a.ST + ((size_t)un.seq * H + h) * (DK * DV), DV, b0, lane);
  }
}

template <int DK, int DV>
__global__ __launch_bounds__(512) void la_scan_fwd_kernel(LaScanArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  la_forward<DK, DV, false>(a, blockIdx.x, smem);
}
template <int DK, int DV>
__global__ __launch_bounds__(512) void la_scan_dq_kernel(LaScanArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  la_forward<DK, DV, true>(a, blockIdx.x, smem);
}

// ---- dk and dv -------------------------------------------------------------
// A workgroup takes a slice of dv's columns (its first NWV waves) and one of dk's; both read
// the same four tiles, of which LDS holds one chunk's at a time.
template <int DK, int DV>
struct LaRevCfg {
  static constexpr int NS = (DK > DV ? DK : DV) / 64;
  static constexpr int BV = DV / NS, BK = DK / NS, NWV = BV / 8, NWK = BK / 8, NW = NWV + NWK, NTHR = 64 * NW;
  using TK = LaTile<DK, NTHR>;
  using TQ = LaTile<DK, NTHR, 16>;
  using TV = LaTile<DV, NTHR>;
  using TD = LaTile<DV, NTHR, 16>;
  static constexpr int OFF_K = TQ::BYTES, OFF_V = OFF_K + TK::BYTES, OFF_D = OFF_V + TV::BYTES, OFF_P = OFF_D + TD::BYTES;
  static constexpr int PB = CH * LS * 2;  // one plane of scores
  static constexpr int OFF_T = OFF_P + 4 * PB, OFF_X = OFF_T + 2 * (int)sizeof(LaTab), OFF_W = OFF_X + NW * 512 * 4;
  static constexpr int LDS = OFF_W + (4 + 4 + NWV) * CH * 4;
  static_assert(NW > 10 && LDS <= 160 * 1024, "a wave a score tile, one for the decays");
};

template <int DK, int DV, bool ISV>
__device__ __forceinline__ void la_reverse(const LaScanArgs& a, unsigned char* smem) {
  using C = LaRevCfg<DK, DV>;
  constexpr int A = ISV ? DK : DV, NG = (ISV ? C::NWV : C::NWK) / 2, TW = 0;  // rows of the role's state, column groups
  __bf16 *sQ = reinterpret_cast<__bf16*>(smem), *sK = reinterpret_cast<__bf16*>(smem + C::OFF_K);
  __bf16 *sV = reinterpret_cast<__bf16*>(smem + C::OFF_V), *sD = reinterpret_cast<__bf16*>(smem + C::OFF_D);
  __bf16* sP = reinterpret_cast<__bf16*>(smem + C::OFF_P);  // planes: q k hi, lo; do v hi, lo
  LaTab* tab = reinterpret_cast<LaTab*>(smem + C::OFF_T);
  float* sRow = reinterpret_cast<float*>(smem + C::OFF_W);  // [j][r], [i][s], [wave][s]
  float *sCol = sRow + 4 * CH, *sB = sCol + 4 * CH, *sEx = reinterpret_cast<float*>(smem + C::OFF_X);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, c = lane & 15;
  const int H = a.geo.H, HK = H / a.geo.G;
  int unit, slice;
  if (!la_slot<C::NS>(blockIdx.x, a.segs.nslot * H, unit, slice)) return;
  LaUnit un;
  if (!la_unit(a.segs, a.geo.T, unit / H, un)) return;
  const int h = unit % H, hk = h / a.geo.G, nc = (un.len + CH - 1) / CH;
  const size_t sk = (size_t)HK * DK * 2, sv = (size_t)H * DV * 2;  // bytes a row
  const bf16_t *q0 = a.q + (un.row0 * HK + hk) * DK, *k0 = a.k + (un.row0 * HK + hk) * DK;
  const bf16_t *v0 = a.v + (un.row0 * H + h) * DV, *d0 = a.dout + (un.row0 * H + h) * DV;
  const float scale = a.geo.scale;
  const auto at = [&](int n) { return nc - 1 - n; };
  const auto rows = [&](int n) { return min(CH, un.len - CH * at(n)); };
  const LaDecays decays(a.geo, un.row0, h, lane);
  const auto decay = [&](int n) { return decays.load(at(n), rows(n)); };
  const int rw = ISV ? wave : wave - C::NWV;  // wave of the role
  const bool hf = rw >= NG;
  const int b0 = (ISV ? C::BV : C::BK) * slice + 16 * (hf ? rw - NG : rw);

  LaState<A> st;  // dS, columns of Dv; or dS^T, columns of Dk
  st.a0 = hf ? A / 2 : 0;
  {
    const float* init = un.last ? (a.dST ? a.dST + ((size_t)un.seq * H + h) * (DK * DV) : nullptr)
                                : a.dS + ((size_t)unit + H) * (DK * DV);
    if (init == nullptr)
      st.zero();
    else if (ISV)
      st.load(init, DV, b0, lane);
    else
      st.load_t(init, b0, lane);
  }
  typename C::TQ tq;
  typename C::TK tk;
  typename C::TV tv;
  typename C::TD td;
  const typename C::TQ::Off oq(sk, tid);
  const typename C::TK::Off ok(sk, tid);
  const typename C::TD::Off od(sv, tid);
  const typename C::TV::Off ov(sv, tid);
  const auto chunk = [&](const void* p, size_t stride, int n, int width) {
    return la_buf(static_cast<const char*>(p) + (size_t)(CH * at(n)) * stride, (size_t)(rows(n) - 1) * stride + width);
  };
  const auto fetch = [&](int n) {
    tq.load(chunk(q0, sk, n, 2 * DK), oq);
    tk.load(chunk(k0, sk, n, 2 * DK), ok);
    tv.load(chunk(v0, sv, n, 2 * DV), ov);
    td.load(chunk(d0, sv, n, 2 * DV), od);
  };
  const auto settle = [&] {
    tq.store(sQ, tid);
    tk.store(sK, tid);
    tv.store(sV, tid);
    td.store(sD, tid);
  };
  const bool part = !ISV && a.Pk != nullptr;
  const size_t so = ISV ? sv : part ? (size_t)H * DK * 4 : sk;
  char* O = ISV ? reinterpret_cast<char*>(a.dv + (un.row0 * H + h) * DV)
                : part ? reinterpret_cast<char*>(a.Pk + (un.row0 * H + h) * DK)
                       : reinterpret_cast<char*>(a.dk + (un.row0 * HK + hk) * DK);
  const int wo = ISV ? 2 * DV : (part ? 4 : 2) * DK;
  const int i0 = hf ? 1 : 0, i1 = hf ? 2 : 3;  // the wave's row tiles
  const unsigned oo[2] = {la_off(16 * i0 + c, so, (part ? 4 : 2) * (b0 + 4 * g)),
                          la_off(16 * i1 + c, so, (part ? 4 : 2) * (b0 + 4 * g))};
  float graw = 0.f;
  if (nc > 0) {
    fetch(0);
    if (wave == TW) {
      la_tables(decay(0), rows(0), tab[0], lane, scale);
      if (nc > 1) graw = decay(1);
    }
    if (wave == 1) {
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        la_zero_tile(sP + m * (CH * LS), 16, 0, lane);
        la_zero_tile(sP + m * (CH * LS), 48, 32, lane);
      }
    }
    settle();
  }
  for (int n = 0; n < nc; ++n) {
    __syncthreads();
    const bool more = n + 1 < nc;
    const LaTab& t = tab[n & 1];
    const int len = rows(n), cn = at(n);
    const size_t row = un.row0 + CH * cn;
    if (more) fetch(n + 1);
    if constexpr (ISV) {
      if ((cn + 1) % kLaAnchor == 0 || n == 0)  // dS behind this chunk
        st.store(a.aD + ((size_t)unit * a.anchors + cn / kLaAnchor) * (DK * DV), DV, b0, lane);
    }
    // scores, P[s][r], four r a lane, and the sums of W
    {
      // the waves of dk take them (two parts of the state to dv's three), dv's first what is over
      const int m = C::NW - 1 - wave;
      if (m < 10) {
        int i, j;
        la_tile_of<C::NW>(m, 0, i, j);
        const f4 d = la_decay_tile<false>(t, i, j, lane) * scale;
        const f4 x = la_score<DK, C::TQ::LD, C::TK::LD>(sQ, sK, 16 * i, 16 * j, lane) * d;
        const f4 y = la_score<DV, C::TD::LD, C::TV::LD>(sD, sV, 16 * i, 16 * j, lane);
        const int p = (16 * j + c) * LS + 16 * i + 4 * g;
        la_split4(sP + p, sP + CH * LS + p, x);
        la_split4(sP + 2 * CH * LS + p, sP + 3 * CH * LS + p, y * d);
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
    }
    if (more && wave == TW) {
      la_tables(graw, rows(n + 1), tab[(n + 1) & 1], lane, scale);
      if (n + 2 < nc) graw = decay(n + 2);
    }
    f4 acc[4];
    st.template read<ISV ? 3 : 2>(ISV ? sK : sV, ISV ? C::TK::LD : C::TV::LD, acc, lane);
    if constexpr (ISV) {
      // b_s over the wave's columns and its half of the state
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
    la_hand(acc, hf, sEx + wave * 512, lane);
    __syncthreads();
    f4 own[2];
    la_take(acc, hf, sEx + (hf ? wave - NG : wave + NG) * 512, own, lane);
    own[0] *= t.T[16 * i0 + c];
    own[1] *= t.T[16 * i1 + c];
    const __bf16* Z = ISV ? sD : sQ;
    constexpr int LDZ = ISV ? C::TD::LD : C::TQ::LD;
    const bf8 z[2] = {ld_tr8(Z, LDZ, 0, b0, lane), ld_tr8(Z, LDZ, 32, b0, lane)};
    const __bf16* Ph = sP + (ISV ? 0 : 2 * CH * LS);
    const __bf16 *p0 = Ph + (16 * i0 + c) * LS + 8 * g, *p1 = Ph + (16 * i1 + c) * LS + 8 * g;
    constexpr int PL = CH * LS;
    own[0] = mma(z[0], ld8(p0 + PL), own[0]);
    own[1] = mma(z[1], ld8(p1 + PL + 32), own[1]);
    own[0] = mma(z[1], ld8(p0 + PL + 32), own[0]);
    own[1] = mma(z[1], ld8(p1 + 32), own[1]);
    own[0] = mma(z[0], ld8(p0), own[0]);
    own[0] = mma(z[1], ld8(p0 + 32), own[0]);
    st.update(ISV ? sQ : sD, ISV ? C::TQ::LD : C::TD::LD, z, t.E, t.eC, lane);
    const auto out = chunk(O, so, n, wo);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (part)
        la_putf(out, oo[i], own[i]);
      else
        la_put4(out, oo[i], own[i]);
    }
    __syncthreads();
    if (wave == C::NW - 1 && lane < len) {
      float x = 0.f;
#pragma unroll
      for (int w = 0; w < C::NWV; ++w) x += sB[w * CH + lane];
      a.pb[((size_t)slice * a.geo.B * a.geo.T + row + lane) * H + h] = x * t.T[lane];
      if (slice == 0) {
        float rs = 0.f, cs = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          rs += j <= g ? sRow[j * CH + lane] : 0.f;
          cs += j >= g ? sCol[j * CH + lane] : 0.f;
        }
        a.prc[(row + lane) * H + h] = rs - cs;
      }
    }
    if (more) settle();
  }
  if constexpr (ISV) {
    if (un.first && a.dS0) st.store(a.dS0 + ((size_t)un.seq * H + h) * (DK * DV), DV, b0, lane);
  }
}

// The two roles meet at the same barriers: both run the same loop over the same chunks.
template <int DK, int DV>
__global__ __launch_bounds__((LaRevCfg<DK, DV>::NTHR)) void la_scan_dkv_kernel(LaScanArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  if (__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) < LaRevCfg<DK, DV>::NWV)
    la_reverse<DK, DV, true>(a, smem);
  else
    la_reverse<DK, DV, false>(a, smem);
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
    hipLaunchKernelGGL((la_segstate_kernel<DK, DV, true>), dim3(grid), dim3(512), 0, st, a);
  else
    hipLaunchKernelGGL((la_segstate_kernel<DK, DV, false>), dim3(grid), dim3(512), 0, st, a);
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
  return la_launch(la_scan_fwd_kernel<DK, DV>, la_grid<C::NS>(a.segs.nslot * a.geo.H), C::NTHR, C::LDS, a, st);
}

template <int DK, int DV>
hipError_t launch_la_scan_bwd(const LaScanArgs& a, hipStream_t st) {
  using CQ = LaFwdCfg<DK, DV, true>;
  using CR = LaRevCfg<DK, DV>;
  const int units = a.segs.nslot * a.geo.H;
  hipError_t e = la_launch(la_scan_dq_kernel<DK, DV>, la_grid<CQ::NS>(units), CQ::NTHR, CQ::LDS, a, st);
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

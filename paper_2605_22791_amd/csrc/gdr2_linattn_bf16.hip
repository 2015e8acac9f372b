// Linear attention with a decay for each head, bf16 problems: scans over the chunks of a
// segment with the state in registers.
//
// Forward and backward are one form.  With X, Y (rows of length A) and Z (rows of length
// B) among q, k, v, dout, and a state St (A x B), a chunk gives
//     out_i = f_i X_i St + sum_j P_ij Z_j,     P_ij = scale D (X_i . Y_j)
//     St   <- exp(G_C) St + sum_j Y_j^T (w_j Z_j)
//   o :  X q, Y k,  Z v;   St = S,     f = scale exp(G_r), w = exp(G_C - G_s), j <= i, first chunk to last
//   dq:  X do, Y v, Z k;   St = S^T,   as above
//   dv:  X k, Y q,  Z do;  St = dS,    f = exp(G_C - G_s), w = scale exp(G_r), j >= i, last chunk to first
//   dk:  X v, Y do, Z q;   St = dS^T,  as dv
// A workgroup runs one of these over one segment of one head.
//
// A wave owns 32 columns of B over all of A: its state tiles are the accumulators of the update,
// and split to bf16 they are the A operand of X St as they lie (the K order of that product is
// permuted to the accumulators' rows), so the state never leaves its registers.  The tiles X, Y,
// Z go through LDS; the scores of a chunk are shared out over the waves, pass through LDS split
// into bf16 parts, and meet the same Z fragments that the update uses (scaled).  Three barriers
// a chunk, each with work on one side that hides the loads of the tiles on the other:
//     X, Z there, Y's place free:  load Y;  X St, Z fragments
//     Y there:                     scores, the decays of the next chunk
//     P there, X, Z done with:     load the next X, Z;  P Z, output, update
// What counts is how many instructions there are: a vector one takes 4 cycles of a SIMD's issue
// and an MFMA 8 (of 16 that it is busy for) when waves share it, and at these rates the chip
// draws its power: its clock falls to 1.6 GHz in the long scans, from 2.2 in short ones.
// Two workgroups a CU (80 KB of LDS each) fill each other's gaps; the waves' priority (the scores,
// short dependent steps that others wait for, over X St, that over the rest) keeps them in
// different parts of a chunk: gradients 552 to 518 us, forward scan 164 to 148.
//
// Precision: inputs are exact bf16 operands.  What is held in 32 bits between them, the state, the
// scores and the decayed Z, enters the products split into three bf16 parts (24 bits, as many as it
// has).  The decays' gradient and the fp32 states need them; o and dk, rounded to bf16 behind, would
// pass their 2e-3 with two (16 bits), in 4 to 9 % less time, but then differ from the same rounding of
// 32-bit values by 1e-4 of their norm, where three parts differ by 3e-5.
//
// Measured, 8 x 4096 tokens, 16 heads of 128 x 128, four segments a sequence: forward scan 148 us
// (537 MB, 3.6 TB/s), segment states 70 and 67 us, the three gradients 518 us (2 GB read and
// written, 3.8 TB/s), the decays' gradient 24 us.  Of the gradients' 518 us, tiles all from the same
// place take 485 and two parts for three 414: it is the instructions of the split products, and the
// power they draw, rather than memory.

#include "gdr2_linattn.hpp"
#include "gdr2_bf16.hpp"

namespace gdr2 {

namespace {

enum LaRole : int { kLaO, kLaDq, kLaDv, kLaDk };

struct LaUnit {
  size_t row0;
  int len, seq, slot;
  bool first, last;
};

// Sequence `lane` of up to 64: its tokens a to b, its slots first to behind (a whole wave calls).
struct LaSpan {
  int a, b, first, behind;
  __device__ __forceinline__ LaSpan(const LaSegs& s, int T) {
    const int lane = threadIdx.x & 63;
    a = b = 0;
    int n = 0;
    if (lane < s.nseq) {
      a = min(max(s.cu[lane], 0), T);
      b = min(max(s.cu[lane + 1], a), T);
      n = max(1, (b - a + s.seg_tokens - 1) / s.seg_tokens);
    }
    behind = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(behind, o);
      if (lane >= o) behind += y;
    }
    first = behind - n;
  }
};

// Segment `slot`; false past the last one in use (uniform).  Table entries are kept in range
// whatever a workspace holds.
__device__ __forceinline__ bool la_unit(const LaSegs& s, int T, int slot, LaUnit& u) {
  u.slot = slot;
  if (s.cu) {
    const LaSpan x(s, T);
    const int lane = threadIdx.x & 63;
    u.seq = __popcll(__ballot(lane < s.nseq && x.behind <= slot));
    if (slot >= s.nslot || u.seq >= s.nseq) return false;
    const int a = __builtin_amdgcn_readlane(x.a, u.seq), b = __builtin_amdgcn_readlane(x.b, u.seq);
    const int first = __builtin_amdgcn_readlane(x.first, u.seq), behind = __builtin_amdgcn_readlane(x.behind, u.seq);
    const int t0 = a + (slot - first) * s.seg_tokens;
    u.row0 = (size_t)t0;
    u.len = max(0, min(s.seg_tokens, b - t0));
    u.first = slot == first;
    u.last = slot + 1 == behind;
    return true;
  }
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

// Workgroup b of the gradients' grid: first dq and dv, the longer ones, of eight units after each
// other, then dk.  Blocks go to the eight XCDs in turn, so a unit's run on one and share its L2.
// (A training step with all three of a unit together: 1 % less at 8 x 4096 tokens, 16 heads of
// 128 x 128, but 2 % more there at 64 x 64 and in packed batches, 5 % more at 128 x 64: a tail of long ones.)
__device__ __forceinline__ bool la_slot(int b, int n, int& unit, int& role) {
  const int n8 = (n + 7) / 8 * 8;
  if (b < 2 * n8) {
    unit = b / 16 * 8 + b % 8;
    role = b / 8 % 2 ? kLaDv : kLaDq;
  } else {
    unit = b - 2 * n8;
    role = kLaDk;
  }
  return unit < n;
}
unsigned la_grid(int n) { return (unsigned)((n + 7) / 8 * 8) * 3; }

// ---- decays of a chunk -----------------------------------------------------
// Sums are taken within the blocks of 16 rows in 64 bits, p_r up to and including r, so that
// no factor is a difference of long sums; they are powers of two (log2 e is multiplied in
// there).  Between blocks j < i, scale D_rs = L_r R_is with L_r = scale exp(p_r) and R_is the
// rest of the way from s to block i; the exponentials are at most 1.
struct alignas(16) LaTab {
  double p[CH];
  float L[CH], R[3][CH], E[CH], T[CH];  // R[i - 1][s]; E: scale exp(G_r), T: exp(G_C - G_s)
  float eC, pad[3];
};

// Row 16 i + c's sum of x[i] over g, in lane 16 i + c (each swap serves two values)
__device__ __forceinline__ float la_sum4(const float (&x)[4]) {
  const auto halves = [](float a, float b) {  // a's sum over halves in the lower lanes, b's in the upper
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
  };
  const float a = halves(x[0], x[2]), b = halves(x[1], x[3]);
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <int CTRL>
__device__ __forceinline__ double la_dpp(double x) {
  const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(x), CTRL, 0xF, 0xF, true);
  const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(x), CTRL, 0xF, 0xF, true);
  return __hiloint2double(hi, lo);
}
// x as if new: lanes' conditions formed from it stay inside the loop they are in, where kept over
// it their masks would take the scalar registers and spill
__device__ __forceinline__ int la_new(int x) {
  asm("" : "+v"(x));
  return x;
}
__device__ __forceinline__ float la_lanef(float x, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane));
}
__device__ __forceinline__ float la_ex(float x) { return ex2(x * kLog2e); }

// One wave, a row a lane: g the row's raw log-decay; rows past the chunk's end do not decay.
// Returns the row's log-decay.
__device__ __forceinline__ float la_tables(float g, int rows, LaTab& t, int lane, float scale) {
  lane = la_new(lane);
  const float g0 = lane < rows ? (g < kLaForget ? kLaForget : g) : 0.f;
  double p = (double)g0 * 1.4426950408889634;
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
  t.L[lane] = scale * ex2(pf);
  t.E[lane] = scale * ex2(before + pf);
  t.T[lane] = ex2(r3 + m3);
  t.R[0][lane] = ex2(r1);  // to block 1: read for rows of block 0
  t.R[1][lane] = ex2(r2);  // to block 2: of blocks 0, 1
  t.R[2][lane] = ex2(r3);
  if (lane == 0) t.eC = ex2((b0 + b1) + (b2 + b3));
  return g0;
}

// ---- memory ----------------------------------------------------------------
typedef unsigned u2v __attribute__((ext_vector_type(2)));
__device__ __forceinline__ __amdgpu_buffer_rsrc_t la_buf(const void* p, size_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)(unsigned)bytes, 0x00020000);
}

// The rows of a segment from a chunk's first on, as a buffer: a load past the last row gives
// zero, a store there is dropped, and a lane's offsets are the same for every chunk (what moves
// is in scalar registers).  A segment spans at most 2^31 bytes (the call cuts it so).
template <bool REV>
struct LaRows {
  const char* p;
  unsigned left;
  __device__ __forceinline__ LaRows(const void* base, unsigned stride, int width, int len) {
    const int first = REV ? (len - 1) / CH : 0;  // the chunk a scan begins with
    p = static_cast<const char*>(base) + (size_t)first * CH * stride;
    left = (len - first * CH - 1) * stride + width;
  }
  __device__ __forceinline__ void next(unsigned stride) {
    const unsigned step = CH * stride;
    if (REV)
      p -= step, left += step;
    else
      p += step, left -= step;
  }
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t buf() const { return la_buf(p, left); }
};

// The log-decay of row `lane` of a chunk as it lies in memory: loaded a step before it is
// needed, and looked at only there.
struct LaDecays {
  const char* base;
  unsigned stride;  // bytes a row; 0: one for every token
  unsigned off;
  __device__ __forceinline__ LaDecays(const LaGeo& a, size_t row0, int h, int lane) {
    base = reinterpret_cast<const char*>(a.per_head ? a.g + h : a.g + row0 * a.H + h);
    stride = a.per_head ? 0 : 4u * a.H;
    off = lane * stride;
  }
  __device__ __forceinline__ float load(int chunk, int rows) const {
    const auto buf = la_buf(base + (size_t)chunk * CH * stride, (rows - 1) * stride + 4);
    return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(buf, off, 0, 0));
  }
};

// ---- tiles -----------------------------------------------------------------
// 64 rows in LDS, 64 columns a plane, the 16-byte pieces of a row exchanged by piece ^ f(row),
// f of the row in its block of 16.  Two ways of reading share the banks: 16-byte fragments
// (which the LDS serves in groups of 16 lanes, rows 0-3 and 12-15 of one piece with rows 4-11
// of the next), and transposed ones (4 rows, every other 8 of 64 bytes).  f keeps both free of
// conflicts, 4 cycles a wave's instruction, where rows padded by 16 bytes took 8 and 4.
// Planes lie apart by a constant that instructions hold, so that few addresses are formed.
constexpr int kLaRow = 128, kLaPlane = CH * kLaRow;  // bytes
constexpr int la_bytes(int cols) { return cols / 64 * kLaPlane; }
__device__ __forceinline__ int la_swz(int row) { return ((row & 2) << 1) ^ ((row & 4) >> 1) ^ ((row & 8) ? 3 : 0); }

// A lane's byte addresses inside a tile
struct LaAt {
  int frag;   // row c, columns 8 g ..; ^ 64: 32 columns on
  int tr[2];  // transposed: rows 8 g + (c >> 2), and 4 on, columns 8 (c & 3) .. + 3; 8 on: the next four; ^ 64: 32 columns on
  int z[2];   // the same of the wave's 32 columns
  int out;    // row c, columns 8 g .. of the wave's
  __device__ __forceinline__ LaAt(int lane, int wave) {
    const int g = lane >> 4, c = lane & 15, mine = (wave >> 1) * kLaPlane, half = 64 * (wave & 1);
    frag = c * kLaRow + ((g ^ la_swz(c)) << 4);
    out = mine + (frag ^ half);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int r = 8 * g + (c >> 2) + 4 * k;
      tr[k] = r * kLaRow + (((c & 3) ^ la_swz(r)) << 4);
      z[k] = mine + (tr[k] ^ half);
    }
  }
};
__device__ __forceinline__ bf8 la_ld16(const unsigned char* p) { return *reinterpret_cast<const bf8*>(p); }
// Transposed fragment: rows 8 g + e of column c, from the two addresses of a lane
__device__ __forceinline__ bf8 la_ld_tr(const unsigned char* p0, const unsigned char* p1) {
  return ld_tr8p(reinterpret_cast<const __bf16*>(p0), reinterpret_cast<const __bf16*>(p1));
}

// A tile's way from memory straight into LDS, a kilobyte (8 rows of a plane) an instruction,
// shared out over NW waves.  Rows past the segment's end become zero (the buffer's range).
// Written out, and waited for with la_landed: as builtins, the compiler would hold every LDS
// read behind them.
template <int COLS, int NW>
struct LaLoad {
  static constexpr int NP = la_bytes(COLS) / 1024 / NW;  // instructions a wave, all of one plane
  static_assert(NP % 2 == 0 && NP <= 8, "whole blocks of 16 rows in one plane");
  unsigned off;
  __device__ __forceinline__ LaLoad(unsigned stride, int lane, int wave) {  // stride: bytes a row, a multiple of 128
    const int k = wave * NP;
    off = (k / 8) * kLaRow + (8 * (k % 8) + lane / 8) * stride + (((lane % 8) ^ la_swz(lane / 8)) << 4);
  }
  template <bool REV>
  __device__ __forceinline__ void load(const LaRows<REV>& r, unsigned stride, unsigned lds, int wave) const {
    const u4v buf = {(unsigned)(uintptr_t)r.p, (unsigned)((uintptr_t)r.p >> 32) & 0xffffu, r.left, 0x00020000u};
    // formed anew at each call: kept over a loop, the many scalar values would spill into vector lanes
    unsigned to = lds + wave * (NP * 1024), step = 8 * stride;
    asm("" : "+s"(to), "+s"(step));
#pragma unroll
    for (int m = 0; m < NP; ++m) {
      const unsigned from = (off ^ (m & 1 ? 0x30 : 0)) + m * step, at = to + m * 1024;  // f(8) = 3
      // m0, the place in LDS, has to be written a wait state before the load reads it
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(at), "v"(from), "s"(buf)
                   : "memory", "m0");
    }
  }
};
// All but the wave's last `after` memory instructions are done (they complete in order).
template <int AFTER>
__device__ __forceinline__ void la_landed() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(AFTER) : "memory");
}
// What lanes of a wave leave for each other in LDS: it serves a wave's instructions in order.
__device__ __forceinline__ void la_wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
__device__ __forceinline__ unsigned la_lds(const void* p) {
  return (unsigned)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

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
constexpr int kLaParts = 3;
struct LaFr {
  bf8 p[kLaParts];  // largest first
};
__device__ __forceinline__ LaFr la_split8(const float (&x)[8]) {
  LaFr f;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    float a = x[e], b = x[e + 1];
#pragma unroll
    for (int k = 0; k < kLaParts; ++k) {
      const bf2 h = la_part(a, b);
      f.p[k][e] = h[0];
      f.p[k][e + 1] = h[1];
      if (k + 1 < kLaParts) la_left(h, a, b);
    }
  }
  return f;
}
__device__ __forceinline__ void la_split4(__bf16* p, int plane, const f4& x) {
  float r[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
  for (int k = 0; k < kLaParts; ++k) {
    const bf2 h0 = la_part(r[0], r[1]), h1 = la_part(r[2], r[3]);
    *reinterpret_cast<bf4*>(p + k * plane) = bf4{h0[0], h0[1], h1[0], h1[1]};
    if (k + 1 < kLaParts) {
      la_left(h0, r[0], r[1]);
      la_left(h1, r[2], r[3]);
    }
  }
}

// ---- a wave's state: 32 columns over the A rows ------------------------------
// Two blocks of 16: element m of block k is the wave's column 8 (m >> 2) + 4 k + (m & 3), so
// that a lane's eight outputs of a row are eight columns side by side.  Rows likewise: element m
// of block t is row 32 (t >> 1) + 8 (m >> 2) + 4 (t & 1) + (m & 3), and a lane's values of two
// blocks are eight rows side by side, which meet 16 bytes of X.
template <int A>
struct LaState {
  f4 s[2][A / 16];  // lane (g, c): elements 4 g + u of block t, element c of block k

  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int t = 0; t < A / 16; ++t) s[k][t] = f4zero();
  }
  __device__ __forceinline__ void decay(float eC) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int t = 0; t < A / 16; ++t) s[k][t] *= eC;
  }
  // Row-major (A, LD), or with TR its transpose, row-major (LD, A).  One offset a lane, the rest
  // in the instructions: sixty-four addresses would not fit.
  template <int LD, bool TR>
  __device__ __forceinline__ static unsigned at(int lane, int wave) {
    const int g = lane >> 4, c = lane & 15, col = 32 * wave + 8 * (c >> 2) + (c & 3);
    return 4 * (TR ? col * A + 8 * g : 8 * g * LD + col);
  }
  template <int LD, bool TR>
  __device__ __forceinline__ void load(const float* src, int lane, int wave) {
    const auto buf = la_buf(src, A * LD * 4);
    const unsigned off = at<LD, TR>(lane, wave);
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int t = 0; t < A / 16; ++t) {
        const int row = 32 * (t >> 1) + 4 * (t & 1);
        if constexpr (TR) {
          s[k][t] = __builtin_bit_cast(f4, __builtin_amdgcn_raw_buffer_load_b128(buf, off + 4 * row, 16 * A * k, 0));
        } else {
#pragma unroll
          for (int u = 0; u < 4; ++u)
            s[k][t][u] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(buf, off + 4 * LD * u + 16 * k, 4 * LD * row, 0));
        }
      }
  }
  template <int LD, bool TR>
  __device__ __forceinline__ void store(float* dst, int lane, int wave) const {
    const auto buf = la_buf(dst, A * LD * 4);
    const unsigned off = at<LD, TR>(lane, wave);
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int t = 0; t < A / 16; ++t) {
        const int row = 32 * (t >> 1) + 4 * (t & 1);
        const f4 x = s[k][t];
        if constexpr (TR) {
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4v, x), buf, off + 4 * row, 16 * A * k, 0);
        } else {
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const float y = x[u];
            __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(y), buf, off + 4 * LD * u + 16 * k, 4 * LD * row, 0);
          }
        }
      }
  }

  // acc[k][i] (elements 4 g + u of block k, row 16 i + c) = X St; St <- eC St
  __device__ __forceinline__ void read(const unsigned char* X, const LaAt& at, float eC, f4 (&acc)[2][4]) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[k][i] = f4zero();
#pragma unroll
    for (int p = 0; p < A / 32; ++p) {
      const unsigned char* xp = X + (p >> 1) * kLaPlane + (at.frag ^ (64 * (p & 1)));
      bf8 b[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) b[i] = la_ld16(xp + 16 * i * kLaRow);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          f4 z = s[k][2 * p + e];
          const f4 y = z * eC;
          asm("" : "+v"(z) : "v"(y));  // the decayed values lie elsewhere: the split takes these ones' place
          s[k][2 * p + e] = y;
#pragma unroll
          for (int u = 0; u < 4; ++u) x[4 * e + u] = z[u];
        }
        const LaFr f = la_split8(x);
#pragma unroll
        for (int q = kLaParts - 1; q >= 0; --q)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[k][i] = mma(f.p[q], b[i], acc[k][i]);
      }
    }
  }

  // St <- St + Y^T (w Z): z[k][kb] block k of the wave's Z columns, rows 32 kb + 8 g + e
  __device__ __forceinline__ void update(const unsigned char* Y, const LaAt& at, const bf8 (&z)[2][2], const float* w, int lane) {
    const int g = lane >> 4;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      float wv[8];
      ldf8(w + 32 * kb + 8 * g, wv);
      LaFr d[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        float x[8];
        unpack8(z[k][kb], x);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= wv[e];
        d[k] = la_split8(x);
      }
#pragma unroll
      for (int t0 = 0; t0 < A / 16; t0 += 4) {
        const unsigned char* yk = Y + 32 * kb * kLaRow + (t0 >> 2) * kLaPlane;
        bf8 y[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) y[t] = la_ld_tr(yk + (at.tr[0] ^ (64 * (t >> 1))) + 8 * (t & 1), yk + (at.tr[1] ^ (64 * (t >> 1))) + 8 * (t & 1));
#pragma unroll
        for (int q = kLaParts - 1; q >= 0; --q)
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int t = 0; t < 4; ++t) s[k][t0 + t] = mma(y[t], d[k].p[q], s[k][t0 + t]);
      }
    }
  }
};

// Z fragments of the wave's columns, rows 32 kb + 8 g + e
__device__ __forceinline__ void la_zfrags(const unsigned char* Z, const LaAt& at, bf8 (&z)[2][2]) {
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const unsigned char* zk = Z + 32 * kb * kLaRow + 8 * k;
      z[k][kb] = la_ld_tr(zk + at.z[0], zk + at.z[1]);
    }
}

// ---- scores ----------------------------------------------------------------
// One 16 x 16 tile of  sum_a Am[16 mi + m][a] Bn[16 ni + n][a]; lane (g, c): rows 4 g + u of Am, row c of Bn
template <int A>
__device__ __forceinline__ f4 la_score(const unsigned char* Am, const unsigned char* Bn, const LaAt& at, int mi, int ni) {
  const unsigned char *a = Am + 16 * mi * kLaRow, *b = Bn + 16 * ni * kLaRow;
  f4 x = f4zero();
#pragma unroll
  for (int p = 0; p < A / 32; ++p) {
    const int o = (p >> 1) * kLaPlane, f = at.frag ^ (64 * (p & 1));
    x = mma(la_ld16(a + f + o), la_ld16(b + f + o), x);
  }
  return x;
}

// Factors scale D_rs of a tile: ROWS_S, the lane's four values are s (r = r0 + c, one a lane), else
// r (s = s0 + c).  i, j: the blocks of r and s, DIAG: the same one; on the diagonal itself D is 1.
template <bool ROWS_S, bool DIAG>
__device__ __forceinline__ f4 la_decay_tile(const LaTab& t, int i, int j, int lane, float scale) {
  lane = la_new(lane);
  const int g = lane >> 4, c = lane & 15;
  f4 d;
  if constexpr (!DIAG) {
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
      const float e = scale * ex2((float)(ROWS_S ? pc - pu : pu - pc));
      d[u] = (ROWS_S ? 4 * g + u <= c : c <= 4 * g + u) ? e : 0.f;
    }
  }
  return d;
}

// The lower tiles (i, j <= i) of a chunk's scores, the six off the diagonal first: blocks of tile n
__device__ __forceinline__ void la_tile_of(int n, int& i, int& j) {
  // (3,0) (3,1) (3,2) (2,0) (2,1) (1,0)
  i = n < 3 ? 3 : n < 5 ? 2 : 1;
  j = n < 3 ? n : n < 5 ? n - 3 : 0;
}

// Score tiles in LDS, 512 bytes each (16 rows of the output, 16 columns that the product with Z
// sums over): twelve a plane, so that the two tiles of a product over 32 columns lie side by
// side, with a tile of zeros where that reaches past the diagonal.
constexpr int kLaScores = 12 * 256;  // bf16 elements a plane
template <bool REV>
__device__ __forceinline__ int la_ptile(int i, int j) {  // row tile i, column tile j
  if constexpr (REV) return i < 2 ? 4 * i + j : 2 * i + 2 + j;  // (i, j): 0 (0,0..3)  4 (1,0..3)  8 (2,2) (2,3)  10 (3,2) (3,3)
  return i < 2 ? 2 * i + j : 4 * (i - 1) + j;                   // 0 (0,0) (0,1)  2 (1,0) (1,1)  4 (2,0..3)  8 (3,0..3)
}

}  // namespace

// ---- a segment's own contribution to the state -----------------------------
// N = sum of Y^T (w Z) over the segment, from zero: S (k, v; first chunk to last) or, REV, dS
// (q, dout; last to first).  Not needed of the segment that ends its chain.
template <int DK, int DV, bool REV>
__global__ __launch_bounds__(2 * DV, 2) void la_segstate_kernel(LaScanArgs a) {
  constexpr int NW = DV / 32, TW = NW - 1;
  constexpr int OFF_Z = la_bytes(DK), BUF = OFF_Z + la_bytes(DV);
  extern __shared__ __align__(16) unsigned char smem[];
  LaTab* tab = reinterpret_cast<LaTab*>(smem + 2 * BUF);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int H = a.geo.H, HK = H / a.geo.G;
  const int unit = blockIdx.x;
  LaUnit un;
  if (!la_unit(a.segs, a.geo.T, unit / H, un)) return;
  if (REV ? un.first : un.last) return;
  const int h = unit % H, hk = h / a.geo.G;
  const int nc = (un.len + CH - 1) / CH;
  const unsigned sy = 2u * HK * DK, sz = 2u * H * DV;  // bytes a row
  LaRows<REV> Y((REV ? a.q : a.k) + (un.row0 * HK + hk) * DK, sy, 2 * DK, un.len);
  LaRows<REV> Z((REV ? a.dout : a.v) + (un.row0 * H + h) * DV, sz, 2 * DV, un.len);
  const float scale = REV ? a.geo.scale : 1.f;
  const auto at = [&](int n) { return REV ? nc - 1 - n : n; };
  const auto rows = [&](int n) { return min(CH, un.len - CH * at(n)); };
  const LaDecays decays(a.geo, un.row0, h, lane);
  const auto decay = [&](int n) { return decays.load(at(n), rows(n)); };
  const unsigned lds = la_lds(smem);
  const LaLoad<DK, NW> ly(sy, lane, wave);
  const LaLoad<DV, NW> lz(sz, lane, wave);
  const auto fetch = [&](int n) {
    const unsigned to = lds + (n & 1) * BUF;
    ly.load(Y, sy, to, wave);
    lz.load(Z, sz, to + OFF_Z, wave);
    Y.next(sy);
    Z.next(sz);
  };
  const LaAt ay(lane, wave);
  double gs = 0.0;
  LaState<DK> st;
  st.zero();
  float graw = 0.f;
  if (nc > 0) {
    // all that comes from memory on its way at once
    const float g0 = wave == TW ? decay(0) : 0.f;
    if (wave == TW && nc > 1) graw = decay(1);
    fetch(0);
    if (wave == TW) gs += (double)la_tables(g0, rows(0), tab[0], lane, scale);
  }
  for (int n = 0; n < nc; ++n) {
    la_landed<0>();
    __syncthreads();
    const bool more = n + 1 < nc;
    if (more) {
      if (wave == TW) {
        gs += (double)la_tables(graw, rows(n + 1), tab[(n + 1) & 1], lane, scale);
        if (n + 2 < nc) graw = decay(n + 2);
      }
      fetch(n + 1);
    }
    const LaTab& t = tab[n & 1];
    const unsigned char *sY = smem + (n & 1) * BUF, *sZ = sY + OFF_Z;
    bf8 z[2][2];
    la_zfrags(sZ, ay, z);
    st.decay(t.eC);
    st.update(sY, ay, z, REV ? t.E : t.T, lane);
  }
  float* N = (REV ? a.dS : a.S) + (size_t)unit * (DK * DV);
  st.template store<DV, false>(N, lane, wave);
  if (wave == TW) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) gs += __shfl_xor(gs, o);
    if (lane == 0) a.dec[unit] = la_ex((float)gs);
  }
}

// The states behind the segments (rev: the gradients before them), in the place of their
// contributions: what the chain's next segment starts from.
__global__ __launch_bounds__(256) void la_segcombine_kernel(LaScanArgs a, int size, int rev) {
  constexpr int AHEAD = 16;
  const int H = a.geo.H, per = size / 1024;
  const int q = blockIdx.x / per, e = ((blockIdx.x % per) * 256 + threadIdx.x) * 4, s = q / H, h = q % H;
  int c0 = s * a.segs.nseg, c1 = c0 + a.segs.nseg;
  if (a.segs.cu) {
    const LaSpan x(a.segs, a.geo.T);
    c0 = min(__builtin_amdgcn_readlane(x.first, s), a.segs.nslot);
    c1 = min(__builtin_amdgcn_readlane(x.behind, s), a.segs.nslot);
  } else if (a.segs.off) {
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
      if (i0 + j < n) {
        const size_t u = (size_t)(rev ? c1 - 1 - (i0 + j) : c0 + i0 + j) * H + h;
        x[j] = *reinterpret_cast<const f4*>(N + u * size + e);
        d[j] = a.dec[u];
      }
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

// ---- the scans ---------------------------------------------------------------

template <int DK, int DV, int ROLE>
struct LaCfg {
  static constexpr bool REV = ROLE == kLaDv || ROLE == kLaDk, TR = ROLE == kLaDq || ROLE == kLaDk;  // state transposed
  static constexpr bool SUMS = ROLE == kLaDq || ROLE == kLaDv;  // gives a term of the decays' gradient
  static constexpr int A = TR ? DV : DK, B = TR ? DK : DV, NW = B / 32;
  static constexpr int OFF_Y = la_bytes(A), OFF_Z = 2 * OFF_Y, OFF_P = OFF_Z + la_bytes(B);
  static constexpr int OFF_S = OFF_P + kLaParts * kLaScores * 2, OFF_T = OFF_S + NW * 2048;
  static constexpr int OFF_A = OFF_T + 2 * (int)sizeof(LaTab);
  static constexpr int LDS = OFF_A + (SUMS ? (NW + 1) * CH * 4 + NW * 64 : 0);
  static_assert(LDS <= 80 * 1024, "two workgroups a CU");
};

// GROUPED: dq and dk of each value head leave in fp32, to be summed over their key head's.
template <int DK, int DV, int ROLE, bool GROUPED>
__device__ __forceinline__ void la_scan(const LaScanArgs& a, int unit, unsigned char* smem) {
  using C = LaCfg<DK, DV, ROLE>;
  constexpr int A = C::A, B = C::B, NW = C::NW, TW = NW - 1;
  constexpr bool REV = C::REV, SUMS = C::SUMS, TR = C::TR;
  constexpr bool PART = GROUPED && (ROLE == kLaDq || ROLE == kLaDk);
  // The output's store instructions a chunk: for each block of 16 rows one of bf16, two of fp32 parts
  constexpr int BLOCKS = CH / 16, STORES = PART ? 2 * BLOCKS : BLOCKS;
  const unsigned char *sX = smem, *sY = smem + C::OFF_Y, *sZ = smem + C::OFF_Z;
  __bf16* sP = reinterpret_cast<__bf16*>(smem + C::OFF_P);
  LaTab* tab = reinterpret_cast<LaTab*>(smem + C::OFF_T);
  float *sA = reinterpret_cast<float*>(smem + C::OFF_A), *sDiag = sA + NW * CH, *sC = sDiag + CH;  // a wave's terms, the scores' diagonal, a wave's sums
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (wave >= NW) return;  // of a wider role beside this one
  const int g = lane >> 4, c = lane & 15;
  const int H = a.geo.H, HK = H / a.geo.G;
  LaUnit un;
  if (!la_unit(a.segs, a.geo.T, unit / H, un)) return;
  const int h = unit % H, hk = h / a.geo.G, nc = (un.len + CH - 1) / CH;
  const unsigned sk = 2u * HK * DK, sv = 2u * H * DV;        // bytes a row
  const unsigned sx = TR ? sv : sk, sz = TR ? sk : sv;       // of X and Y; of Z, the output and E
  const size_t rk = (un.row0 * HK + hk) * DK, rv = (un.row0 * H + h) * DV;
  const bf16_t *q0 = a.q + rk, *k0 = a.k + rk, *v0 = a.v + rv, *d0 = a.dout + rv;
  // output: grouped heads' parts in fp32, a row for each value head, or bf16
  const unsigned so = PART ? 4u * H * DK : sz;
  void* out0 = PART ? (void*)((ROLE == kLaDq ? a.Pq : a.Pk) + (un.row0 * H + h) * DK)
                    : (void*)(ROLE == kLaO ? a.o + rv : ROLE == kLaDv ? a.dv + rv : (ROLE == kLaDq ? a.dq : a.dk) + rk);
  LaRows<REV> X(ROLE == kLaO ? q0 : ROLE == kLaDq ? d0 : ROLE == kLaDv ? k0 : v0, sx, 2 * A, un.len);
  LaRows<REV> Y(ROLE == kLaO ? k0 : ROLE == kLaDq ? v0 : ROLE == kLaDv ? q0 : d0, sx, 2 * A, un.len);
  LaRows<REV> Z(ROLE == kLaO ? v0 : ROLE == kLaDq ? k0 : ROLE == kLaDv ? d0 : q0, sz, 2 * B, un.len);
  LaRows<REV> E(ROLE == kLaDq ? q0 : v0, sz, 2 * B, un.len);  // what the output is multiplied with for the decays' gradient
  LaRows<REV> out(out0, so, PART ? 4 * B : 2 * B, un.len);
  const float scale = a.geo.scale;
  const auto at = [&](int n) { return REV ? nc - 1 - n : n; };
  const auto rows = [&](int n) { return min(CH, un.len - CH * at(n)); };
  const LaDecays decays(a.geo, un.row0, h, lane);
  const auto decay = [&](int n) { return decays.load(at(n), rows(n)); };

  const unsigned lds = la_lds(smem);
  const LaLoad<A, NW> lx(sx, lane, wave);
  const LaLoad<B, NW> lz(sz, lane, wave);
  const LaAt ax(lane, wave);
  // Rows of E and of the output in memory are four lanes' sixteen bytes (a quarter of the address
  // cycles of a row a lane); they pass through the wave's own two kilobytes, 32 rows at a time.
  const unsigned o0 = (lane >> 2) * sz + 64 * wave + 16 * (lane & 3);
  unsigned char* sS = smem + C::OFF_S + 2048 * wave;
  const int sm = 64 * (lane >> 2) + (((lane & 3) ^ (-(lane >> 4) & 3)) << 4);  // as in memory: row lane >> 2, piece lane & 3
  const int sr = 64 * c + ((g ^ (-(c >> 2) & 3)) << 4);                        // as the products have it: row c, piece g
  // all that comes from memory on its way at once
  float g0 = 0.f, graw = 0.f;
  if (nc > 0) {
    if (wave == TW) {
      g0 = decay(0);
      if (nc > 1) graw = decay(1);
    }
    lx.load(X, sx, lds, wave);
    lz.load(Z, sz, lds + C::OFF_Z, wave);
  }
  LaState<A> st;
  {
    const float* given = REV ? a.dST : a.S0;
    const float* init = (REV ? un.last : un.first) ? (given ? given + ((size_t)un.seq * H + h) * (DK * DV) : nullptr)
                                                   : (REV ? a.dS + ((size_t)unit + H) * (DK * DV)
                                                          : a.S + ((size_t)unit - H) * (DK * DV));
    if (init == nullptr)
      st.zero();
    else
      st.template load<B, TR>(init, lane, wave);
  }
  if (nc > 0) {
    if (wave == TW) la_tables(g0, rows(0), tab[0], lane, scale);
    if (wave == 0) {  // the tiles past the diagonal
#pragma unroll
      for (int k = 0; k < kLaParts; ++k) {
        *reinterpret_cast<bf4*>(sP + k * kLaScores + (REV ? la_ptile<REV>(1, 0) : la_ptile<REV>(0, 1)) * 256 + 4 * lane) = bf4{};
        *reinterpret_cast<bf4*>(sP + k * kLaScores + (REV ? la_ptile<REV>(3, 2) : la_ptile<REV>(2, 3)) * 256 + 4 * lane) = bf4{};
      }
    }
  }
  la_landed<0>();
  // chunk n's terms over the waves, a barrier after they were left
  const auto total = [&](int n) {
    float x = sA[lane] + sA[CH + lane];
    if (NW == 4) x += sA[2 * CH + lane] + sA[3 * CH + lane];
    if (lane < rows(n)) (ROLE == kLaDq ? a.pa : a.pb)[(un.row0 + CH * at(n) + lane) * H + h] = x;
    if (lane < 16) {
      float y = sC[lane] + sC[16 + lane];
      if (NW == 4) y += sC[32 + lane] + sC[48 + lane];
      (ROLE == kLaDq ? a.ca : a.cb)[((size_t)unit * (a.segs.seg_tokens / CH) + at(n)) * 16 + lane] = y;
    }
  };
  const auto scores = [&](auto count, auto diag, int n0, const LaTab& t) {
    constexpr int N = decltype(count)::value;
    constexpr bool DIAG = decltype(diag)::value;
    f4 x[N];
    int io[N], jz[N];  // output's and Z's block
#pragma unroll
    for (int m = 0; m < N; ++m) {
      int i = n0 + m, j = i;
      if (!DIAG) la_tile_of(n0 + m, i, j);
      io[m] = REV ? j : i, jz[m] = REV ? i : j;
      x[m] = la_score<A>(sY, sX, ax, jz[m], io[m]) * la_decay_tile<!REV, DIAG>(t, i, j, lane, scale);
    }
#pragma unroll
    for (int m = 0; m < N; ++m) {
      if constexpr (SUMS && DIAG) {
        // the diagonal cancels between a and b: it is kept out of both and added to the output by itself
        const int u0 = la_new(c - 4 * g);
        if ((unsigned)u0 < 4u)
          sDiag[16 * io[m] + c] = u0 < 2 ? (u0 == 0 ? x[m][0] : x[m][1]) : (u0 == 2 ? x[m][2] : x[m][3]);
#pragma unroll
        for (int u = 0; u < 4; ++u) x[m][u] = u == u0 ? 0.f : x[m][u];
      }
      la_split4(sP + la_ptile<REV>(io[m], jz[m]) * 256 + 16 * c + 4 * g, kLaScores, x[m]);
    }
  };
  for (int n = 0; n < nc; ++n) {
    __builtin_amdgcn_s_setprio(1);
    __syncthreads();  // X and Z are there; Y, P and the terms of the chunk before are done with
    lx.load(Y, sx, lds + C::OFF_Y, wave);
    Y.next(sx);
    const bool more = n + 1 < nc;
    const LaTab& t = tab[n & 1];
    const int cn = at(n);
    if constexpr (ROLE == kLaDv) {
      if ((cn + 1) % kLaAnchor == 0 && n > 0)  // dS behind this chunk
        st.template store<B, TR>(a.aD + ((size_t)unit * a.anchors + cn / kLaAnchor) * (DK * DV), lane, wave);
    }
    f4 acc[2][4];
    st.read(sX, ax, t.eC, acc);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float f = (REV ? t.T : t.E)[16 * i + c];
      acc[0][i] *= f;
      acc[1][i] *= f;
    }
    bf8 z[2][2];
    la_zfrags(sZ, ax, z);
    la_landed<0>();
    __syncthreads();  // Y is there
    __builtin_amdgcn_s_setprio(2);
    u4v er[SUMS ? 4 : 1];
    bf8 zr[SUMS ? 4 : 1];  // Z as the output lies
    if constexpr (SUMS) {
      if (wave == 0 && n > 0) total(n - 1);
      const auto be = E.buf();
      E.next(sz);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        er[i] = __builtin_amdgcn_raw_buffer_load_b128(be, o0 + 16 * i * sz, 0, 0);  // in L1 or L2 since the tiles' loads
        zr[i] = la_ld16(sZ + ax.out + 16 * i * kLaRow);
      }
    }
    // scores: rows of the output by rows of Z, four of the latter a lane.  The first half of the waves
    // shares the tiles off the diagonal, the others have those on it, the last but one (and the
    // decays of the next chunk).  Up to three of a wave's tiles run side by side.
    const auto off = std::false_type{};
    const auto diagonal = std::true_type{};
    const auto one = std::integral_constant<int, 1>{};
    const auto two = std::integral_constant<int, 2>{};
    const auto three = std::integral_constant<int, 3>{};
    if constexpr (NW == 4) {
      if (wave < 2)
        scores(three, off, 3 * wave, t);
      else if (wave == 2)
        scores(three, diagonal, 0, t);
      else
        scores(one, diagonal, 3, t);
    } else {
      if (wave == 0) {
        scores(three, off, 0, t);
        scores(three, off, 3, t);
      } else {
        scores(two, diagonal, 0, t);
        scores(two, diagonal, 2, t);
      }
    }
    if (more && wave == TW) {
      la_tables(graw, rows(n + 1), tab[(n + 1) & 1], lane, scale);
      if (n + 2 < nc) graw = decay(n + 2);
    }
    if constexpr (SUMS) {
      // here, so that no wait for them stands behind the tiles' loads
#pragma unroll
      for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(er[i]));
    }
    __syncthreads();  // P is there; X and Z are done with
    __builtin_amdgcn_s_setprio(0);
    if (more) {
      X.next(sx);
      Z.next(sz);
      lx.load(X, sx, lds, wave);
      lz.load(Z, sz, lds + C::OFF_Z, wave);
    }
    bf8 ev[SUMS ? 4 : 1];
    if constexpr (SUMS) {
      float y = 0.f;  // what the state gives to a chunk's sum
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i % 2 == 0) {
          *reinterpret_cast<u4v*>(sS + sm) = er[i];
          *reinterpret_cast<u4v*>(sS + sm + 1024) = er[i + 1];
          la_wave_order();
        }
        ev[i] = la_ld16(sS + sr + 1024 * (i % 2));
#pragma unroll
        for (int u = 0; u < 4; ++u) y += acc[0][i][u] * (float)ev[i][u] + acc[1][i][u] * (float)ev[i][4 + u];
        if (i % 2) la_wave_order();
      }
      y += row_partner16(y, (lane & 16) != 0);
      y += row_partner32(y, lane >= 32);
      if (g == 0) sC[16 * wave + c] = y;
    }
    const __bf16* pf = sP + 256 * (g >> 1) + 16 * c + 8 * (g & 1);
#pragma unroll
    for (int q = kLaParts - 1; q >= 0; --q)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (REV ? (kb == 1 || i < 2) : (kb == 0 || i >= 2)) {
            const bf8 p = ld8(pf + q * kLaScores + 256 * la_ptile<REV>(i, 2 * kb));
#pragma unroll
            for (int k = 0; k < 2; ++k) acc[k][i] = mma(z[k][kb], p, acc[k][i]);
          }
    float sum[SUMS ? BLOCKS : 1];
    const auto bo = out.buf();
    out.next(so);
#pragma unroll
    for (int i0 = 0; i0 < BLOCKS; i0 += 2) {
      if constexpr (SUMS) {
#pragma unroll
        for (int i = i0; i < i0 + 2; ++i) {
          float x = 0.f;
#pragma unroll
          for (int u = 0; u < 4; ++u) x += acc[0][i][u] * (float)ev[i][u] + acc[1][i][u] * (float)ev[i][4 + u];
          sum[i] = x;
          const float d = sDiag[16 * i + c];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            acc[0][i][u] += d * (float)zr[i][u];
            acc[1][i][u] += d * (float)zr[i][4 + u];
          }
        }
      }
      if constexpr (PART) {
#pragma unroll
        for (int i = i0; i < i0 + 2; ++i)
#pragma unroll
          for (int k = 0; k < 2; ++k)
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4v, acc[k][i]), bo,
                                                   (16 * i + c) * so + 4 * (32 * wave + 8 * g + 4 * k), 0, 0);
      } else {
#pragma unroll
        for (int i = i0; i < i0 + 2; ++i) {
          bf8 v;
#pragma unroll
          for (int u = 0; u < 4; ++u) v[u] = (__bf16)acc[0][i][u], v[4 + u] = (__bf16)acc[1][i][u];
          *reinterpret_cast<bf8*>(sS + sr + 1024 * (i - i0)) = v;
        }
        la_wave_order();
#pragma unroll
        for (int i = i0; i < i0 + 2; ++i)
          __builtin_amdgcn_raw_buffer_store_b128(*reinterpret_cast<const u4v*>(sS + sm + 1024 * (i - i0)), bo, o0 + 16 * i * sz, 0, 0);
        la_wave_order();
      }
    }
    if constexpr (SUMS) sA[wave * CH + lane] = la_sum4(sum);
    st.update(sY, ax, z, REV ? t.E : t.T, lane);
    if constexpr (ROLE == kLaDq) {
      if (more ? (n + 1) % kLaAnchor == 0 : un.last && a.dST != nullptr)
        st.template store<B, TR>(a.aS + ((size_t)unit * a.anchors + n / kLaAnchor) * (DK * DV), lane, wave);
    }
    la_landed<STORES>();  // behind the tiles' loads lie the output's stores, at an anchor more
  }
  if constexpr (SUMS) {
    __syncthreads();
    if (wave == 0 && nc > 0) total(nc - 1);
  }
  if constexpr (ROLE == kLaO) {
    if (un.last && a.ST) st.template store<B, TR>(a.ST + ((size_t)un.seq * H + h) * (DK * DV), lane, wave);
  }
  if constexpr (ROLE == kLaDv) {
    if (un.first && a.dS0) st.template store<B, TR>(a.dS0 + ((size_t)un.seq * H + h) * (DK * DV), lane, wave);
  }
}

template <int DK, int DV>
__global__ __launch_bounds__(2 * DV, 2) void la_scan_fwd_kernel(LaScanArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  la_scan<DK, DV, kLaO, false>(a, blockIdx.x, smem);
}
// The gradients side by side.
template <int DK, int DV, bool GROUPED>
__global__ __launch_bounds__(2 * (DK > DV ? DK : DV), 2) void la_scan_bwd_kernel(LaScanArgs a) {
  extern __shared__ __align__(16) unsigned char smem[];
  int unit, role;
  if (!la_slot(blockIdx.x, a.segs.nslot * a.geo.H, unit, role)) return;
  if (role == kLaDq)
    la_scan<DK, DV, kLaDq, GROUPED>(a, unit, smem);
  else if (role == kLaDk)
    la_scan<DK, DV, kLaDk, GROUPED>(a, unit, smem);
  else
    la_scan<DK, DV, kLaDv, GROUPED>(a, unit, smem);
}

// ---- the decays' gradient --------------------------------------------------
// With a_t = q_t . dq_t and b_t = v_t . dv_t, dg_t is <S, dS> behind any later token plus the sum
// of a - b from t up to it, taken in 64 bits.  Where t and that token are in one chunk, a and b
// count without the diagonal's part, the same in both; chunks between count with what their a and
// b have from the states alone, for pairs of tokens inside a chunk cancel, and what would be left
// of them is rounding (1.8e-6 of dg at 4096 tokens of mean log-decay -0.13, against 0.8e-6).  A
// stretch of up to kLaAnchor chunks from one <S, dS> a workgroup, a chunk a wave, a token a lane.
template <int DK, int DV>
__global__ __launch_bounds__(kLaAnchor * CH) void la_dg_kernel(LaScanArgs a) {
  constexpr int NTHR = kLaAnchor * CH;
  __shared__ double part[NTHR / 64], phi[NTHR / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int H = a.geo.H, unit = blockIdx.x / a.anchors, k = blockIdx.x % a.anchors, h = unit % H;
  LaUnit un;
  if (!la_unit(a.segs, a.geo.T, unit / H, un)) return;
  const int t0 = k * NTHR, len = min(NTHR, un.len - t0);
  if (len <= 0) return;
  double x = 0.0;
  const size_t row = un.row0 + t0 + tid;
  if (tid < len) x = (double)a.pa[row * H + h] - a.pb[row * H + h];
  double y = 0.0;
  if (wave * CH < len && lane < 16) {
    const size_t i = ((size_t)unit * (a.segs.seg_tokens / CH) + k * kLaAnchor + wave) * 16 + lane;
    y = (double)a.ca[i] - a.cb[i];
  }
  double f = 0.0;
  // S and dS behind the stretch: left by the scans, or behind the segment those that came before them
  const bool end = t0 + len == un.len;
  if (!(un.last && end && a.dST == nullptr)) {
    const float* S = end && !un.last ? a.S + (size_t)unit * (DK * DV) : a.aS + (size_t)blockIdx.x * (DK * DV);
    const float* D = !end      ? a.aD + (size_t)blockIdx.x * (DK * DV)
                     : un.last ? a.dST + ((size_t)un.seq * H + h) * (DK * DV)
                               : a.dS + ((size_t)unit + H) * (DK * DV);
    for (int e = 4 * tid; e < DK * DV; e += 4 * NTHR) {
      const float4 p = ld4(S + e), q = ld4(D + e);
      f += (double)(p.x * q.x + p.y * q.y) + (double)(p.z * q.z + p.w * q.w);
    }
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double z = __shfl_down(x, o);
    if (lane + o < 64) x += z;
    f += __shfl_xor(f, o);
    y += __shfl_xor(y, o);
  }
  if (lane == 0) {
    part[wave] = y;
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
  constexpr size_t lds = 2 * (la_bytes(DK) + la_bytes(DV) + sizeof(LaTab));
  const auto kernel = rev ? la_segstate_kernel<DK, DV, true> : la_segstate_kernel<DK, DV, false>;
  return la_launch(kernel, (unsigned)(a.segs.nslot * a.geo.H), 2 * DV, lds, a, st);
}

hipError_t launch_la_segcombine(const LaScanArgs& a, int size, bool rev, hipStream_t st) {
  hipLaunchKernelGGL(la_segcombine_kernel, dim3((unsigned)(a.segs.nseq * a.geo.H * (size / 1024))), dim3(256), 0, st, a, size,
                     rev ? 1 : 0);
  return hipGetLastError();
}

template <int DK, int DV>
hipError_t launch_la_scan_fwd(const LaScanArgs& a, hipStream_t st) {
  return la_launch(la_scan_fwd_kernel<DK, DV>, (unsigned)(a.segs.nslot * a.geo.H), 2 * DV, LaCfg<DK, DV, kLaO>::LDS, a, st);
}

template <int DK, int DV>
hipError_t launch_la_scan_bwd(const LaScanArgs& a, hipStream_t st) {
  constexpr size_t lq = LaCfg<DK, DV, kLaDq>::LDS, lk = LaCfg<DK, DV, kLaDk>::LDS, lv = LaCfg<DK, DV, kLaDv>::LDS;
  constexpr size_t lds = lq > lk ? (lq > lv ? lq : lv) : (lk > lv ? lk : lv);
  const int units = a.segs.nslot * a.geo.H;
  const auto kernel = a.Pq ? la_scan_bwd_kernel<DK, DV, true> : la_scan_bwd_kernel<DK, DV, false>;
  hipError_t e = la_launch(kernel, la_grid(units), 2 * (DK > DV ? DK : DV), lds, a, st);
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

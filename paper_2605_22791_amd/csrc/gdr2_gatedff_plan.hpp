// Gated feed-forward block (include/gdr2_gatedff.h): how a product is laid out on the card.  Host
// arithmetic alone, with nothing of HIP in it, so that it can be compiled and checked without a GPU.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstddef>
#include <cstdint>

namespace gdr2 {

// Products C = A B, A (M, K), B (K, N), fp32 accumulation.  An operand lies with its sum along the rows
// of memory ("rows") or across them ("columns"):
//     FF_ROWS     A (M, K), B^T (N, K)     x Wg^T, x Wu^T, h Wd^T
//     FF_MIXED    A (M, K), B (K, N)       dy Wd, dg Wg + du Wu
//     FF_COLUMNS  A^T (K, M), B (K, N)     dg^T x, du^T x, dy^T h
enum FfForm : int { FF_ROWS = 0, FF_MIXED = 1, FF_COLUMNS = 2 };
// What becomes of C:
//     FF_STORE  rounded and stored
//     FF_GATE   B is a pair, C a pair g, u: h = act(g) u, and g, u themselves where asked for
//     FF_GRAD   C is dh: dg and du from it and the stored g, u
enum FfEnd : int { FF_STORE = 0, FF_GATE = 1, FF_GRAD = 2 };

constexpr int kFfCUs = 256;
constexpr int kFfStep = 128;  // bytes of a row that one step takes
constexpr int ff_waves_m(int bm) { return bm == 64 ? 2 : bm / 64; }  // waves along M, two along N
constexpr int ff_threads(int bm) { return 128 * ff_waves_m(bm); }

// How a call is laid out: the tile size and what the tiles left over are cut into, by the time that they
// would take, in us: rounds of as many tiles as there are places, a part of a round for those that are
// cut, and parts' way through memory and a launch.  Rates measured: 256 x 256 tiles 1.2 PFLOP/s in bf16, 128 x 128
// 1.0, 64 x 64 (FF_GATE: 64 x 128) 0.6; in fp32 0.1 either way.  Places are taken as one, two and four a
// CU; registers and LDS have room for one, two, and five of 64 x 64, three of 64 x 128.  Against each size by itself, 18 bf16
// and 7 fp32 problems of 64 to 16000 rows, the choice was the best or within 9 % of it, both ways.
struct FfPlan {
  int bm, bn, slots;
  int tm[2], tn[2], tiles, full, split;
  double us;
};
// sizes of one or two products with the same sum
struct FfSize {
  int64_t M[2], N[2], K;
  int pairs;
};
inline FfPlan ff_plan(int end, const FfSize& z, int E, int bm, int bn, int a_cu, double rate) {
  FfPlan q{};
  q.bm = bm;
  q.bn = bn;
  q.slots = a_cu * kFfCUs;
  int64_t tiles = 0;
  for (int k = 0; k < 2; ++k) {
    const int bnc = end == FF_GATE ? bn / 2 : bn;
    q.tm[k] = (int)((z.M[k] + bm - 1) / bm);
    q.tn[k] = (int)((z.N[k] + bnc - 1) / bnc);
    tiles += (int64_t)q.tm[k] * q.tn[k];
  }
  q.tiles = (int)tiles;
  const int64_t steps = (z.K + kFfStep / E - 1) / (kFfStep / E) * z.pairs, left = tiles % q.slots;
  const double tile = 2e-9 * bm * bn * (double)(steps * (kFfStep / E)) / (rate / q.slots);  // us; rate in PFLOP/s
  q.full = q.tiles;
  q.split = 1;
  q.us = tile * (double)((tiles + q.slots - 1) / q.slots);
  for (int64_t split = 2; left > 0 && split <= q.slots / left && split <= steps / 4; ++split) {
    const double us = tile * ((double)(tiles / q.slots) + 1.0 / split) + 4.0 + (double)left * split * bm * bn * 8.0 / 4.8e6;
    if (us < q.us) {
      q.us = us;
      q.split = (int)split;
      q.full = (int)(tiles - left);
    }
  }
  // A launch has less than 2^32 threads.  For the up to 2^36 values of a product, tiles of 128 x 64 and larger ones
  // always have; 64 x 64 ones come to it near that end, with 32 columns (FF_GATE in fp32) from half of it.
  if (((double)q.full + (double)(q.tiles - q.full) * q.split) * ff_threads(bm) >= 4294967296.0) q.us = HUGE_VAL;
  return q;
}
inline FfPlan ff_choose(int end, const FfSize& z, int E) {
  const FfPlan mid = ff_plan(end, z, E, 128, 128, 2, E == 2 ? 1.0 : 0.1);
  const FfPlan small = ff_plan(end, z, E, 64, E == 2 && end == FF_GATE ? 128 : 64, 4, E == 2 ? 0.6 : 0.1);
  const FfPlan& best = small.us < mid.us ? small : mid;
  if (E == 4) return best;
  const FfPlan large = ff_plan(end, z, E, 256, 256, 1, 1.2);
  return best.us < large.us ? best : large;
}
inline size_t ff_part_bytes(const FfPlan& q) { return (size_t)(q.tiles - q.full) * q.split * q.bm * q.bn * 4; }

// Up to 64 rows; wide weights in bf16 up to 32, for every workgroup reads all of A.  A forward of 33, 48, 64
// rows: 4096 -> 11008 (45 M weights) 82, 95, 104 us, 85 in tiles; 2048 -> 5504 (11 M) 33, 36, 40, and 37; 1024 -> 2816
// 15 to 17, and 27.  Nothing between 11 M and 45 M was measured; the bound keeps 2048 -> 5504 whole, which gains up to 48
// rows and loses 3 us at 64.  fp32 64 rows of 4096 -> 11008 263, and 349.  (A saving forward gives the bits of the backward's own g and u.)
inline bool ff_thin_rows(int64_t M, int64_t N, int64_t K, int E) { return M <= (E == 2 && N * K > 12000000 ? 32 : 64); }

}  // namespace gdr2

// Gated linear recurrence (include/gdr2_gatedrec.h): the launch interface between the C ABI and
// the kernels.
#pragma once

#include "gdr2_kernels.hpp"

namespace gdr2 {

constexpr int kRecWaves = 8;    // waves of a workgroup
constexpr int kRecBlock = 64;   // tokens of a workgroup of the backward, which starts from the states between them
constexpr int kRecTile = 128;   // and of the forward, or half of it

// Channels of a workgroup: two a lane where their pairs are aligned and fill a wave.
inline int rec_channels(int D) { return D % 2 == 0 && D > 64 ? 128 : 64; }
// groups of channels, and workgroups of kRecBlock tokens of them
inline int rec_groups(int D) { return (D + rec_channels(D) - 1) / rec_channels(D); }
inline int64_t rec_blocks(int64_t rows, int D) { return (rows + kRecBlock - 1) / kRecBlock * rec_groups(D); }
// How many times eight tiles a tile looks back over for a state: kRecFar (half as many with two channels a
// lane, for the LDS) where the chain is long beside the channels and has few workgroups that could hide it:
// 65536 tokens of 64 channels 32 and 53 us each way (176 and 187 with eight tiles), 16384 of 512 31 and 61 (46
// and 68); 4096 of 2048, below the bound, would take 27 and 54 (29 and 43), 2 x 8192 of 4096 153 and 364 (154 and 267).
constexpr int kRecFar = 16;
// (len: the tokens of a sequence; of a packed batch, whose lengths are on the device, in the mean: one long sequence
// among many short ones of few channels gets the look over eight tiles: 63536 tokens behind
// 200 sequences of ten, 64 channels, 185 and 186 us, where alone they take 36 and 64)
inline bool rec_far(int len, int64_t rows, int D) {
  return len / kRecBlock >= 8 * rec_groups(D) && rec_blocks(rows, D) <= 4096;
}
// Tokens of a forward workgroup.  Tiles of 128 make a shorter chain (65536 tokens of 2048 channels: 257 us,
// 334 with 64); where the chain is not what counts, eight workgroups a CU are needed to hide their
// waits (9 packed prompts of 8192 tokens, four a CU with 128: 62 us, 57 with 64).
inline int rec_tile(int len, int64_t rows, int D) {
  return rec_far(len, rows, D) || rec_blocks(rows, D) >= 4096 ? kRecTile : kRecTile / 2;
}

// What tiles hand to the tiles behind them, in the order in which they are taken: pref (tiles, D) the
// state behind a tile, agg (tiles, D, 2) the factor and the addend that a tile takes it there by.
// All ones: not there yet.
struct RecChain {
  float* pref;
  float* agg;
  uint32_t* ticket;  // the next tile to take, a word in 16 for every group of channels; zero before the launch
};

template <typename T>
struct RecArgs {
  const T *x, *i;       // i nullable
  const float *g, *h0;  // h0 nullable
  const int32_t* cu;    // packed: nseq + 1 offsets; else NULL
  T* o;                 // nullable: the states alone
  float* hT;            // nullable
  float* states;        // nullable: behind every kRecBlock tokens, (blocks, D)
  RecChain chain;
  int nseq, len;        // sequences; tokens of one (fixed length) or of the batch
  int rows, D, normalize;
};

template <typename T>
struct RecBwdArgs {
  const T *x, *i, *dout;
  const float *g, *h0, *dhT;
  const float* states;  // behind every kRecBlock tokens, (blocks, D)
  const int32_t* cu;
  T *dx, *di;
  float *dg, *dh0;
  RecChain chain;
  int nseq, len;
  int rows, D, normalize;
};

template <typename T>
struct RecStepArgs {
  const T *x, *i;
  const float* g;
  const int32_t* cu;
  T* o;
  float* h;
  int nseq, len;
  int D, normalize;
};

template <typename T>
hipError_t launch_rec_fwd(const RecArgs<T>& a, hipStream_t st);
template <typename T>
hipError_t launch_rec_bwd(const RecBwdArgs<T>& a, hipStream_t st);
template <typename T>
hipError_t launch_rec_step(const RecStepArgs<T>& a, hipStream_t st);
// `words` 16-byte words of all ones, but zero the first `zeros`: a chain as a launch finds it
struct RecClear {
  void* p;
  size_t words, zeros;
};
hipError_t launch_rec_clear(const RecClear& x, const RecClear& y, hipStream_t st);

}  // namespace gdr2

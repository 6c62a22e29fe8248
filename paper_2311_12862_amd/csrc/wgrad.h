// Device-side pieces shared by the weight-gradient kernels that walk pair lists (wgrad.hip, wgrad_q8.hip): their arguments, the
// pieces of the list, and where a staged batch stands in LDS.
#pragma once
#include "common.h"
#include "lds_tiles.h"

namespace spc {

struct Split {
  int pieces;    // at most so many (grid, partial tiles)
  int length;    // pairs of a piece as asked for, or 0: chosen by
  float weight;  // sqrt(time of a pair in a piece / time of a partial tile), and at least
  int unit;      // so many
  int per_round;  // pieces that make one workgroup per CU
};

struct WgradParams {
  const void* feats;   // [n_in][C_in]
  const void* dout;    // [n_out][C_out]
  const int2* pairs;   // (n, j), offset-major
  const int* seg;      // [V+1]
  float* partial;      // [piece][C_in][C_out]
  unsigned feats_bytes, dout_bytes, pairs_bytes;
  int C_in, C_out, V;
  Split split;
  const unsigned char* exps;  // feats is the data of a checkpoint, these its exponents (wgrad_q8.hip)
  unsigned exps_bytes;
};

// wgrad_q8.hip: the kernel for one tile size (16-bit types); SPCONV_EINVAL for a tile it does not have
int wgrad_q8_launch(const WgradParams& p, int tile, spconv_dtype dtype, dim3 grid, hipStream_t st);

namespace {

constexpr unsigned kNoRow = 0xFFFFC000u;  // beyond every buffer

// Pairs per piece; computed by every workgroup, as the pair count may only be known on the device.
// g pieces take time ~ pairs / g (a workgroup's serial part) + g * (a tile written and read): least at g ~ sqrt(pairs).
// Long pieces then go down to whole rounds of one workgroup per CU, each offset's last piece counted: two workgroups of a CU
// gather at half the rate each, and the launch waits for the CUs that have one more (421k pairs 128 -> 128, 410 pieces 47.2 us,
// 249 pieces 40.9; 256 -> 128, 604 workgroups 80.0, 510 69.1).  Not where that takes too many of them (271k pairs 256 ->
// 128, 496 workgroups 47.9 us, 256 57.1), nor where pieces are short, so that their start is what counts (127k pairs 256
// -> 128: 32.9 us, in one round 35.3).
__device__ __forceinline__ int split_length(const Split& s, int pairs, int V) {
  if (s.length > 0) return s.length;
  int g = min(s.pieces - V, (int)(s.weight * sqrtf((float)pairs)) + 1);
  const int whole = (g + V) / s.per_round * s.per_round - V;
  const int least = s.per_round == 256 ? g / 2 : g - g / 4;  // (a single column of tiles: rounds are finer)
  if (whole >= least && pairs / g >= 900) g = whole;
  return max(s.unit, (pairs + g - 1) / g);
}
// Lane k < V of a wave: the pieces of the offsets before k, and of k.
struct Pieces {
  int before, count;
};
__device__ __forceinline__ Pieces pieces_of(const Split& s, int bound, int V, int lane) {  // bound: lane k <= V holds seg[k]
  const int length = split_length(s, __builtin_amdgcn_readlane(bound, V), V);
  const int pairs = __shfl_down(bound, 1) - bound;
  const int count = lane < V ? (pairs + length - 1) / length : 0;
  int incl = count;
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up(incl, o);
    if (lane >= o) incl += up;
  }
  return {incl - count, count};
}

template <int N> __device__ __forceinline__ void wait_loads() {  // all but the N youngest; own LDS reads are done as well
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"i"(N) : "memory");
}

// Where chunk c (16 bytes) of row r of a staged batch stands.  16-bit types: the transposing read of 32 lanes takes rows
// r..r+3 and r+8..r+11 at one 32-byte block each; fp32: four rows at one 64-byte block.  Eight (four) blocks span
// the LDS banks, so the block number is XORed (six blocks: rotated) by the row.
template <int E, int CPR> __device__ __forceinline__ int chunk_block_shift(int r) {
  if constexpr (E == 4) return CPR >= 16 ? (r & 3) : (r >> 1) & 1;
  else if constexpr (CPR == 4) return (r >> 3) & 1;
  else if constexpr (CPR == 8) return ((r >> 1) & 1) | (((r >> 3) & 1) << 1);
  else if constexpr (CPR == 12) return (r >> 3) & 1;
  else return (r & 3) | (((r >> 3) & 1) << 2);
}
// block b of row r stands at block place_of(b), and place q holds block block_at(q)
template <int E, int CPR> __device__ __forceinline__ int place_of(int b, int r) {
  if constexpr (E == 2 && CPR == 12) {
    const int q = b + chunk_block_shift<E, CPR>(r);
    return q >= 6 ? q - 6 : q;
  } else {
    return b ^ chunk_block_shift<E, CPR>(r);
  }
}
template <int E, int CPR> __device__ __forceinline__ int block_at(int q, int r) {
  if constexpr (E == 2 && CPR == 12) {
    const int b = q - chunk_block_shift<E, CPR>(r);
    return b < 0 ? b + 6 : b;
  } else {
    return q ^ chunk_block_shift<E, CPR>(r);
  }
}

}  // namespace
}  // namespace spc

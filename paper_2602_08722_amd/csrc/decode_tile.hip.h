// What the attention kernels for a few tokens over a cache in pages share (paged_decode.hip, cross_few.hip): how a wave's tile of rows lies in LDS.
#pragma once
#include <type_traits>

#include "pages.hip.h"

namespace quoka {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef s16x4 __attribute__((address_space(3))) * tr_ptr;

constexpr int kPdTile = 32;        // list slots a wave handles at a time

template <int D, bool FP8, int WAVES>
struct PdTile {
  static constexpr int KS = D / 16, DB = D / 32;
  static constexpr int LPR = D * (FP8 ? 1 : 2) / 16;   // lanes per row
  static constexpr int NLD = kPdTile * LPR / 64;       // rows of a group of lanes
  static constexpr int LD = D + 8;         // K rows in LDS: 16 bytes of padding (conflict-free 16-byte reads)
  static constexpr int LDV = D + 32;       // V rows: 64 bytes apart modulo 256 (transposing reads)
  // The first row of a group of lanes.  8-bit rows: eight lanes of a store to LDS have to cover 128 bytes, and are one row (D = 64: two,
  // whose places of K are 64 bytes apart modulo 128).  A lane's two pieces of K lie half a row apart (the contraction index may
  // be permuted: Q follows), and of V side by side, the other way round in the upper half of a row (D = 64: in every other four rows).
  __device__ static __forceinline__ int first_row(int group) {
    if constexpr (!FP8) return group * NLD;
    if constexpr (D == 128) return group * NLD;
    return 4 * (group & 7) + 2 * (group >> 3);
  }
  static constexpr size_t kKBytes = (size_t)kPdTile * LD * 2;
  static constexpr size_t kWaveBytes = kKBytes + (size_t)kPdTile * LDV * 2;
  static constexpr int kRec = 32 * (D + 2);   // floats of a block's partial: O[32][D], m[32], l[32]
  static constexpr int LDO = D + 4;        // LDS pitch of a wave's output rows (floats)
  static constexpr size_t kMergeBytes = (size_t)WAVES * 32 * (LDO + 3) * 4;
  static constexpr size_t kLdsBytes = WAVES * kWaveBytes > kMergeBytes ? WAVES * kWaveBytes : kMergeBytes;
};

// Value of lane `i` of the caller's group of W lanes (i folds to a constant).
template <int W>
__device__ __forceinline__ uint32_t group_lane(uint32_t v, int i) {
  if constexpr (W == 16) return row16_lane(v, i);
  if constexpr (W == 8) {
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xF, 0xF, false);   // row_ror:8: the other half's
    const uint32_t lower_i = row16_lane(v, i), upper_i = row16_lane(hi, i);   // lanes i and i + 8 of the row of 16
    return (threadIdx.x & 8) != 0 ? upper_i : lower_i;
  }
  switch (i) {   // quad_perm
    case 0: return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x00, 0xF, 0xF, true);
    default: return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x55, 0xF, 0xF, true);
  }
}

}  // namespace quoka

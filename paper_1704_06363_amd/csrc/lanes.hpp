// lanes.hpp -- what the lanes of a wave do together: compaction through ballots, order statistics, sorted lists
// of (value, index) keys with one key per lane.
#pragma once
#include "common.hpp"

namespace hmoe {

// Set bits of `mask` below this lane.
__device__ __forceinline__ int lanes_below(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// Orders a wave's LDS writes before its later reads by other lanes of the same wave.
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The m-th largest over the lanes of x (with multiplicity), m <= 16: each row of 16 lanes is sorted
// (bitonic, each merge starting with the mirrored pair, so that every step keeps the larger value
// in the lower lane), then the 16 largest of two rows are the larger ones of one row and the other
// reversed, sorted again.  A step is a lane move and a median with +inf or -inf: about 50
// instructions (130 in a full sort by selects of minima and maxima).  NaN counts as -inf: the median of two
// NaN and +inf is +inf, which no lane holds.
__device__ __forceinline__ float mth_lane_value(float x, int m, int l) {
  x = fmaxf(x, -INFINITY);
  const auto step = [&](float y, int bit) {
    x = __builtin_amdgcn_fmed3f(x, y, (l & bit) ? -INFINITY : INFINITY);  // the smaller : the larger
  };
  const auto xor1 = [&] { step(dpp<0xB1>(x), 1); };           // quad_perm [1,0,3,2]
  const auto xor2 = [&] { step(dpp<0x4E>(x), 2); };           // quad_perm [2,3,0,1]
  const auto xor4 = [&] { step(dpp<0x1B>(dpp<0x141>(x)), 4); };  // half mirror, quad mirror
  const auto xor8 = [&] { step(dpp<0x128>(x), 8); };          // row_ror:8
  xor1();
  step(dpp<0x1B>(x), 2);  // quad mirror
  xor1();
  step(dpp<0x141>(x), 4);  // half mirror
  xor2();
  xor1();
  step(dpp<0x140>(x), 8);  // row mirror
  xor4();
  xor2();
  xor1();
  // rows 0 and 2 take the best of rows 0, 1 and 2, 3
  unsigned y = __float_as_uint(dpp<0x140>(x));
  x = fmaxf(x, __uint_as_float(__builtin_amdgcn_permlane16_swap(y, y, false, false)[1]));
  xor8();
  xor4();
  xor2();
  xor1();
  // row 0 the best of all
  y = __float_as_uint(dpp<0x140>(x));
  x = fmaxf(x, __uint_as_float(__builtin_amdgcn_permlane32_swap(y, y, false, false)[1]));
  xor8();
  xor4();
  xor2();
  xor1();
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), m - 1));
}

// ------------------------------------------------------------------ keys of (value, index)

// 64-bit keys whose order is (value descending, index ascending) with the largest first: the value's
// bits made to sort as integers, above the index's complement.  -0 counts as +0.  NaN ranks
// last; 0 is no entry and ranks after everything.
__device__ __forceinline__ uint32_t sortable(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return x != x ? 0u : (u & 0x80000000u ? ~u : u | 0x80000000u);
}
__device__ __forceinline__ uint64_t rank_key(float x, uint32_t index) {
  return ((uint64_t)sortable(x) << 32) | (uint32_t)~index;
}
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t s = (uint32_t)(k >> 32);
  return __uint_as_float(s & 0x80000000u ? s & 0x7fffffffu : ~s);
}
__device__ __forceinline__ uint32_t key_index(uint64_t k) { return ~(uint32_t)k; }
constexpr uint32_t kKeyMinusInf = 0x007fffffu;  // sortable(-inf)

// v of the lane whose number differs in bit D, in registers.
template <int D>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v) {
  if constexpr (D == 1) return __builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true);
  if constexpr (D == 2) return __builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true);
  if constexpr (D == 4) {  // the eight lanes mirrored, then each four of them
    const int h = __builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, true);
    return __builtin_amdgcn_update_dpp(0, h, 0x1B, 0xf, 0xf, true);
  }
  if constexpr (D == 8) return __builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, true);
  if constexpr (D == 16) {
    const auto x = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return (threadIdx.x & 16) ? x[0] : x[1];
  }
  if constexpr (D == 32) {
    const auto x = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return (threadIdx.x & 32) ? x[0] : x[1];
  }
}
template <int D>
__device__ __forceinline__ uint64_t lane_xor(uint64_t v) {
  return ((uint64_t)lane_xor<D>((uint32_t)(v >> 32)) << 32) | lane_xor<D>((uint32_t)v);
}
// One step of a bitonic network: lanes whose number lacks bit D keep the larger key of the pair where
// `desc`, the smaller one otherwise.
template <int D>
__device__ __forceinline__ void pair_step(uint64_t& k, bool desc) {
  const uint64_t o = lane_xor<D>(k);
  const bool larger = ((threadIdx.x & D) == 0) == desc;
  k = (o > k) == larger ? o : k;
}
template <int D>
__device__ __forceinline__ void merge_steps(uint64_t& k, bool desc) {
  pair_step<D>(k, desc);
  if constexpr (D > 1) merge_steps<D / 2>(k, desc);
}
// The wave's 64 keys sorted over the lanes, descending or ascending.  Entered by whole waves.
__device__ __forceinline__ void wave_sort(uint64_t& k, bool desc) {
  const int l = threadIdx.x & 63;
  merge_steps<1>(k, (l & 2) == 0);
  merge_steps<2>(k, (l & 4) == 0);
  merge_steps<4>(k, (l & 8) == 0);
  merge_steps<8>(k, (l & 16) == 0);
  merge_steps<16>(k, (l & 32) == 0);
  merge_steps<32>(k, desc);
}
// best (descending) becomes the 64 largest of itself and the wave's other 64 keys.
__device__ __forceinline__ void wave_merge(uint64_t& best, uint64_t other) {
  wave_sort(other, false);
  best = other > best ? other : best;  // descending against ascending: the larger halves, bitonic
  merge_steps<32>(best, true);
}
__device__ __forceinline__ uint64_t lane_value(uint64_t v, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)v, lane), hi = __builtin_amdgcn_readlane((uint32_t)(v >> 32), lane);
  return ((uint64_t)hi << 32) | lo;
}

}  // namespace hmoe

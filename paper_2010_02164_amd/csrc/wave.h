// Cross-lane combines within one 64-lane wave without going through LDS
// (gfx950). A full combine takes six stages; stage s pairs each lane with
// one partner so that after stages 0..s every lane holds the combination of
// 2^(s+1) lanes:
//   0: lane ^ 1            (DPP quad_perm [1,0,3,2])
//   1: lane ^ 2            (DPP quad_perm [2,3,0,1])
//   2: 7 - lane within 8   (DPP row_half_mirror)
//   3: 15 - lane within 16 (DPP row_mirror)
//   4: rows 0 <-> 1, 2 <-> 3 of 16 lanes (v_permlane16_swap)
//   5: lanes 0-31 <-> 32-63             (v_permlane32_swap)
// Stages 0-3 hand each lane its partner's value; stages 4-5 hand both lanes
// of a pair the same two values (first: the even row / low half, second:
// the odd row / high half), so a combine that is symmetric in its operands
// gives identical results in every lane.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sb {

template <int S>
__device__ __forceinline__ uint32_t dpp_partner(uint32_t x) {
  static_assert(S >= 0 && S <= 3, "DPP stages are 0..3");
  constexpr int ctrl = S == 0 ? 0xB1 : S == 1 ? 0x4E : S == 2 ? 0x141 : 0x140;
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, 0xF, 0xF, false);
}

// Stages 4 (rows) and 5 (halves): the pair's two values, even/low first.
template <int S>
__device__ __forceinline__ void swap_pair(uint32_t x, uint32_t &first, uint32_t &second) {
  static_assert(S == 4 || S == 5, "swap stages are 4 and 5");
  if constexpr (S == 4) {
    const auto p = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    first = p[0];
    second = p[1];
  } else {
    const auto p = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    first = p[0];
    second = p[1];
  }
}

// Stage S applied to a 64-bit value: (own-or-first, partner-or-second).
template <int S>
__device__ __forceinline__ void stage64(unsigned long long x, unsigned long long &a, unsigned long long &b) {
  const uint32_t lo = (uint32_t)x, hi = (uint32_t)(x >> 32);
  if constexpr (S <= 3) {
    a = x;
    b = ((unsigned long long)dpp_partner<S>(hi) << 32) | dpp_partner<S>(lo);
  } else {
    uint32_t l0, l1, h0, h1;
    swap_pair<S>(lo, l0, l1);
    swap_pair<S>(hi, h0, h1);
    a = ((unsigned long long)h0 << 32) | l0;
    b = ((unsigned long long)h1 << 32) | l1;
  }
}

template <int S>
__device__ __forceinline__ void stage32(uint32_t x, uint32_t &a, uint32_t &b) {
  if constexpr (S <= 3) {
    a = x;
    b = dpp_partner<S>(x);
  } else {
    swap_pair<S>(x, a, b);
  }
}

// Sums over the lanes up to each, through the lanes' own paths (a shuffle
// through LDS takes about 130 cycles).
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned long long from_before(unsigned long long v) {   // 0 where nothing comes
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(v >> 32), CTRL, ROWS, 0xF, false);
  return ((unsigned long long)hi << 32) | lo;
}
__device__ __forceinline__ unsigned long long wave_scan(unsigned long long v) {   // inclusive
  v += from_before<0x111, 0xF>(v);   // within 16 lanes: from 1, 2, 4, 8 before
  v += from_before<0x112, 0xF>(v);
  v += from_before<0x114, 0xF>(v);
  v += from_before<0x118, 0xF>(v);
  v += from_before<0x142, 0xA>(v);   // the last of the first and third 16 to the next
  v += from_before<0x143, 0xC>(v);   // the last of the first 32 to the others
  return v;
}

}  // namespace sb

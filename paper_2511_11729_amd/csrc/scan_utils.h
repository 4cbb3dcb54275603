// Sums and scans over the lanes of a wave.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

namespace harli {

typedef unsigned long long u64;

// Lane moves of the vector ALU (not of LDS): a step of a scan adds what the lanes `CTRL` below hold; lanes without one add zero.
template <int CTRL, int ROWS, typename T>
__device__ __forceinline__ T lanes_below(T v) {
  if constexpr (sizeof(T) == 8) {
    const u64 u = __builtin_bit_cast(u64, v);
    const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)u, CTRL, ROWS, 0xf, false);
    const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)(u >> 32), CTRL, ROWS, 0xf, false);
    return __builtin_bit_cast(T, (u64)hi << 32 | lo);
  } else {
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
  }
}
template <typename T>
__device__ __forceinline__ T row_scan(T v) {  // inclusive, inside rows of 16 lanes
  v += lanes_below<0x111, 0xf>(v);
  v += lanes_below<0x112, 0xf>(v);
  v += lanes_below<0x114, 0xf>(v);
  v += lanes_below<0x118, 0xf>(v);
  return v;
}
template <typename T>
__device__ __forceinline__ T wave_scan(T v) {  // inclusive
  v = row_scan(v);
  v += lanes_below<0x142, 0xa>(v);  // the row before, to the second and fourth
  v += lanes_below<0x143, 0xc>(v);  // the half before, to the third and fourth
  return v;
}
template <typename T>
__device__ __forceinline__ T lane_value(T v, int lane) {  // lane: uniform
  if constexpr (sizeof(T) == 8) {
    const u64 u = __builtin_bit_cast(u64, v);
    const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)u, lane), hi = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)(u >> 32), lane);
    return __builtin_bit_cast(T, (u64)hi << 32 | lo);
  } else {
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
  }
}

__device__ __forceinline__ float wave_top(float v) {  // of values that are not NaN
  auto step = [&](auto ctrl) { v = fmaxf(v, __uint_as_float((unsigned)__builtin_amdgcn_update_dpp((int)0xff800000, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, false))); };
  step(std::integral_constant<int, 0x111>{});
  step(std::integral_constant<int, 0x112>{});
  step(std::integral_constant<int, 0x114>{});
  step(std::integral_constant<int, 0x118>{});
  step(std::integral_constant<int, 0x142>{});
  step(std::integral_constant<int, 0x143>{});
  return lane_value(v, 63);
}

}  // namespace harli

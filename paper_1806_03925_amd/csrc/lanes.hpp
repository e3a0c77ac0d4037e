// Sums over a wavefront by moves between lanes (gfx950 only).
#pragma once

#include "gear_internal.hpp"

namespace gear {
namespace {

// sums of this and the lower lanes' v, by moves between lanes that need no LDS: within 16 lanes, then over the four
template <int CTRL, int ROWS> __device__ __forceinline__ int add_moved(int v) { return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int wave_scan(int v) {
  v = add_moved<0x111, 0xf>(v);   // one lane up, two, four, eight
  v = add_moved<0x112, 0xf>(v);
  v = add_moved<0x114, 0xf>(v);
  v = add_moved<0x118, 0xf>(v);
  v = add_moved<0x142, 0xa>(v);   // lane 15 to the second sixteen and 47 to the fourth
  return add_moved<0x143, 0xc>(v);   // lane 31 to the upper half
}
__device__ __forceinline__ int wave_add(int v) { return __builtin_amdgcn_readlane(wave_scan(v), kWave - 1); }

}  // namespace
}  // namespace gear

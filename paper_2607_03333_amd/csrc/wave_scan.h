// Prefix sums over a wave's lanes.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace spork {
namespace {

// Sum over lanes 0 .. lane of a wave, in register moves between lanes.
template <int kCtrl, int kRows>
__device__ __forceinline__ int add_from(int x) {
  return x + __builtin_amdgcn_update_dpp(0, x, kCtrl, kRows, 0xF, false);
}
__device__ __forceinline__ int wave_scan(int x) {
  x = add_from<0x111, 0xF>(x);  // row_shr 1, 2, 4, 8: sums in each 16 lanes
  x = add_from<0x112, 0xF>(x);
  x = add_from<0x114, 0xF>(x);
  x = add_from<0x118, 0xF>(x);
  x = add_from<0x142, 0xA>(x);  // the sum of lanes 0-15 to 16-31, of 32-47 to 48-63
  return add_from<0x143, 0xC>(x);  // and of 0-31 to 32-63
}
// (64 bits as three limbs, so that no carry is lost: 64 limbs of 22 bits fit.)
__device__ __forceinline__ int64_t wave_scan(int64_t x) {
  const int lo = wave_scan(static_cast<int>(x & 0x3FFFFF)), mid = wave_scan(static_cast<int>((x >> 22) & 0x3FFFFF)),
            hi = wave_scan(static_cast<int>(x >> 44));
  return lo + (static_cast<int64_t>(mid) << 22) + (static_cast<int64_t>(hi) << 44);
}

}  // namespace
}  // namespace spork

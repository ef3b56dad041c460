// Sums, scans and maxima over the lanes of a wavefront.
#pragma once
#include <hip/hip_runtime.h>

namespace hb {

// Over the wavefront by data-parallel moves (a permute through LDS per step costs ten times as much):
// inclusive sum over the lanes up to each, and the maximum of values >= 0.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp0(int x) {
  return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int scan_lanes(int x) {
  x += dpp0<0x111, 0xf>(x);  // the lane 1, 2, 4, 8 below in the row of sixteen
  x += dpp0<0x112, 0xf>(x);
  x += dpp0<0x114, 0xf>(x);
  x += dpp0<0x118, 0xf>(x);
  x += dpp0<0x142, 0xa>(x);  // the last lane of the row below, then of the first two rows
  x += dpp0<0x143, 0xc>(x);
  return x;
}
__device__ __forceinline__ int sum_lanes(int x) { return __builtin_amdgcn_readlane(scan_lanes(x), 63); }
__device__ __forceinline__ int max_lanes(int x) {
  x = max(x, dpp0<0x111, 0xf>(x));
  x = max(x, dpp0<0x112, 0xf>(x));
  x = max(x, dpp0<0x114, 0xf>(x));
  x = max(x, dpp0<0x118, 0xf>(x));
  x = max(x, dpp0<0x142, 0xa>(x));
  x = max(x, dpp0<0x143, 0xc>(x));
  return __builtin_amdgcn_readlane(x, 63);
}

}  // namespace hb

// Scans over a wave's 64 lanes in vector instructions (internal header): row
// shifts, then the row totals carried into the rows after them.
#pragma once

#include <hip/hip_runtime.h>

namespace ekv {
namespace {

// Inclusive scan with op, whose neutral element is 0 (sums; the maximum of values >= 0).
template <typename F>
__device__ __forceinline__ int wave_scan(int x, F op) {
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true));    // row_shr:1
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true));    // row_shr:2
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true));    // row_shr:4
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true));    // row_shr:8
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));   // row_bcast:15 into rows 1 and 3
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));   // row_bcast:31 into rows 2 and 3
  return x;
}
__device__ __forceinline__ int sum_scan(int x) {
  return wave_scan(x, [](int a, int b) { return a + b; });
}
__device__ __forceinline__ int max_scan(int x) {
  return wave_scan(x, [](int a, int b) { return a > b ? a : b; });
}
__device__ __forceinline__ int last_lane(int x) { return __builtin_amdgcn_readlane(x, 63); }


}  // namespace
}  // namespace ekv

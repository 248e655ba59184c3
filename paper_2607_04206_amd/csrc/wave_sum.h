// Sums over the lanes of a wave, by DPP moves: within rows of 16 lanes, then from
// row to row.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sangam {

// x of the lane that a DPP control names, 0 where there is none.
template <int CONTROL, int ROWS>
__device__ __forceinline__ uint64_t from_lane(uint64_t x) {
    const int low = __builtin_amdgcn_update_dpp(0, int(x), CONTROL, ROWS, 0xF, false);
    const int high = __builtin_amdgcn_update_dpp(0, int(x >> 32), CONTROL, ROWS, 0xF, false);
    return uint64_t(uint32_t(high)) << 32 | uint32_t(low);
}
template <int CONTROL, int ROWS>
__device__ __forceinline__ int from_lane(int x) { return __builtin_amdgcn_update_dpp(0, x, CONTROL, ROWS, 0xF, false); }
// Sum over the lanes up to this one: within rows of 16, then from row to row.
__device__ __forceinline__ uint64_t wave_up_to(uint64_t x) {
    x += from_lane<0x111, 0xF>(x);  // row_shr 1, 2, 4, 8
    x += from_lane<0x112, 0xF>(x);
    x += from_lane<0x114, 0xF>(x);
    x += from_lane<0x118, 0xF>(x);
    x += from_lane<0x142, 0xA>(x);  // row_bcast 15 into rows 1 and 3
    x += from_lane<0x143, 0xC>(x);  // row_bcast 31 into rows 2 and 3
    return x;
}

template <int CONTROL, int ROWS>
__device__ __forceinline__ double from_lane(double x) {
    return __builtin_bit_cast(double, from_lane<CONTROL, ROWS>(__builtin_bit_cast(uint64_t, x)));
}
__device__ __forceinline__ double wave_up_to(double x) {
    x += from_lane<0x111, 0xF>(x);
    x += from_lane<0x112, 0xF>(x);
    x += from_lane<0x114, 0xF>(x);
    x += from_lane<0x118, 0xF>(x);
    x += from_lane<0x142, 0xA>(x);
    x += from_lane<0x143, 0xC>(x);
    return x;
}
__device__ __forceinline__ int wave_up_to(int x) {
    x += from_lane<0x111, 0xF>(x);
    x += from_lane<0x112, 0xF>(x);
    x += from_lane<0x114, 0xF>(x);
    x += from_lane<0x118, 0xF>(x);
    x += from_lane<0x142, 0xA>(x);
    x += from_lane<0x143, 0xC>(x);
    return x;
}

}  // namespace sangam

// Sums of 64-bit floats over a wavefront (whole numbers below 2^53 are exact).
#pragma once

#include "device_util.h"

namespace surel {

// Sums over the lanes up to this one, by moves inside the vector unit (through LDS each of the six steps takes ten times as
// long, where a launch waits for one workgroup's sums).
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ double moved_from(double x) {   // zero for lanes without a source
    const uint64_t u = (uint64_t)__double_as_longlong(x);
    return __longlong_as_double((long long)((uint64_t)dpp_move<CTRL, ROWS>(0u, (uint32_t)(u >> 32)) << 32 | dpp_move<CTRL, ROWS>(0u, (uint32_t)u)));
}
__device__ __forceinline__ double sum_till(double x) {
    x += moved_from<0x111>(x);        // row_shr:1, 2, 4, 8
    x += moved_from<0x112>(x);
    x += moved_from<0x114>(x);
    x += moved_from<0x118>(x);
    x += moved_from<0x142, 0xA>(x);   // row_bcast:15 to rows 1 and 3
    x += moved_from<0x143, 0xC>(x);   // row_bcast:31 to rows 2 and 3
    return x;
}
// Of the lanes of the same 16 up to this one.
__device__ __forceinline__ double sum_till_in_16(double x) {
    x += moved_from<0x111>(x);
    x += moved_from<0x112>(x);
    x += moved_from<0x114>(x);
    x += moved_from<0x118>(x);
    return x;
}
__device__ __forceinline__ uint32_t sum_till_in_16(uint32_t x) {
    x += dpp_move<0x111>(0u, x);
    x += dpp_move<0x112>(0u, x);
    x += dpp_move<0x114>(0u, x);
    x += dpp_move<0x118>(0u, x);
    return x;
}
// What a lane (the same in all) has.
__device__ __forceinline__ double of_lane(double x, int lane) {
    const uint64_t u = (uint64_t)__double_as_longlong(x);
    return __longlong_as_double((long long)((uint64_t)wave_bcast_u32((uint32_t)(u >> 32), lane) << 32 | wave_bcast_u32((uint32_t)u, lane)));
}

// What comes before the thread's `mine` in a workgroup of up to 16 waves, and the workgroup's sum; of_wave: 16 words of LDS.
__device__ __forceinline__ double before_in_group(double mine, double* of_wave, double* all) {
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
    const double x = sum_till(mine), till = moved_from<0x138>(x);   // wave_shr:1
    __syncthreads();   // (of_wave may still be read from an earlier sum)
    if (lane == 63) of_wave[wave] = x;
    __syncthreads();
    const double waves = sum_till_in_16((lane & 15) < (int)(blockDim.x >> 6) ? of_wave[lane & 15] : 0.0);
    *all = of_lane(waves, 15);
    return (wave == 0 ? 0.0 : of_lane(waves, wave - 1)) + till;
}
__device__ __forceinline__ uint32_t before_in_group(uint32_t mine, uint32_t* of_wave, uint32_t* all) {
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
    const uint32_t x = wave_incl_sum(mine);
    __syncthreads();
    if (lane == 63) of_wave[wave] = x;
    __syncthreads();
    const uint32_t waves = sum_till_in_16((lane & 15) < (int)(blockDim.x >> 6) ? of_wave[lane & 15] : 0u);
    *all = wave_bcast_u32(waves, 15);
    return (wave == 0 ? 0u : wave_bcast_u32(waves, wave - 1)) + x - mine;
}

}  // namespace surel

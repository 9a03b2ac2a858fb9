// Sums over the lanes of a wave and the threads of a workgroup, by DPP.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace atf {
namespace scan {

// x plus another lane's (kCtrl), in the rows of 16 lanes that kRows names
template <int kCtrl, int kRows, typename Int>
__device__ __forceinline__ Int add_dpp(Int x) {
    if constexpr (sizeof(Int) == 4) {
        return x + __builtin_amdgcn_update_dpp(0, x, kCtrl, kRows, 0xF, false);
    } else {
        const int lo = __builtin_amdgcn_update_dpp(0, int(x), kCtrl, kRows, 0xF, false);
        const int hi = __builtin_amdgcn_update_dpp(0, int(x >> 32), kCtrl, kRows, 0xF, false);
        return x + (Int(hi) << 32 | uint32_t(lo));
    }
}
// Each lane's sum of the lanes up to it: of its row of 16, of the wave.
template <typename Int>
__device__ __forceinline__ Int row16(Int x) {
    x = add_dpp<0x111, 0xF>(x);  // from the lane 1, 2, 4, 8 below in the row of 16
    x = add_dpp<0x112, 0xF>(x);
    x = add_dpp<0x114, 0xF>(x);
    return add_dpp<0x118, 0xF>(x);
}
template <typename Int>
__device__ __forceinline__ Int wave(Int x) {
    x = row16(x);
    x = add_dpp<0x142, 0xA>(x);  // from the last lane of rows 0 and 2 to the rows after them
    return add_dpp<0x143, 0xC>(x);  // from that of row 1 to rows 2 and 3
}
template <typename Int>
__device__ __forceinline__ Int lane_of(Int x, int lane) {
    if constexpr (sizeof(Int) == 4)
        return __builtin_amdgcn_readlane(x, lane);
    else
        return Int(__builtin_amdgcn_readlane(int(x >> 32), lane)) << 32 | uint32_t(__builtin_amdgcn_readlane(int(x), lane));
}

// x: each thread's sums of the threads up to it, of a workgroup of kWaves waves (at most 16); all: the
// sums of all.  `part` is free again after the next barrier.
template <int kWaves, int N, typename Int>
__device__ __forceinline__ void block(Int (&x)[N], Int (&all)[N], Int (*part)[kWaves]) {
    static_assert(kWaves <= 16, "a row of 16 lanes adds up the waves' sums");
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = wave(x[i]);
        if (lane == 63) part[i][w] = x[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const Int sums = row16(part[i][min(lane & 15, kWaves - 1)]);
        all[i] = lane_of(sums, kWaves - 1);
        if (w > 0) x[i] += lane_of(sums, w - 1);
    }
}

}  // namespace scan
}  // namespace atf

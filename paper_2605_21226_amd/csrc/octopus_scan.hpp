// Running sums over a wavefront's lanes and a workgroup's threads.
#ifndef OCTOPUS_SCAN_HPP_
#define OCTOPUS_SCAN_HPP_

#include <hip/hip_runtime.h>

namespace octopus {

constexpr int kScanLanes = 64;

// x of the lane that CTRL names, 0 where there is none (rows outside ROWS, lanes before a row's first).
template <int CTRL, int ROWS>
__device__ __forceinline__ int lane_before(int x) {
    return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double lane_before(double x) {
    const long long b = __double_as_longlong(x);
    const unsigned lo = static_cast<unsigned>(lane_before<CTRL, ROWS>(static_cast<int>(b)));
    const unsigned hi = static_cast<unsigned>(lane_before<CTRL, ROWS>(static_cast<int>(b >> 32)));
    return __longlong_as_double(static_cast<long long>(static_cast<unsigned long long>(hi) << 32 | lo));
}

// Inclusive sums: within rows of 16 lanes, then a row's last sum into the next row, then the lower half's into the upper.
template <class T>
__device__ __forceinline__ T wave_scan(T x) {
    x += lane_before<0x111, 0xf>(x);   // row_shr:1
    x += lane_before<0x112, 0xf>(x);
    x += lane_before<0x114, 0xf>(x);
    x += lane_before<0x118, 0xf>(x);
    x += lane_before<0x142, 0xa>(x);   // row_bcast:15 into rows 1 and 3
    x += lane_before<0x143, 0xc>(x);   // row_bcast:31 into rows 2 and 3
    return x;
}

// x of one lane (the same for all), for all.
__device__ __forceinline__ double wave_lane(double x, int lane) {
    const long long b = __double_as_longlong(x);
    const unsigned lo = static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(b), lane));
    const unsigned hi = static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(b >> 32), lane));
    return __longlong_as_double(static_cast<long long>(static_cast<unsigned long long>(hi) << 32 | lo));
}
__device__ __forceinline__ double wave_last(double x) { return wave_lane(x, kScanLanes - 1); }

// Inclusive sums over a workgroup's threads, and everybody's.  All threads call it; `room` is free again after the next barrier.
template <int THREADS, class T>
__device__ __forceinline__ T block_scan(T x, T *room, T *total) {
    constexpr int WAVES = THREADS / kScanLanes;
    const int lane = threadIdx.x % kScanLanes, wave = threadIdx.x / kScanLanes;
    const T upto = wave_scan(x);
    __syncthreads();
    if (lane == kScanLanes - 1) room[wave] = upto;
    __syncthreads();
    T before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const T n = room[w];
        before += w < wave ? n : T(0);
        all += n;
    }
    *total = all;
    return before + upto;
}

}  // namespace octopus

#endif

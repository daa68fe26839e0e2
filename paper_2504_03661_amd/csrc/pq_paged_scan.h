// Running sums over a workgroup of 1024 threads, and the bisection that finds an entry's owner in them: what the kernels that work
// requests and blocks out share (gfx950).
#pragma once

#include "pq_paged_tile.h"

namespace {

constexpr int SCAN_THREADS = 1024;
constexpr int SCAN_WAVES = SCAN_THREADS / 64;

struct scan_room {
    int wave[2][SCAN_WAVES];
};

// Inclusive sums over the workgroup's threads of two numbers, and their totals.
__device__ inline void scan_two(int &x, int &y, scan_room &room, int &all_x, int &all_y)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    x = lane_scan(x);
    y = lane_scan(y);
    if (lane == 63) {
        room.wave[0][wave] = x;
        room.wave[1][wave] = y;
    }
    __syncthreads();
    int before_x = 0, before_y = 0;
    all_x = all_y = 0;
#pragma unroll
    for (int w = 0; w < SCAN_WAVES; ++w) {
        const int of_x = room.wave[0][w], of_y = room.wave[1][w];
        before_x += w < wave ? of_x : 0;
        before_y += w < wave ? of_y : 0;
        all_x += of_x;
        all_y += of_y;
    }
    __syncthreads();
    x += before_x;
    y += before_y;
}

__device__ inline int between(int n, int most) { return n < 0 ? 0 : n > most ? most : n; }
__device__ inline int at_most(int x, int most) { return x > most ? most : x; }

// the last i of [0, n) with sums[i] <= x, for x >= sums[0] = 0
__device__ inline int owner(const int *sums, int n, int x)
{
    int low = 0, high = n;
    while (high - low > 1) {
        const int mid = (low + high) >> 1;
        if (sums[mid] <= x)
            low = mid;
        else
            high = mid;
    }
    return low;
}

}  // namespace

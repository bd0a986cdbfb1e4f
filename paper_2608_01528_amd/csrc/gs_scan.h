// Prefix sums over a work-group of 1024 threads.
#pragma once

#include "gs_internal.h"

namespace gs {

__device__ __forceinline__ int64_t wave_scan(int64_t v, int lanes) {
    const int l = threadIdx.x & 63;
    for (int d = 1; d < lanes; d <<= 1) {
        const int64_t x = __shfl_up((long long)v, d);
        if (l >= d) v += x;
    }
    return v;
}

// Exclusive sums of v, and their total; room: 16 values that no thread may still
// be reading (one barrier lies between its writes and its reads).
__device__ __forceinline__ int64_t group_scan(int64_t v, int64_t *room, int64_t *total) {
    const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t s = wave_scan(v, 64);
    if (l == 63) room[w] = s;
    __syncthreads();
    const int64_t waves = wave_scan(l < 16 ? room[l] : 0, 16);
    *total = __shfl((long long)waves, 15);
    const int64_t before = __shfl((long long)waves, w ? w - 1 : 0);
    return (w ? before : 0) + s - v;
}

}  // namespace gs

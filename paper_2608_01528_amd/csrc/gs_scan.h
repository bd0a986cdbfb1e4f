// Prefix sums over a wave and over a work-group of 1024 threads.
#pragma once

#include <string.h>

#include "gs_internal.h"

namespace gs {

// Moves between lanes within the vector unit; lanes without a source get 0.
template <int CTRL, int ROWS, typename V> __device__ __forceinline__ V lane_moved(V v) {
    static_assert(sizeof(V) == 4 || sizeof(V) == 8, "one register or two");
    int x[sizeof(V) / 4];
    memcpy(x, &v, sizeof v);
#pragma unroll
    for (unsigned i = 0; i < sizeof(V) / 4; ++i) x[i] = __builtin_amdgcn_update_dpp(0, x[i], CTRL, ROWS, 0xf, false);
    memcpy(&v, x, sizeof v);
    return v;
}
// The value of a lane that all lanes name alike.
template <typename V> __device__ __forceinline__ V lane_value(V v, int lane) {
    int x[sizeof(V) / 4];
    memcpy(x, &v, sizeof v);
#pragma unroll
    for (unsigned i = 0; i < sizeof(V) / 4; ++i) x[i] = __builtin_amdgcn_readlane(x[i], lane);
    memcpy(&v, x, sizeof v);
    return v;
}

// Sums over this and the lanes before it: within rows of 16 lanes by 1, 2, 4, 8,
// then from the rows before.
template <typename V> __device__ __forceinline__ V row_upto(V v) {
    v += lane_moved<0x111, 0xf>(v);
    v += lane_moved<0x112, 0xf>(v);
    v += lane_moved<0x114, 0xf>(v);
    return v + lane_moved<0x118, 0xf>(v);
}
template <typename V> __device__ __forceinline__ V wave_upto(V v) {
    v = row_upto(v);
    v += lane_moved<0x142, 0xa>(v);         // lane 15 of the row before, into rows 1 and 3
    return v + lane_moved<0x143, 0xc>(v);   // lane 31, into rows 2 and 3
}

// Exclusive sums of v over 1024 threads, and their total; room: 16 values that no
// thread may still be reading (one barrier lies between its writes and its reads).
template <typename V> __device__ __forceinline__ V group_scan(V v, V *room, V *total) {
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const V s = wave_upto(v);
    if (l == 63) room[w] = s;
    __syncthreads();
    const V waves = row_upto(l < 16 ? room[l] : V(0));
    *total = lane_value(waves, 15);
    return (w ? lane_value(waves, w - 1) : V(0)) + s - v;
}

}  // namespace gs

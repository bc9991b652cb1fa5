// Sums over the 64 lanes of a wavefront by DPP (a lane exchange through LDS takes some 100 cycles,
// a DPP step 8): inclusive scans in the order of the lanes, and totals.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <string.h>

namespace olive {

// The lane that CTRL names; 0 where it names none, and in the rows of 16 lanes that ROWS leaves out.
template <int CTRL, int ROWS = 0xf, typename V>
__device__ __forceinline__ V wave_take(V v) {
    static_assert(sizeof(V) == 4 || sizeof(V) == 8, "");
    int w[sizeof(V) / 4];
    memcpy(w, &v, sizeof(V));
#pragma unroll
    for (int i = 0; i < (int)sizeof(V) / 4; ++i) w[i] = __builtin_amdgcn_update_dpp(0, w[i], CTRL, ROWS, 0xf, false);
    memcpy(&v, w, sizeof(V));
    return v;
}
// The value of a lane that is the same for all.
template <typename V>
__device__ __forceinline__ V wave_read(V v, int lane) {
    int w[sizeof(V) / 4];
    memcpy(w, &v, sizeof(V));
#pragma unroll
    for (int i = 0; i < (int)sizeof(V) / 4; ++i) w[i] = __builtin_amdgcn_readlane(w[i], lane);
    memcpy(&v, w, sizeof(V));
    return v;
}
// v of this lane and those before it.
template <typename V>
__device__ __forceinline__ V wave_scan(V v) {
    v += wave_take<0x111>(v);           // the lane 1, 2, 4, 8 before, within 16
    v += wave_take<0x112>(v);
    v += wave_take<0x114>(v);
    v += wave_take<0x118>(v);
    v += wave_take<0x142, 0xa>(v);      // lane 15 of the 16 before, for the 2nd and the 4th 16
    v += wave_take<0x143, 0xc>(v);      // lane 31, for the second half
    return v;
}
// v of the lane before (0 for the first).
template <typename V>
__device__ __forceinline__ V wave_before(V v) { return wave_take<0x138>(v); }
template <typename V>
__device__ __forceinline__ V wave_sum(V v) { return wave_read(wave_scan(v), 63); }
// The largest value (of values of at least 0).
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    v = max(v, wave_take<0x111>(v));
    v = max(v, wave_take<0x112>(v));
    v = max(v, wave_take<0x114>(v));
    v = max(v, wave_take<0x118>(v));
    v = max(v, wave_take<0x142, 0xa>(v));
    v = max(v, wave_take<0x143, 0xc>(v));
    return wave_read(v, 63);
}

}  // namespace olive

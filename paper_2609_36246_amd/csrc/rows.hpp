// Rows of bf16 or fp32 elements, VEC at a time, in fp32 registers.
#pragma once

#include "olive_device.hpp"

namespace olive {

template <typename T> struct RowElem;
template <> struct RowElem<float> {
    static __device__ __forceinline__ float get(float v) { return v; }
    static __device__ __forceinline__ float put(float v) { return v; }
};
template <> struct RowElem<uint16_t> {
    static __device__ __forceinline__ float get(uint16_t v) { return bf16_bits_to_f32(v); }
    static __device__ __forceinline__ uint16_t put(float v) { return (uint16_t)(pack_bf16x2(v, v) & 0xffffu); }
};

// 16 bytes of a row as they lie in memory, at any alignment of their type (one instruction all the
// same; rows that lie on 16 bytes are the fast case, by the memory system).
struct Lot { uint32_t w[4]; };
template <typename T> constexpr int kLot = 16 / (int)sizeof(T);      // its elements

template <typename T>
__device__ __forceinline__ Lot read_lot(const T *p) {
    struct __attribute__((packed, aligned(sizeof(T)))) Loose { uint32_t w[4]; };
    const Loose y = *(const Loose *)p;
    return Lot{{y.w[0], y.w[1], y.w[2], y.w[3]}};
}
template <typename T>
__device__ __forceinline__ void write_lot(T *p, const Lot &x) {
    struct __attribute__((packed, aligned(sizeof(T)))) Loose { uint32_t w[4]; };
    *(Loose *)p = Loose{{x.w[0], x.w[1], x.w[2], x.w[3]}};
}
// The same past the caches, for outputs that they would not hold until they are read.
template <typename T>
__device__ __forceinline__ void stream_lot(T *p, const Lot &x) {
    typedef uint32_t Words __attribute__((ext_vector_type(4)));
    typedef Words Loose __attribute__((aligned(2)));
    __builtin_nontemporal_store((Words){x.w[0], x.w[1], x.w[2], x.w[3]}, (Loose *)p);
}
template <typename T>
__device__ __forceinline__ void write_lot(T *p, const Lot &x, bool stream) {
    if (stream) stream_lot(p, x);
    else write_lot(p, x);
}
// The first element goes, the last is that of `in` (each half of it for 16 bits).
template <typename T>
__device__ __forceinline__ void drop_first(Lot &x, uint32_t in) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t above = j < 3 ? x.w[j + 1] : in;
        x.w[j] = sizeof(T) == 4 ? above : x.w[j] >> 16 | above << 16;
    }
}
// The elements of a row from i on, `fill` from `end` on.
template <typename T>
__device__ __forceinline__ Lot load_lot(const T *row, int i, int end, uint32_t fill) {
    Lot x{{fill, fill, fill, fill}};
    if (i >= end) return x;
    const int from = min(i, end - kLot<T>);      // (at the end the 16 bytes before it, shifted)
    if (from >= 0) {
        x = read_lot(row + from);
#pragma unroll 1
        for (int j = from; j < i; ++j) drop_first<T>(x, fill);
    } else {
#pragma unroll 1
        for (int j = i; j < i + kLot<T>; ++j) {
            uint32_t v = fill;
            if (j < end) {
                T e = row[j];
                memcpy(&v, &e, sizeof(T));
            }
            drop_first<T>(x, v);
        }
    }
    return x;
}
template <typename T>
__device__ __forceinline__ void store_lot(T *row, int i, int end, Lot x) {
    if (i + kLot<T> <= end) return write_lot(row + i, x);
#pragma unroll 1
    for (; i < end; ++i) {
        T e;
        memcpy(&e, &x, sizeof(T));
        row[i] = e;
        drop_first<T>(x, 0);
    }
}
template <typename T>
__device__ __forceinline__ void unpack_lot(const Lot &u, float (&x)[kLot<T>]) {
#pragma unroll
    for (int j = 0; j < kLot<T>; ++j) {
        if constexpr (sizeof(T) == 4) x[j] = __uint_as_float(u.w[j]);
        else x[j] = __uint_as_float(j & 1 ? u.w[j >> 1] & 0xffff0000u : u.w[j >> 1] << 16);
    }
}
template <typename T>
__device__ __forceinline__ Lot pack_lot(const float (&x)[kLot<T>]) {
    Lot u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 4) u.w[j] = __float_as_uint(x[j]);
        else u.w[j] = pack_bf16x2(x[2 * j], x[2 * j + 1]);
    }
    return u;
}

}  // namespace olive

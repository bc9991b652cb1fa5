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

template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) RowVec { T v[VEC]; };

template <typename T, int VEC>
__device__ __forceinline__ void get_vec(const T *p, float (&x)[VEC]) {
    const RowVec<T, VEC> u = *(const RowVec<T, VEC> *)p;
#pragma unroll
    for (int j = 0; j < VEC; ++j) x[j] = RowElem<T>::get(u.v[j]);
}
template <typename T, int VEC>
__device__ __forceinline__ void put_vec(T *p, const float (&x)[VEC]) {
    RowVec<T, VEC> u;
#pragma unroll
    for (int j = 0; j < VEC; ++j) u.v[j] = RowElem<T>::put(x[j]);
    *(RowVec<T, VEC> *)p = u;
}

}  // namespace olive

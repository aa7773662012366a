// Vectors of VEC tensor elements as float32: 16 bytes of either type, for the kernels that pass over rows.
#pragma once

#include "psa_device.h"
#include "psa_internal.h"

namespace psa {

template <typename T> constexpr int kVec = 16 / sizeof(T);      // elements of a 16-byte access

// element conversions: exact to float32, round-to-nearest-even back
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16_t x) { return __uint_as_float((uint32_t)x.x << 16); }
__device__ __forceinline__ void from_f32(float& o, float x) { o = x; }
__device__ __forceinline__ void from_f32(bf16_t& o, float x) { o.x = f32_to_bf16(x); }

// a 16-byte access at an element's alignment: the memory unit takes any
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Chunk { uint32_t w[4]; };

__device__ __forceinline__ void unpack(const uint32_t (&w)[4], float (&v)[4], float) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
}
__device__ __forceinline__ void unpack(const uint32_t (&w)[4], float (&v)[8], bf16_t) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = bf16_lo(w[i]); v[2 * i + 1] = bf16_hi(w[i]); }
}
__device__ __forceinline__ void pack(uint32_t (&w)[4], const float (&v)[4], float) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(v[i]);
}
__device__ __forceinline__ void pack(uint32_t (&w)[4], const float (&v)[8], bf16_t) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = cvt_pk_bf16(v[2 * i], v[2 * i + 1]);
}

// n (1 .. kVec) elements from p; the others are zero.
template <typename T>
__device__ __forceinline__ void load_vec(float (&v)[kVec<T>], const T* p, int n) {
    if (n >= kVec<T>) {
        const Chunk<T> c = *reinterpret_cast<const Chunk<T>*>(p);
        unpack(c.w, v, T{});
    } else {
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) v[i] = i < n ? to_f32(p[i]) : 0.f;
    }
}
// the same without the conversion: to be asked for ahead of its use
template <typename T>
__device__ __forceinline__ Chunk<T> load_chunk(const T* p, int n) {
    Chunk<T> c;
    if (n >= kVec<T>) {
        c = *reinterpret_cast<const Chunk<T>*>(p);
    } else {
        float v[kVec<T>];
        load_vec(v, p, n);
        pack(c.w, v, T{});
    }
    return c;
}
template <typename T>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[kVec<T>], int n) {
    if (n >= kVec<T>) {
        Chunk<T> c;
        pack(c.w, v, T{});
        *reinterpret_cast<Chunk<T>*>(p) = c;
    } else {
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) if (i < n) from_f32(p[i], v[i]);
    }
}

}  // namespace psa

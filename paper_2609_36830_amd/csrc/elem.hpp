// The element types of the operators that read logits, tokens and updates:
// 16-byte vectors of them as binary32 values and back.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_util.hpp"

namespace pace {

enum ElemType : int { kF32 = 0, kBf16 = 1, kF16 = 2 };
constexpr int kElemTypes = 3;
inline int elem_bytes_of(int dtype) { return dtype == kF32 ? 4 : 2; }

// Runs f with the C++ type of a checked dtype.
struct bf16_t { uint16_t x; };
typedef _Float16 f16_t;
template <typename F>
auto with_elem(int dtype, F f) {
    switch (dtype) {
        case kF32: return f(float{});
        case kBf16: return f(bf16_t{});
        default: return f(f16_t{});
    }
}

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(bf16_t v) { return __builtin_bit_cast(float, (uint32_t)v.x << 16); }
__device__ __forceinline__ float to_f32(f16_t v) { return (float)v; }

// Rounded to nearest, ties to even.
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ f16_t from_f32<f16_t>(float v) { return (f16_t)v; }
template <> __device__ __forceinline__ bf16_t from_f32<bf16_t>(float v) {
    return bf16_t{__builtin_bit_cast(uint16_t, (__bf16)v)};
}

// The elements of 16 bytes.
template <typename T> constexpr int kVecOf = 16 / (int)sizeof(T);

template <typename T> __device__ __forceinline__ void unpack16(const uint4 &r, float (&v)[kVecOf<T>]);
template <> __device__ __forceinline__ void unpack16<float>(const uint4 &r, float (&v)[4]) {
    v[0] = __builtin_bit_cast(float, r.x), v[1] = __builtin_bit_cast(float, r.y);
    v[2] = __builtin_bit_cast(float, r.z), v[3] = __builtin_bit_cast(float, r.w);
}
template <> __device__ __forceinline__ void unpack16<bf16_t>(const uint4 &r, float (&v)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        v[2 * k] = __builtin_bit_cast(float, w[k] << 16);
        v[2 * k + 1] = __builtin_bit_cast(float, w[k] & 0xffff0000u);
    }
}
template <> __device__ __forceinline__ void unpack16<f16_t>(const uint4 &r, float (&v)[8]) {
    typedef f16_t h2 __attribute__((ext_vector_type(2)));
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const h2 h = __builtin_bit_cast(h2, w[k]);
        v[2 * k] = (float)h.x;
        v[2 * k + 1] = (float)h.y;
    }
}

template <typename T> __device__ __forceinline__ uint4 pack16(const float (&v)[kVecOf<T>]) {
    struct alignas(16) { T e[kVecOf<T>]; } p;
#pragma unroll
    for (int k = 0; k < kVecOf<T>; ++k) p.e[k] = from_f32<T>(v[k]);
    return __builtin_bit_cast(uint4, p);
}

}  // namespace pace

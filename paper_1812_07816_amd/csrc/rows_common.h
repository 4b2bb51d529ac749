// Eight values, or one, of a bf16 (uint16_t) or fp32 tensor at a time: what the operators over rows share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "split_f32.h"

namespace mi3d {

template <typename T, int V>
__device__ __forceinline__ void load_values(const T* p, float (&f)[V]) {
    if constexpr (V == 1) {
        if constexpr (sizeof(T) == 2) f[0] = __builtin_bit_cast(float, (uint32_t)*p << 16);
        else f[0] = *p;
    } else if constexpr (sizeof(T) == 2) {
        const uint4 v = *(const uint4*)p;
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __builtin_bit_cast(float, w[i] << 16);
            f[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xFFFF0000u);
        }
    } else {
        const float4 a = ((const float4*)p)[0], b = ((const float4*)p)[1];
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
}
// rounds to nearest even
template <typename T, int V>
__device__ __forceinline__ void store_values(T* p, const float (&f)[V]) {
    if constexpr (V == 1) {
        if constexpr (sizeof(T) == 2) *p = (uint16_t)pack_bf16(f[0], 0.f);
        else *p = f[0];
    } else if constexpr (sizeof(T) == 2) {
        *(uint4*)p = uint4{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])};
    } else {
        ((float4*)p)[0] = float4{f[0], f[1], f[2], f[3]};
        ((float4*)p)[1] = float4{f[4], f[5], f[6], f[7]};
    }
}
// eight values at any address of their type (the memory system takes unaligned pieces)
template <typename T>
__device__ __forceinline__ void load8_anywhere(const T* p, float (&f)[8]) {
    typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)), aligned(2))) uint32_t u32x4;
    uint4 v[sizeof(T) / 2];
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) {
        const u32x4 u = ((const u32x4*)p)[i];
        v[i] = uint4{u[0], u[1], u[2], u[3]};
    }
    load_values<T, 8>((const T*)v, f);
}
template <typename T>
__device__ __forceinline__ void store8_anywhere(T* p, const float (&f)[8]) {
    typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)), aligned(2))) uint32_t u32x4;
    uint4 v[sizeof(T) / 2];
    store_values<T, 8>((T*)v, f);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) ((u32x4*)p)[i] = u32x4{v[i].x, v[i].y, v[i].z, v[i].w};
}
// the same for 8 values that stay out of the way of what is read again soon
template <typename T>
__device__ __forceinline__ void store_streamed(T* p, const float (&f)[8]) {
    typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;
    typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;
    if constexpr (sizeof(T) == 2) {
        __builtin_nontemporal_store(u32x4{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])}, (u32x4*)p);
    } else {
        __builtin_nontemporal_store(f32x4{f[0], f[1], f[2], f[3]}, (f32x4*)p);
        __builtin_nontemporal_store(f32x4{f[4], f[5], f[6], f[7]}, (f32x4*)p + 1);
    }
}
inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace mi3d

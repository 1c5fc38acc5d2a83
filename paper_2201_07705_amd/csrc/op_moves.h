// Moves of several consecutive elements that need no more alignment than the
// elements have: rows of any stride and matrices of any width then take the
// same wide loads and stores. (Global memory takes them at any address on
// this target; at aligned ones they cost what aligned moves do. Direct loads
// to LDS and LDS itself are not meant.)
#pragma once
#include <hip/hip_runtime.h>

namespace gemel {

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned short u16x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

template <typename F4>
__device__ __forceinline__ F4 get_f32x4(const void *p) {
    return __builtin_bit_cast(F4, *(const f32x4_any *)p);
}
__device__ __forceinline__ uint4 get_16b(const void *p) { return __builtin_bit_cast(uint4, *(const u32x4_any *)p); }
__device__ __forceinline__ ushort4 get_u16x4(const void *p) { return __builtin_bit_cast(ushort4, *(const u16x4_any *)p); }
template <typename F4>
__device__ __forceinline__ void put_f32x4(void *p, F4 v) {
    *(f32x4_any *)p = __builtin_bit_cast(f32x4_any, v);
}
__device__ __forceinline__ void put_u16x4(void *p, ushort4 v) { *(u16x4_any *)p = __builtin_bit_cast(u16x4_any, v); }

}  // namespace gemel

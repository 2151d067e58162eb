// What the kernels of the quantised inference share: the floating types at the boundary, and moves between lanes.
#pragma once
#include "common.h"

namespace zkmi {

typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

static const float kInf = __builtin_inff();

inline size_t dtype_bytes(int dtype) { return dtype == ZK_F32 ? 4 : (dtype == ZK_F16 || dtype == ZK_BF16 || dtype == ZK_I16) ? 2 : 0; }
inline bool aligned(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

__device__ __forceinline__ float bits_float(uint32_t b) { return __builtin_bit_cast(float, b); }
__device__ __forceinline__ uint32_t float_bits(float f) { return __builtin_bit_cast(uint32_t, f); }

// Element e of a 32-bit word of 16-bit ones, as a float.
template <int DT>
__device__ __forceinline__ float half_of(uint32_t word, int e) {
    const uint32_t h = e ? word >> 16 : word & 0xffffu;
    if constexpr (DT == ZK_BF16) return bits_float(h << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)h);
}

template <int DT>
__device__ __forceinline__ float load_one(const void* p, size_t i) {
    if constexpr (DT == ZK_F32) return ((const float*)p)[i];
    return half_of<DT>(((const uint16_t*)p)[i], 0);
}

// Rounded to nearest, ties to even, as the conversions of the host's types do.
template <int DT>
__device__ __forceinline__ void store_one(void* p, size_t i, float f) {
    if constexpr (DT == ZK_F32) ((float*)p)[i] = f;
    if constexpr (DT == ZK_F16) ((_Float16*)p)[i] = (_Float16)f;
    if constexpr (DT == ZK_BF16) ((__bf16*)p)[i] = (__bf16)f;
}

template <int DT>
__device__ __forceinline__ uint16_t half_bits(float f) {
    if constexpr (DT == ZK_F16) return __builtin_bit_cast(uint16_t, (_Float16)f);
    return __builtin_bit_cast(uint16_t, (__bf16)f);
}

}  // namespace zkmi

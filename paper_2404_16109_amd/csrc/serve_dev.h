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

#define kInf __builtin_inff()

inline size_t dtype_bytes(int dtype) { return dtype == ZK_F32 ? 4 : (dtype == ZK_F16 || dtype == ZK_BF16 || dtype == ZK_I16) ? 2 : 0; }
inline bool aligned(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// A value that is the same in all lanes, for the compiler to know.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }

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

// f as it is, rounded to 32 bits: a product is not joined with the rounding to 16 that follows (v_fma_mix has one rounding for both).
__device__ __forceinline__ float as_it_is(float f) {
    asm("" : "+v"(f));
    return f;
}

// Over the 64 lanes of a wavefront, in every lane: moves within rows of 16 lanes, then two broadcasts from row to row, all at
// the rate of the vector ALU (lanes_sum in reduce_dev.h has the same steps).  Lanes without a partner keep their own.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t from_lane(uint32_t old, uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)x, CTRL, ROWS, 0xf, false);
}
template <typename Op>
__device__ __forceinline__ uint32_t over_wave(uint32_t x, uint32_t none, Op op) {
    x = op(x, from_lane<0x111, 0xf>(none, x));  // row_shr 1, 2, 4, 8: a row's last lane has the row
    x = op(x, from_lane<0x112, 0xf>(none, x));
    x = op(x, from_lane<0x114, 0xf>(none, x));
    x = op(x, from_lane<0x118, 0xf>(none, x));
    x = op(x, from_lane<0x142, 0xa>(none, x));  // row_bcast 15 into rows 1 and 3
    x = op(x, from_lane<0x143, 0xc>(none, x));  // row_bcast 31 into rows 2 and 3
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
__device__ __forceinline__ float wave_add(float x) {
    return bits_float(over_wave(float_bits(x), 0u, [](uint32_t a, uint32_t b) { return float_bits(bits_float(a) + bits_float(b)); }));
}
__device__ __forceinline__ float wave_max(float x) {
    return bits_float(over_wave(float_bits(x), float_bits(-kInf), [](uint32_t a, uint32_t b) { return float_bits(fmaxf(bits_float(a), bits_float(b))); }));
}
__device__ __forceinline__ uint32_t wave_add(uint32_t x) {
    return over_wave(x, 0u, [](uint32_t a, uint32_t b) { return a + b; });
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
    return over_wave(x, 0u, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

}  // namespace zkmi

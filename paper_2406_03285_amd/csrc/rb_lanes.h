// What the kernels of the training step share: bfloat16 numbers, and values exchanged between the lanes of a wavefront.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace {

typedef uint32_t sc_vec __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float sc_neg_inf() { return -__builtin_huge_valf(); }
__device__ __forceinline__ float sc_nan() { return __builtin_nanf(""); }

struct Bf16 { uint16_t bits; };
typedef __bf16 sc_bf16x2 __attribute__((ext_vector_type(2)));
typedef float sc_floatx2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t sc_bf16_pair(float a, float b)      // to nearest, ties to even; NaN stays NaN (one instruction)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((sc_floatx2{a, b}), sc_bf16x2));
}
__device__ __forceinline__ uint32_t sc_bf16_bits(float x) { return sc_bf16_pair(x, x) & 0xffffu; }

// ---- between lanes -----------------------------------------------------------

// The value of lane ^ D, without a trip through LDS.
template <int D>
__device__ __forceinline__ uint32_t sc_xor(uint32_t v)
{
    static_assert(D == 1 || D == 2 || D == 4 || D == 8 || D == 16 || D == 32, "a power of two within a wavefront");
    const int x = (int)v;
    if constexpr (D == 1) return (uint32_t)__builtin_amdgcn_update_dpp(0, x, 0xB1, 0xf, 0xf, false);             // quad_perm 1 0 3 2
    if constexpr (D == 2) return (uint32_t)__builtin_amdgcn_update_dpp(0, x, 0x4E, 0xf, 0xf, false);             // quad_perm 2 3 0 1
    if constexpr (D == 4) return (uint32_t)__builtin_amdgcn_update_dpp(0, __builtin_amdgcn_update_dpp(0, x, 0x141, 0xf, 0xf, false), 0x1B, 0xf, 0xf, false);   // halves of a row mirrored, quads mirrored
    if constexpr (D == 8) return (uint32_t)__builtin_amdgcn_update_dpp(0, x, 0x128, 0xf, 0xf, false);            // rows of 16 turned by 8
    if constexpr (D == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);      // [0]: odd rows hold the even ones, [1]: even rows the odd ones
        return threadIdx.x & 16 ? r[0] : r[1];
    }
    if constexpr (D == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return threadIdx.x & 32 ? r[0] : r[1];
    }
}
template <int D> __device__ __forceinline__ float sc_xor(float v) { return __uint_as_float(sc_xor<D>(__float_as_uint(v))); }
template <int D> __device__ __forceinline__ uint64_t sc_xor(uint64_t v)
{
    return ((uint64_t)sc_xor<D>((uint32_t)(v >> 32)) << 32) | sc_xor<D>((uint32_t)v);
}

}  // namespace

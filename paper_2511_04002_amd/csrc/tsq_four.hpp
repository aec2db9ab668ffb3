// The elements of a cache in 4 bits, for its kernels (tsq_four_rows.hip, tsq_attend_four.hip).
//
// A sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6: one bit of a fraction below two of an exponent.  32 elements of a token
// share a scale, a power of two whose exponent + 127 is a byte; 255 says that all of them are NaN.  An element is then
// exact in either 16-bit type, and the conversion instructions make two of them at once, scale included.
#pragma once

#include <hip/hip_runtime.h>

#include "tsq_cache_internal.hpp"

namespace tsq {
namespace {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

constexpr uint32_t kNotANumber = 255;

// The scales that a cache of this type can have: those whose 0.5 and 6 the type holds exactly, of bfloat16 without the
// smallest, which are of no use and close to what the matrix instructions would lose.
template <bool BF16> struct FourScales { static constexpr int lowest = BF16 ? 127 - 120 : 127 - 23, highest = BF16 ? 127 + 125 : 127 + 13; };

// Bits of a scale's byte as binary32 (infinity of 255, which the conversions take as NaN).
__device__ __forceinline__ float four_scale(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// ... of a word's byte, in one instruction (the compiler takes two).
template <int BYTE> __device__ __forceinline__ float four_scale_at(uint32_t w) {
    float f;
    const uint32_t by = 23;
    if constexpr (BYTE == 0) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_0" : "=v"(f) : "v"(by), "v"(w));
    else if constexpr (BYTE == 1) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_1" : "=v"(f) : "v"(by), "v"(w));
    else if constexpr (BYTE == 2) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_2" : "=v"(f) : "v"(by), "v"(w));
    else asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_3" : "=v"(f) : "v"(by), "v"(w));
    return f;
}

// Two elements of a word's byte, in 16 bits each.
template <bool BF16, int BYTE> __device__ __forceinline__ uint32_t four_pair(uint32_t w, float scale) {
    if constexpr (BF16) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, BYTE));
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, BYTE));
}
// A word's eight.
template <bool BF16> __device__ __forceinline__ uint4_t four_eight(uint32_t w, float scale) {
    return uint4_t{four_pair<BF16, 0>(w, scale), four_pair<BF16, 1>(w, scale), four_pair<BF16, 2>(w, scale), four_pair<BF16, 3>(w, scale)};
}

// Two binary32 numbers rounded to a 16-bit type each, in one instruction.
template <bool BF16> __device__ __forceinline__ uint32_t pack_two(float a, float b) {
    if constexpr (BF16) return __builtin_bit_cast(uint32_t, bf16x2_t{(__bf16)a, (__bf16)b});
    else return __builtin_bit_cast(uint32_t, half2_t{(_Float16)a, (_Float16)b});
}

}  // namespace
}  // namespace tsq

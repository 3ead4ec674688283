// bf16 values to microscaled 4-bit codes, in registers (the format and the rounding: mx.hip).
#pragma once
#include "rtl_internal.h"

namespace rtl {
namespace {

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ u16x2 magnitudes(uint32_t w) { return __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu); }
__device__ __forceinline__ u16x2 max2(u16x2 a, u16x2 b) { return __builtin_elementwise_max(a, b); }

// Scale byte of a block whose largest magnitude has these bits.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    const uint32_t field = top >> 7;
    return field == 255 ? 255u : field > 2 ? field - 2 : 0u;
}
// The power of two of a scale byte (0: 2^-127, subnormal); 0xFF has none, the caller's codes are zero there.
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte ? byte << 23 : 0x00400000u); }

// Codes of eight values.
__device__ __forceinline__ uint32_t codes8(const uint32_t (&w)[4], uint32_t byte) {
    const float s = scale_value(byte);
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w[0]), s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w[1]), s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w[2]), s, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w[3]), s, 3);
    return byte == 255 ? 0u : r;
}

// Eight neighbouring values of a row in each of four neighbouring lanes: the scale byte of the 32, in all four.
__device__ __forceinline__ uint32_t row_scale_byte(const uint4& v) {
    const u16x2 m = max2(max2(magnitudes(v.x), magnitudes(v.y)), max2(magnitudes(v.z), magnitudes(v.w)));
    int top = max((int)m[0], (int)m[1]);
    top = max(top, __builtin_amdgcn_mov_dpp(top, 0xB1, 0xF, 0xF, true));     // lane ^ 1
    top = max(top, __builtin_amdgcn_mov_dpp(top, 0x4E, 0xF, 0xF, true));     // lane ^ 2
    return scale_byte((uint32_t)top);
}
// The bytes of four blocks (16 lanes) as one word, in all of them.
__device__ __forceinline__ uint32_t word_of_bytes(uint32_t byte) {
    int w = (int)(byte << (8 * ((threadIdx.x >> 2) & 3)));
    w |= __builtin_amdgcn_mov_dpp(w, 0x124, 0xF, 0xF, true);                 // 4 lanes round the 16
    w |= __builtin_amdgcn_mov_dpp(w, 0x128, 0xF, 0xF, true);                 // 8
    return (uint32_t)w;
}

}  // namespace
}  // namespace rtl

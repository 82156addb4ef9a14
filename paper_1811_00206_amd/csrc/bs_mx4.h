// MX 4-bit matrices (bs.h: bs_mx4_pack): E2M1 codes with a power of two for every block of 32.
//
// The matrix unit takes such numbers as they are, with both sides' scale bytes: products of codes are exact, and so is a block's sum
// before it joins the fp32 one.  Lane l of a 32x32x64 (16x16x128) instruction brings row l % 32 (l % 16) and block l / 32 (l / 16), the
// 16 bytes of a block as they lie in memory, and the scale byte of its own block.
#pragma once

#include "bs_q4.h"

namespace bs {

constexpr int64_t mx4_chunks(int64_t K) { return (K + 127) / 128; }         // of four blocks
constexpr int64_t mx4_row_bytes(int64_t K) { return 64 * mx4_chunks(K); }
constexpr int64_t mx4_scale_pitch(int64_t K) { return 4 * mx4_chunks(K); }
inline Rows mx4_codes_place(const uint8_t* codes, int64_t M, int64_t K) { return Rows(codes, 1, M * mx4_row_bytes(K), 0, 1); }
inline Rows mx4_scales_place(const uint8_t* scales, int64_t M, int64_t K) { return Rows(scales, 1, M * mx4_scale_pitch(K), 0, 1); }

#ifdef __HIPCC__

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// the scale byte of a block whose largest magnitude has these bits (compared as whole numbers, so that NaN counts as the largest)
__device__ __forceinline__ uint32_t mx4_scale(uint32_t most) {
    const uint32_t e = most >> 23;
    return e == 255 ? 255u : e < 2 ? 0u : e - 2;
}
// 2^(127 - s), the factor before rounding; 0 for blocks that are NaN, whose codes are 0
__device__ __forceinline__ float mx4_factor(uint32_t s) { return s == 255 ? 0.f : __builtin_bit_cast(float, (254u - s) << 23); }

// 8 values of a block as codes.  |v| factor < 8 is exact, or so small that its code is 0; the hardware's conversion rounds halfway
// cases to the even code.
__device__ __forceinline__ uint32_t mx4_codes(const float (&v)[8], float factor) {
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = __builtin_amdgcn_fmed3f(v[i] * factor, -6.f, 6.f);
    uint32_t word = 0;
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, q[0], q[1], 1.0f, 0);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, q[2], q[3], 1.0f, 1);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, q[4], q[5], 1.0f, 2);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, q[6], q[7], 1.0f, 3);
    return factor == 0.f ? 0u : word;
}
__device__ __forceinline__ uint32_t mx4_most(const float (&v)[8]) {
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max(most, __builtin_bit_cast(uint32_t, v[i]) & 0x7fffffffu);
    return most;
}
// the largest of four neighbouring lanes' numbers
__device__ __forceinline__ uint32_t max_of_4(uint32_t v) {
    v = max(v, (uint32_t)dpp_move_i<0xB1>((int)v));
    return max(v, (uint32_t)dpp_move_i<0x4E>((int)v));
}

__device__ __forceinline__ i32x8 mx4_operand(uint4 a) { return i32x8{(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}; }

#endif  // __HIPCC__

}  // namespace bs

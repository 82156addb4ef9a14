// 4-bit matrices (bs.h: bs_q4_pack): the walk that their products share.
//
// A wavefront multiplies 16 rows of the matrix by 16 "virtual rows" of activations with one 16x16x32 matrix
// instruction per 32 columns.  Lane l = 16 * kb + r brings 8 columns, 32 * step + 8 * kb .. + 7, of matrix row r and of
// virtual row r, and ends with the sums of matrix row r and virtual rows 4 * kb .. 4 * kb + 3.  E2M1 values are exact in
// bfloat16 and binary16 (`v_cvt_scalef32_pk_*_fp4`: two values an instruction), products are exact in the matrix unit,
// sums are fp32, and the group's scale is applied to the fp32 sum of the group: no weight is ever rounded.
//
// A 16-bit activation is one virtual row.  An fp32 activation is three (`split3`): its leading 8 bits, the next 8 and the
// last 8, each exact in bfloat16, so that the product keeps all 24 bits at the cost of rows that a few tokens leave empty.
#pragma once

#include "bs_internal.h"

namespace bs {

constexpr int kQ4Chunk = 128;      // columns of a 16-byte load per lane: 4 lanes cover 64 bytes of a row

constexpr bool q4_group_ok(int group) { return group == 32 || group == 64 || group == 128; }
constexpr int q4_group_shift(int group) { return group == 32 ? 0 : group == 64 ? 1 : 2; }   // log2(group / 32)
constexpr int64_t q4_row_bytes(int64_t K) { return 16 * ((K + 31) / 32); }
constexpr int64_t q4_groups(int64_t K, int group) { return (K + group - 1) / group; }
constexpr int64_t q4_padded(int64_t K) { return (K + kQ4Chunk - 1) / kQ4Chunk * kQ4Chunk; }
constexpr int dtype_bytes(int dtype) { return dtype == BS_F32 ? 4 : 2; }

#ifdef __HIPCC__

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// element types of activations: how a value becomes fp32 and back, and which matrix instruction takes it
struct F32 {
    using type = float;
    static constexpr int kParts = 3, kSlots = 4;      // virtual rows of a token, and the rows set aside for it
    static constexpr bool kHalf = false;
    static __device__ __forceinline__ float load(float v) { return v; }
    static __device__ __forceinline__ float store(float v) { return v; }
};
struct F16 {
    using type = uint16_t;
    static constexpr int kParts = 1, kSlots = 1;
    static constexpr bool kHalf = true;
    static __device__ __forceinline__ float load(uint16_t v) { return (float)__builtin_bit_cast(_Float16, v); }
    static __device__ __forceinline__ uint16_t store(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
};
struct BF16 {
    using type = uint16_t;
    static constexpr int kParts = 1, kSlots = 1;
    static constexpr bool kHalf = false;
    static __device__ __forceinline__ float load(uint16_t v) { return __builtin_bit_cast(float, (uint32_t)v << 16); }
    static __device__ __forceinline__ uint16_t store(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
};

// x = a + b + c with 8 leading bits each; an infinity is its own first part, a number that is none stays none in b
__device__ __forceinline__ void split3(float x, uint32_t& a, uint32_t& b, uint32_t& c) {
    a = __builtin_bit_cast(uint32_t, x) & 0xffff0000u;
    const float r = __builtin_isinf(x) ? 0.f : x - __builtin_bit_cast(float, a);
    b = __builtin_bit_cast(uint32_t, r) & 0xffff0000u;
    c = __builtin_bit_cast(uint32_t, r - __builtin_bit_cast(float, b));
}
// the upper halves of two words: the first in the low half
__device__ __forceinline__ uint32_t upper_halves(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302u); }

template <bool HALF>
__device__ __forceinline__ uint4 q4_values(uint32_t w) {   // 8 codes as 8 binary16 / bfloat16 values
    uint4 v;
    if constexpr (HALF) {
        v.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 0));
        v.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 1));
        v.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 2));
        v.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 3));
    } else {
        v.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 0));
        v.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 1));
        v.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 2));
        v.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 3));
    }
    return v;
}

template <bool HALF>
__device__ __forceinline__ f32x4 mfma_16x16x32(uint4 a, uint4 b, f32x4 c) {
    if constexpr (HALF)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Rows of 16 lanes trade places: a = (a0, a1, b0, b1), b = (a2, a3, b2, b3) / a = (a0, b0, a2, b2), b = (a1, b1, a3, b3).
// (Wait states as in add_across_16; the asm form also takes two copies of one value.)
__device__ __forceinline__ void swap_halves(uint32_t& a, uint32_t& b) {
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b));
}
__device__ __forceinline__ void swap_rows(uint32_t& a, uint32_t& b) {
    asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(a), "+v"(b));
}

// The walk of one wavefront over chunks c, c + step, ... of 16 * R matrix rows against NT tiles of 16 virtual rows.
// U chunks' loads are issued together.  `a(t, k)`: the lane's 16 bytes of tile t at column k (a multiple of 32) + 8 * kb;
// columns behind K are zero there.  GL = log2(group / 32).
template <bool HALF, int NT, int R, int GL, int U>
struct Q4Walk {
    const uint8_t* codes[R];      // the lane's row, at its 16 bytes of chunk 0
    const uint16_t* scales[R];    // the lane's row
    int kb, blocks;               // blocks: 32-column blocks of a row; a chunk is four, one for each kb
    uint4 q[R][U];
    uint32_t s[R][U];

    __device__ __forceinline__ void rows(int r, const uint8_t* c, const uint16_t* sc) { codes[r] = c + 16 * kb; scales[r] = sc; }

    __device__ __forceinline__ void load(int c, int step, int end) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int cc = c + u * step, block = 4 * cc + kb;
            const bool in = cc < end && block < blocks;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                q[r][u] = in ? *reinterpret_cast<const uint4*>(codes[r] + (int64_t)cc * 64) : uint4{0, 0, 0, 0};
                // every lane has use for the scale of a chunk that only others' columns reach
                s[r][u] = cc < end ? scales[r][min(block, blocks - 1) >> GL] : 0;
            }
        }
    }

    template <typename A>
    __device__ __forceinline__ void eat(int c, int step, int end, A&& a, f32x4 (&acc)[R][NT]) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int cc = c + u * step;
            if (cc >= end) break;
            uint32_t w[R][4];
            float sc[R][4];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                // lane kb holds block kb, words 0..3; step i wants word kb of block i
                w[r][0] = q[r][u].x; w[r][1] = q[r][u].y; w[r][2] = q[r][u].z; w[r][3] = q[r][u].w;
                swap_halves(w[r][0], w[r][2]);
                swap_halves(w[r][1], w[r][3]);
                swap_rows(w[r][0], w[r][1]);
                swap_rows(w[r][2], w[r][3]);
                // lane kb holds the scale of block kb; step i wants that of block i in every lane
                uint32_t s0 = __builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(_Float16, (uint16_t)s[r][u])), s2 = s0;
                if constexpr (GL < 2) swap_halves(s0, s2);
                uint32_t s1 = s0, s3 = s2;
                if constexpr (GL < 1) { swap_rows(s0, s1); swap_rows(s2, s3); }
                sc[r][0] = __builtin_bit_cast(float, s0); sc[r][1] = __builtin_bit_cast(float, s1);
                sc[r][2] = __builtin_bit_cast(float, s2); sc[r][3] = __builtin_bit_cast(float, s3);
            }
            f32x4 d[R][NT];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint4 x[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) x[t] = a(t, cc * kQ4Chunk + 32 * i);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const uint4 v = q4_values<HALF>(w[r][i]);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        if (i % (1 << GL) == 0) d[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
                        d[r][t] = mfma_16x16x32<HALF>(x[t], v, d[r][t]);
                        if ((i + 1) % (1 << GL) == 0) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) acc[r][t][j] = fmaf(sc[r][i], d[r][t][j], acc[r][t][j]);
                        }
                    }
                }
            }
        }
    }
};

// 8 activations from column k on; zero behind K.  `whole`: rows start on 16-byte boundaries.
template <typename XT>
__device__ __forceinline__ void load8(const typename XT::type* row, int64_t k, int64_t K, bool whole, float (&v)[8]) {
    if (whole && k + 8 <= K) {
        if constexpr (sizeof(typename XT::type) == 4) {
            const f32x4 a = *reinterpret_cast<const f32x4*>(row + k), b = *reinterpret_cast<const f32x4*>(row + k + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
        } else {
            const uint4 a = *reinterpret_cast<const uint4*>(row + k);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = XT::load((uint16_t)(word_of(a, i >> 1) >> (16 * (i & 1))));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = k + i < K ? XT::load(row[k + i]) : 0.f;
    }
}

// the three parts of 8 fp32 values, 16 bytes each
__device__ __forceinline__ void split8(const float (&v)[8], uint4 (&p)[3]) {
    uint32_t a[8], b[8], c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) split3(v[i], a[i], b[i], c[i]);
    p[0] = {upper_halves(a[0], a[1]), upper_halves(a[2], a[3]), upper_halves(a[4], a[5]), upper_halves(a[6], a[7])};
    p[1] = {upper_halves(b[0], b[1]), upper_halves(b[2], b[3]), upper_halves(b[4], b[5]), upper_halves(b[6], b[7])};
    p[2] = {upper_halves(c[0], c[1]), upper_halves(c[2], c[3]), upper_halves(c[4], c[5]), upper_halves(c[6], c[7])};
}

// 8 activations as the virtual rows' 16-byte pieces
template <typename XT>
__device__ __forceinline__ void pieces8(const typename XT::type* row, int64_t k, int64_t K, bool whole, uint4 (&p)[XT::kParts]) {
    if constexpr (XT::kParts == 3) {
        float v[8];
        load8<XT>(row, k, K, whole, v);
        split8(v, p);
    } else if (whole && k + 8 <= K) {
        p[0] = *reinterpret_cast<const uint4*>(row + k);
    } else {
        uint32_t h[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = k + i < K ? row[k + i] : 0;
        p[0] = {h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16};
    }
}

// 64-bit whole numbers in the order of what is chosen first: the larger value, then the lower index.  -0 counts as 0, a value
// that is no number comes last.  None of them is 0, none is the largest 64-bit number.
__device__ __forceinline__ uint64_t order_key(float v, uint32_t index) {
    const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.f);
    const uint32_t o = v != v ? 0u : b & 0x80000000u ? ~b : b | 0x80000000u;
    return (uint64_t)o << 32 | (0xfffffffeu - index);
}
__device__ __forceinline__ uint32_t index_of_key(uint64_t key) { return 0xfffffffeu - (uint32_t)key; }
__device__ __forceinline__ float value_of_key(uint64_t key) {
    const uint32_t o = (uint32_t)(key >> 32);
    return o ? __builtin_bit_cast(float, o & 0x80000000u ? o & 0x7fffffffu : ~o) : __builtin_nanf("");
}
__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
    for (int o = 1; o < 64; o *= 2) {
        const uint64_t other = (uint64_t)(uint32_t)__shfl_xor((int)(v >> 32), o) << 32 | (uint32_t)__shfl_xor((int)v, o);
        v = other > v ? other : v;
    }
    return v;
}

#endif  // __HIPCC__

}  // namespace bs

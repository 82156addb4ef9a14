// 4-bit matrices (bs.h: bs_q4_pack): the walk that their products share.
//
// A wavefront multiplies 16 rows of the matrix by 16 "virtual rows" of activations with one 16x16x32 matrix
// instruction per 32 columns.  Lane l = 16 * kb + r brings 8 columns, 32 * step + 8 * kb .. + 7, of matrix row r and of
// virtual row r, and ends with the sums of matrix row r and virtual rows 4 * kb .. 4 * kb + 3.  E2M1 values are exact in
// bfloat16 and binary16 (`v_cvt_scalef32_pk_*_fp4`: two values an instruction), products are exact in the matrix unit,
// sums are fp32, and the group's scale is applied to the fp32 sum of the group: no weight is ever rounded.  Sums of a walk are those of
// W x over kQ4Unit.
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

// A group's scale comes after its sum, which may therefore be larger than the result: up to 6 * 128 times an activation.  So bfloat16
// values are multiplied by 2^-10 when they are made, for nothing, and a walk's sums by kQ4Unit where they become results: both are exact,
// and nothing overflows but what a result overflows by.  (What it costs is at the other end: fp32 activations below 2^-99 lose bits, 2^-109
// otherwise.)  Binary16 activations are too small to overflow fp32 sums.
template <bool HALF>
constexpr float kQ4Unit = HALF ? 1.0f : 1024.0f;

template <bool HALF>
__device__ __forceinline__ uint4 q4_values(uint32_t w) {   // 8 codes as 8 binary16 / bfloat16 values, over kQ4Unit
    uint4 v;
    constexpr float kOver = 1.0f / kQ4Unit<HALF>;
    if constexpr (HALF) {
        v.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, kOver, 0));
        v.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, kOver, 1));
        v.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, kOver, 2));
        v.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, kOver, 3));
    } else {
        v.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, kOver, 0));
        v.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, kOver, 1));
        v.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, kOver, 2));
        v.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, kOver, 3));
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

// The walk of one wavefront over K, in steps of U adjacent chunks, of 16 * R matrix rows against NT tiles of 16 virtual rows.
// A row gives 64 bytes to a chunk, half a cache line: adjacent chunks are the same wavefront's, or the other half is fetched
// again where rows are a power of two apart (16384 x 8192: 20 us instead of 15).  Loads have no branch around them: chunks and
// blocks behind the end are read as the last ones and count for nothing, because activations behind K are zero and a code is
// always a number.  Of the scales a lane loads those of one chunk of the step, chunk kb % U, and lane exchanges spread them.
// GL = log2(group / 32).
template <bool HALF, int NT, int R, int GL, int U>
struct Q4Walk {
    static_assert(U == 2 || U == 4);
    static constexpr int kHalves = 4 >> GL, kWords = kHalves > 1 ? kHalves / 2 : 1;      // scales of a chunk
    const uint8_t* codes[R];               // the first of 16 rows (the same for all lanes)
    const uint16_t* scales[R];
    uint32_t code_at[R], scale_at[R];      // the lane's row in them
    int kb, blocks, groups;                // blocks: 32-column blocks of a row; a chunk is four, one for each kb
    uint4 next_q[R][U], q[R][U];
    uint32_t next_s[R][kWords], s[R][kWords];

    // tile i: matrix rows row .. row + 15 of a matrix of `rows` (those behind it repeat its last row)
    __device__ __forceinline__ void tile(int i, const uint8_t* c, const uint16_t* sc, int64_t row, int64_t rows, int64_t K, int lane) {
        const int64_t pitch = q4_row_bytes(K);
        row = min(row, rows - 1);
        const uint32_t r = (uint32_t)min((int64_t)(lane & 15), rows - 1 - row);
        kb = lane >> 4;
        blocks = (int)((K + 31) >> 5);
        groups = (int)((K + (32 << GL) - 1) >> (5 + GL));
        codes[i] = c + row * pitch;
        scales[i] = sc + row * groups;
        code_at[i] = r * (uint32_t)pitch;
        scale_at[i] = r * (uint32_t)groups;
    }

    __device__ __forceinline__ void load(int c) {      // chunks c .. c + U - 1
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t block = (uint32_t)min(4 * (c + u) + kb, blocks - 1);
#pragma unroll
            for (int r = 0; r < R; ++r) next_q[r][u] = *reinterpret_cast<const uint4*>(codes[r] + (code_at[r] + 16 * block));
        }
        const int first = (c + (kb & (U - 1))) * kHalves;
        if ((c + U) * kHalves <= groups) {
#pragma unroll
            for (int r = 0; r < R; ++r) __builtin_memcpy(next_s[r], scales[r] + (scale_at[r] + (uint32_t)first), 2 * kHalves);
        } else {
            uint16_t h[4];
#pragma unroll
            for (int r = 0; r < R; ++r) {
#pragma unroll
                for (int i = 0; i < kHalves; ++i) h[i] = scales[r][scale_at[r] + (uint32_t)min(first + i, groups - 1)];
                __builtin_memcpy(next_s[r], h, 2 * kHalves);
            }
        }
    }

    // Takes what load() has brought.  The copies are real ones (the empty statements), so that the registers a load writes are
    // free again and the next step can fly while this one is multiplied.
    __device__ __forceinline__ void take() {
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                q[r][u] = next_q[r][u];
                asm volatile("" : "+v"(q[r][u].x), "+v"(q[r][u].y), "+v"(q[r][u].z), "+v"(q[r][u].w));
            }
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                s[r][i] = next_s[r][i];
                asm volatile("" : "+v"(s[r][i]));
            }
        }
    }

    // chunks c + U0 .. c + U1 - 1 of the step; x(t, c, u, i): the lane's 16 bytes of tile t at column 32 * i + 8 * kb of chunk
    // c + u.  Chunks from `end` on are left out.
    template <int U0, int U1, typename X>
    __device__ __forceinline__ void eat(int c, int end, X&& x, const uint32_t (&sc)[R][kWords][4], f32x4 (&acc)[R][NT]) {
#pragma unroll
        for (int u = U0; u < U1; ++u) {
            if (c + u >= end) break;
            uint32_t w[R][4];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                // lane kb holds block kb, words 0..3; step i wants word kb of block i
                w[r][0] = q[r][u].x; w[r][1] = q[r][u].y; w[r][2] = q[r][u].z; w[r][3] = q[r][u].w;
                swap_halves(w[r][0], w[r][2]);
                swap_halves(w[r][1], w[r][3]);
                swap_rows(w[r][0], w[r][1]);
                swap_rows(w[r][2], w[r][3]);
            }
            f32x4 d[R][NT];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint4 v[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) v[t] = x(t, c, u, i);
                const int g = i >> GL;      // the group in the chunk
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const uint4 b = q4_values<HALF>(w[r][i]);
                    const uint32_t word = sc[r][g >> 1][u];
                    const float scale = (float)__builtin_bit_cast(_Float16, (uint16_t)(g & 1 ? word >> 16 : word));
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        if (i % (1 << GL) == 0) d[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
                        d[r][t] = mfma_16x16x32<HALF>(v[t], b, d[r][t]);
                        if ((i + 1) % (1 << GL) == 0) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) acc[r][t][j] = fmaf(scale, d[r][t][j], acc[r][t][j]);
                        }
                    }
                }
            }
        }
    }

    __device__ __forceinline__ void spread(uint32_t (&sc)[R][kWords][4]) {      // the scales of chunk c + u in every lane
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                uint32_t s0 = s[r][i], s2 = s0;
                if constexpr (U == 4) swap_halves(s0, s2);
                uint32_t s1 = s0, s3 = s2;
                swap_rows(s0, s1);
                if constexpr (U == 4) swap_rows(s2, s3);
                sc[r][i][0] = s0; sc[r][i][1] = s1; sc[r][i][2] = s2; sc[r][i][3] = s3;
            }
    }

    // Steps c, c + stride, ... before `end`, the first of which is loaded already.  x.fetch(c, u) issues the loads of chunk
    // c + u of x, where it has any; they come before those of the next step, because loads arrive in order: whoever waits for
    // x does not wait for them.  FETCH: chunks of x that are held at once.
    template <int FETCH, typename X>
    __device__ __forceinline__ void rest(int c, int stride, int end, X& x, f32x4 (&acc)[R][NT]) {
        static_assert(FETCH == U || (FETCH == 1 && U == 2));
        while (c < end) {
            const int now = c;
            take();
            c += stride * U;
            uint32_t sc[R][kWords][4];
#pragma unroll
            for (int u = 0; u < FETCH; ++u) x.fetch(now, u);
            if constexpr (FETCH == 1) {
                spread(sc);
                eat<0, 1>(now, end, x, sc, acc);
                x.fetch(now, 1);
            }
            if (c < end) load(c);
            if constexpr (FETCH == 1) {
                eat<1, 2>(now, end, x, sc, acc);
            } else {
                spread(sc);
                eat<0, U>(now, end, x, sc, acc);
            }
        }
    }
};

__device__ __forceinline__ uint4 bits8(const uint16_t* row, int64_t k, int64_t K);

// x of a walk, read from memory: virtual rows at[t], 16-byte pieces from column 8 * kb on, zero behind `columns`, which are
// whole chunks unless RAGGED.  Chunks are read as far as there are any.  A lane without a virtual row loads nothing (few rows
// cost few of the cache's cycles) and brings what its registers hold: that reaches sums of that row alone, which nobody reads.
template <int NT, int FETCH, bool RAGGED>
struct RowsOfX {
    const uint16_t* at[NT];     // nullptr: none
    int kb, columns, last;      // last: the last chunk
    uint4 v[NT][FETCH][4];
    __device__ __forceinline__ void fetch(int c, int u) {
        const int k = min(c + u, last) * kQ4Chunk;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            uint4 (&w)[4] = v[t][u % FETCH];
#pragma unroll
            for (int i = 0; i < 4; ++i) asm volatile("" : "=v"(w[i].x), "=v"(w[i].y), "=v"(w[i].z), "=v"(w[i].w));
            if (!at[t]) continue;
            if (!RAGGED || k + kQ4Chunk <= columns) {
#pragma unroll
                for (int i = 0; i < 4; ++i) __builtin_memcpy(&w[i], at[t] + k + 32 * i + 8 * kb, 16);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = bits8(at[t], k + 32 * i + 8 * kb, columns);
            }
        }
    }
    __device__ __forceinline__ uint4 operator()(int t, int, int u, int i) const { return v[t][u % FETCH][i]; }
};

// x of a walk in LDS: virtual rows at[t], zero behind K
template <int NT>
struct LdsRowsOfX {
    const uint16_t* at[NT];      // the lane's piece of column 0
    __device__ __forceinline__ void fetch(int, int) {}
    __device__ __forceinline__ uint4 operator()(int t, int c, int u, int i) const {
        return *reinterpret_cast<const uint4*>(at[t] + (c + u) * kQ4Chunk + 32 * i);
    }
};

// x of a walk as the matrix unit takes it: 1 KB, the wavefront's 16-byte pieces side by side, for every tile, chunk and 32
// columns of it (tile by tile, `chunks` chunks each)
template <int NT, int FETCH>
struct TilesOfX {
    const uint16_t* at[NT];      // the lane's piece of a tile's chunk 0
    int last;
    uint4 v[NT][FETCH][4];
    __device__ __forceinline__ void fetch(int c, int u) {
        const int cc = min(c + u, last);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[t][u % FETCH][i] = *reinterpret_cast<const uint4*>(at[t] + (cc * 4 + i) * 512);
    }
    __device__ __forceinline__ uint4 operator()(int t, int, int u, int i) const { return v[t][u % FETCH][i]; }
};

// 8 elements of a row that were loaded from column `from` = min(k, K - 8), as those from column k on, zero behind K
__device__ __forceinline__ uint4 moved8(uint4 v, int64_t k, int64_t from, int64_t K) {
    if (k == from) return v;
    return k < K ? __builtin_bit_cast(uint4, __builtin_bit_cast(unsigned __int128, v) >> (16 * (int)(k - from))) : uint4{0, 0, 0, 0};
}
__device__ __forceinline__ void moved8(float (&v)[8], int64_t k, int64_t from) {
    if (k == from) return;
    const int by = (int)min(k - from, (int64_t)8);      // 3 bits of the distance, one after the other; 8: nothing is left
#pragma unroll
    for (int step = 4; step; step /= 2)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = by & step ? (i + step < 8 ? v[i + step] : 0.f) : v[i];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = by & 8 ? 0.f : v[i];
}

// 8 elements of a row from column k on, zero behind K; the row may start anywhere.  A piece that is not whole is the row's
// last 8 elements, moved: no lane loads element by element, which would be eight trips to memory one after the other.
__device__ __forceinline__ uint4 bits8(const uint16_t* row, int64_t k, int64_t K) {
    uint4 v{0, 0, 0, 0};
    if (K >= 8) {
        const int64_t from = min(k, K - 8);
        __builtin_memcpy(&v, row + from, 16);
        v = moved8(v, k, from, K);
    } else {
        uint32_t h[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = k + i < K ? row[k + i] : 0;
        v = {h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16};
    }
    return v;
}

template <typename XT>
__device__ __forceinline__ void load8(const typename XT::type* row, int64_t k, int64_t K, float (&v)[8]) {
    if constexpr (sizeof(typename XT::type) == 2) {
        const uint4 a = bits8(row, k, K);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = XT::load((uint16_t)(word_of(a, i >> 1) >> (16 * (i & 1))));
    } else if (K >= 8) {
        const int64_t from = min(k, K - 8);
        __builtin_memcpy(v, row + from, 32);
        moved8(v, k, from);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = k + i < K ? row[k + i] : 0.f;
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
__device__ __forceinline__ void pieces8(const typename XT::type* row, int64_t k, int64_t K, uint4 (&p)[XT::kParts]) {
    if constexpr (XT::kParts == 3) {
        float v[8];
        load8<XT>(row, k, K, v);
        split8(v, p);
    } else {
        p[0] = bits8(row, k, K);
    }
}

// the largest of a wavefront's values, in every lane; what is no number counts only where nothing else does
__device__ __forceinline__ float max_of_wave(float v) {
    v = fmaxf(v, dpp_move<0xB1>(v));
    v = fmaxf(v, dpp_move<0x4E>(v));
    v = fmaxf(v, dpp_move<0x141>(v));
    v = fmaxf(v, dpp_move<0x140>(v));
    uint32_t a = __builtin_bit_cast(uint32_t, v), b = a;
    swap_rows(a, b);
    v = fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
    a = b = __builtin_bit_cast(uint32_t, v);
    swap_halves(a, b);
    return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}
__device__ __forceinline__ float sum_of_wave(float v) { return add_across_32(add_across_16(group_sum<16>(v))); }

// Of `all` workgroups that have stored their sums with the scope of the whole GPU, by all threads: whether this one is the last,
// and may load all of them with that scope.  Sums stored that way are where everybody sees them as soon as each lane has waited
// for its own; a fence of that scope would write back all that the cache holds, which took 16 us.  `found`: a word of LDS.
__device__ __forceinline__ bool last_of(uint32_t* done, int all, int* found) {
    pin_order();      // the wait is for all stores before it, and the count comes after it
    wait_vm_and_lds<0>();
    pin_order();
    __syncthreads();
    if (threadIdx.x == 0) *found = (int)__hip_atomic_fetch_add(done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    return *found == all - 1;
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
// the largest of a wavefront's 64-bit numbers, in every lane
template <int CTRL>
__device__ __forceinline__ uint64_t max_moved(uint64_t v) {
    const uint64_t other = (uint64_t)(uint32_t)dpp_move_i<CTRL>((int)(v >> 32)) << 32 | (uint32_t)dpp_move_i<CTRL>((int)v);
    return other > v ? other : v;
}
__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
    v = max_moved<0xB1>(v);
    v = max_moved<0x4E>(v);
    v = max_moved<0x141>(v);
    v = max_moved<0x140>(v);
    uint32_t h0 = (uint32_t)(v >> 32), h1 = h0, l0 = (uint32_t)v, l1 = l0;
    swap_rows(h0, h1);
    swap_rows(l0, l1);
    uint64_t a = (uint64_t)h0 << 32 | l0, b = (uint64_t)h1 << 32 | l1;
    v = a > b ? a : b;
    h0 = h1 = (uint32_t)(v >> 32), l0 = l1 = (uint32_t)v;
    swap_halves(h0, h1);
    swap_halves(l0, l1);
    a = (uint64_t)h0 << 32 | l0, b = (uint64_t)h1 << 32 | l1;
    return a > b ? a : b;
}

#endif  // __HIPCC__

}  // namespace bs

// Dense matrix to 4-bit codes with group scales, and back (bs.h: bs_q4_pack, bs_q4_unpack).  Bound: HBM, each side once.
//
// A lane holds 8 consecutive elements of a row, 4 to 16 lanes a group: the group's largest magnitude is a few lane
// exchanges away.  A code is the nearest one for every input, halfway cases to the even one:
//   fp32       magnitudes are compared with the halfway points times the scale, which are exact products in fp32 (a halfway
//              point has at most 3 significant bits, a binary16 scale 11).  Three comparisons, each with the point that the ones
//              before leave in question; the points at which an even code wins the tie (.75, 1.75, 3.5) are those of the first two.
//   16 bits    w / s, for w and s of at most 11 bits and a halfway point h of 3, is either h or 2^-15 of it away.  So the product
//              with the reciprocal, off by 2^-21 at most, is rounded to 18 bits, is then h where it should be, and the
//              hardware's conversion (two values an instruction, halfway cases to even) has the last word: 16384 x 8192 in
//              bfloat16 105 us with comparisons, 72 with it (the least of a trace; its median, over three matrices in turn, is 82).
#include "bs_q4.h"

namespace bs {
namespace {

typedef uint32_t Unaligned __attribute__((ext_vector_type(4), aligned(2)));      // 16 bytes anywhere

template <int W>
__device__ __forceinline__ float group_max(float v) {       // of W = 4, 8 or 16 neighbouring lanes
    v = fmaxf(v, dpp_move<0xB1>(v));
    v = fmaxf(v, dpp_move<0x4E>(v));
    if constexpr (W >= 8) v = fmaxf(v, dpp_move<0x141>(v));
    if constexpr (W >= 16) v = fmaxf(v, dpp_move<0x140>(v));
    return v;
}

// the piece of 8 elements that a thread has: row, and number inside the row (`pieces` of them, whole groups)
__device__ __forceinline__ void piece_of(uint32_t pieces, uint32_t magic, int64_t& row, uint32_t& piece) {
    const uint32_t e = blockIdx.x * 256 + threadIdx.x, q = div_magic_any(e, pieces, magic);
    row = q;
    piece = e - q * pieces;
}

template <typename XT, int GL>
__global__ __launch_bounds__(256) void q4_pack_kernel(const typename XT::type* W, int64_t M, int64_t K, uint32_t pieces,
                                                      uint32_t magic, uint8_t* codes, uint16_t* scales) {
    int64_t row;
    uint32_t piece;
    piece_of(pieces, magic, row, piece);
    float v[8] = {};
    const int64_t k = (int64_t)piece * 8;
    if (row < M) load8<XT>(W + row * K, k, K, v);
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(v[i]));
    most = group_max<(4 << GL)>(most);
    if (row >= M) return;
    // binary16 is as near as a scale needs to be (the codes are a hundred times coarser); larger ones than it holds are cut
    const _Float16 scale = (_Float16)fminf(most * (1.0f / 6.0f), 65504.0f);
    const float s = (float)scale;
    uint32_t word = 0;
    if constexpr (sizeof(typename XT::type) == 4) {
        const float h0 = 0.25f * s, h1 = 0.75f * s, h2 = 1.25f * s, h3 = 1.75f * s, h4 = 2.5f * s, h5 = 3.5f * s, h6 = 5.0f * s;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float a = fabsf(v[i]);
            const bool c4 = a >= h3;
            const bool c2 = a >= (c4 ? h5 : h1);
            const float lo = c4 ? h4 : h0, hi = c4 ? h6 : h2;
            const bool c1 = a > (c2 ? hi : lo);
            uint32_t code = (c4 ? 4 : 0) | (c2 ? 2 : 0) | (c1 ? 1 : 0);
            if (s == 0.f) code = 0;
            word |= (code | (v[i] < 0.f ? 8u : 0u)) << (4 * i);
        }
    } else {
        const float inverse = s == 0.f ? 0.f : __builtin_amdgcn_rcpf(s);
        float q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {      // (+ 0 makes a negative zero a positive one, whose code has no sign)
            const uint32_t bits = __builtin_bit_cast(uint32_t, fmaf(v[i], inverse, 0.f));
            q[i] = __builtin_bit_cast(float, (bits + 0x20u) & ~0x3fu);
            if (s == 0.f) q[i] = v[i] < 0.f ? -0.f : 0.f;
        }
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, q[0], q[1], 1.0f, 0);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, q[2], q[3], 1.0f, 1);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, q[4], q[5], 1.0f, 2);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, q[6], q[7], 1.0f, 3);
    }
    const int64_t pitch = q4_row_bytes(K);
    if (k / 2 < pitch) *reinterpret_cast<uint32_t*>(codes + row * pitch + k / 2) = word;
    if (piece % (4 << GL) == 0) scales[row * (pieces >> (2 + GL)) + (piece >> (2 + GL))] = __builtin_bit_cast(uint16_t, scale);
}

template <typename XT, int GL>
__global__ __launch_bounds__(256) void q4_unpack_kernel(const uint8_t* codes, const uint16_t* scales, int64_t M, int64_t K,
                                                        uint32_t pieces, uint32_t magic, typename XT::type* W) {
    int64_t row;
    uint32_t piece;
    piece_of(pieces, magic, row, piece);
    const int64_t k = (int64_t)piece * 8;
    if (row >= M || k >= K) return;
    const int64_t groups = (K + (32 << GL) - 1) >> (5 + GL);
    const uint32_t word = *reinterpret_cast<const uint32_t*>(codes + row * q4_row_bytes(K) + k / 2);
    const float s = (float)__builtin_bit_cast(_Float16, scales[row * groups + (k >> (5 + GL))]);
    const f32x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 1),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 3)};
    uint32_t out[sizeof(typename XT::type) * 2];      // 8 elements
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const auto v = XT::store(p[i / 2][i % 2] * s);
        if constexpr (sizeof(v) == 4) out[i] = __builtin_bit_cast(uint32_t, v);
        else out[i / 2] = i % 2 ? out[i / 2] | (uint32_t)v << 16 : v;
    }
    typename XT::type* to = W + row * K + k;
    if (k + 8 <= K) {      // wherever the row starts
#pragma unroll
        for (int i = 0; i < (int)sizeof(typename XT::type) / 2; ++i)
            reinterpret_cast<Unaligned*>(to)[i] = Unaligned{out[4 * i], out[4 * i + 1], out[4 * i + 2], out[4 * i + 3]};
        return;
    }
    // a row's last piece, two elements of 16 bits to a word
    for (int i = 0; k + i < K; ++i) {
        uint32_t w = out[0];
#pragma unroll
        for (int j = 1; j < (int)(sizeof(out) / 4); ++j) w = (int)(i * sizeof(*to) / 4) == j ? out[j] : w;
        if constexpr (sizeof(*to) == 4) to[i] = __builtin_bit_cast(float, w);
        else to[i] = (uint16_t)(w >> (16 * (i & 1)));
    }
}

template <typename XT, int GL>
int launch(const void* W, int64_t M, int64_t K, uint8_t* codes, uint16_t* scales, void* out, hipStream_t st) {
    const int group = 32 << GL;
    const uint32_t pieces = (uint32_t)(q4_groups(K, group) * (group / 8));
    using T = typename XT::type;
    const int64_t most = ((int64_t)1 << 31) / pieces;      // rows of a launch: a grid has fewer than 2^32 lanes
    for (int64_t r = 0; r < M; r += most) {
        const int64_t rows = M - r < most ? M - r : most;
        const dim3 grid((unsigned)((rows * pieces + 255) / 256));
        uint8_t* const c = codes + r * q4_row_bytes(K);
        uint16_t* const s = scales + r * q4_groups(K, group);
        if (out)
            hipLaunchKernelGGL((q4_unpack_kernel<XT, GL>), grid, dim3(256), 0, st, c, s, rows, K, pieces, magic_u32(pieces),
                               static_cast<T*>(out) + r * K);
        else
            hipLaunchKernelGGL((q4_pack_kernel<XT, GL>), grid, dim3(256), 0, st, static_cast<const T*>(W) + r * K, rows, K, pieces,
                               magic_u32(pieces), c, s);
        const int rc = hip_status(hipGetLastError());
        if (rc != BS_OK) return rc;
    }
    return BS_OK;
}

template <typename XT>
int launch_group(const void* W, int64_t M, int64_t K, int group, uint8_t* codes, uint16_t* scales, void* out, hipStream_t st) {
    switch (q4_group_shift(group)) {
        case 0: return launch<XT, 0>(W, M, K, codes, scales, out, st);
        case 1: return launch<XT, 1>(W, M, K, codes, scales, out, st);
        default: return launch<XT, 2>(W, M, K, codes, scales, out, st);
    }
}

}  // namespace

// `out`: nullptr to pack W, else where the codes' values go
int launch_q4_pack(const void* W, int dtype, int64_t M, int64_t K, int group, uint8_t* codes, uint16_t* scales, void* out, hipStream_t st) {
    switch (dtype) {
        case BS_F32: return launch_group<F32>(W, M, K, group, codes, scales, out, st);
        case BS_F16: return launch_group<F16>(W, M, K, group, codes, scales, out, st);
        default: return launch_group<BF16>(W, M, K, group, codes, scales, out, st);
    }
}

}  // namespace bs

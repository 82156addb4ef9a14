// Dense matrix to MX 4-bit and back (bs.h: bs_mx4_pack, bs_mx4_unpack).  Bound: HBM, each side once.
//
// A lane holds 8 consecutive elements of a row and four lanes a block, so that the largest magnitude is two lane exchanges away; 16
// lanes gather the four scale bytes of a word.  Magnitudes are compared as whole numbers, infinities and NaN the largest.
// 6000 x 3000 in fp32 13.5 us and back 16.3, 16384 x 8192 in bfloat16 66 to 76 and 57 to 61 (a copy of as many bytes 16.0 and 66).
#include "bs_mx4.h"

namespace bs {
namespace {

typedef uint32_t Unaligned __attribute__((ext_vector_type(4), aligned(2)));      // 16 bytes anywhere

// the piece of 8 elements that a thread has: row, and number inside the row (`pieces` of them, whole chunks)
__device__ __forceinline__ void piece_of(uint32_t pieces, uint32_t magic, int64_t& row, uint32_t& piece) {
    const uint32_t e = blockIdx.x * 256 + threadIdx.x, q = div_magic_any(e, pieces, magic);
    row = q;
    piece = e - q * pieces;
}

template <typename XT>
__global__ __launch_bounds__(256) void mx4_pack_kernel(const typename XT::type* W, int64_t M, int64_t K, int64_t ld, uint32_t pieces,
                                                       uint32_t magic, uint8_t* codes, uint8_t* scales) {
    int64_t row;
    uint32_t piece;
    piece_of(pieces, magic, row, piece);
    float v[8] = {};
    const int64_t k = (int64_t)piece * 8;
    if (row < M && k < K) load8<XT>(W + row * ld, k, K, v);
    const uint32_t s = mx4_scale(max_of_4(mx4_most(v)));
    const uint32_t word = mx4_codes(v, mx4_factor(s));
    // the scale bytes of 16 lanes, one from each four
    uint32_t bytes = (k / 32 * 32 < K ? s : 127u) << (piece / 4 % 4 * 8);
    bytes |= (uint32_t)dpp_move_i<0x141>((int)bytes);
    bytes |= (uint32_t)dpp_move_i<0x140>((int)bytes);
    if (row >= M) return;
    reinterpret_cast<uint32_t*>(codes)[row * pieces + piece] = word;
    if (piece % 16 == 0) reinterpret_cast<uint32_t*>(scales)[row * (pieces / 16) + piece / 16] = bytes;
}

template <typename XT>
__global__ __launch_bounds__(256) void mx4_unpack_kernel(const uint8_t* codes, const uint8_t* scales, int64_t M, int64_t K,
                                                         uint32_t pieces, uint32_t magic, typename XT::type* W) {
    int64_t row;
    uint32_t piece;
    piece_of(pieces, magic, row, piece);
    const int64_t k = (int64_t)piece * 8;
    if (row >= M || k >= K) return;
    const uint32_t word = reinterpret_cast<const uint32_t*>(codes)[row * pieces + piece];
    const uint32_t b = scales[row * (pieces / 4) + piece / 4];
    const float s = __builtin_bit_cast(float, b == 255 ? 0x7fc00000u : b ? b << 23 : 0x00400000u);
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
#pragma unroll
    for (int i = 0; i < 8; ++i) {      // a row's last piece
        if (k + i >= K) break;
        if constexpr (sizeof(*to) == 4) to[i] = __builtin_bit_cast(float, out[i]);
        else to[i] = (uint16_t)(out[i / 2] >> (16 * (i & 1)));
    }
}

// rows of a launch: a grid has fewer than 2^32 lanes
int64_t most_rows(int64_t K) { return ((int64_t)1 << 31) / (16 * mx4_chunks(K)); }

template <typename XT>
int pack(const void* W, int64_t M, int64_t K, int64_t ld, uint8_t* codes, uint8_t* scales, hipStream_t st) {
    const uint32_t pieces = (uint32_t)(16 * mx4_chunks(K));
    for (int64_t r = 0, most = most_rows(K); r < M; r += most) {
        const int64_t rows = M - r < most ? M - r : most;
        hipLaunchKernelGGL(mx4_pack_kernel<XT>, dim3((unsigned)((rows * pieces + 255) / 256)), dim3(256), 0, st,
                           static_cast<const typename XT::type*>(W) + r * ld, rows, K, ld, pieces, magic_u32(pieces),
                           codes + r * mx4_row_bytes(K), scales + r * mx4_scale_pitch(K));
        const int rc = hip_status(hipGetLastError());
        if (rc != BS_OK) return rc;
    }
    return BS_OK;
}

template <typename XT>
int unpack(const uint8_t* codes, const uint8_t* scales, int64_t M, int64_t K, void* W, hipStream_t st) {
    const uint32_t pieces = (uint32_t)(16 * mx4_chunks(K));
    for (int64_t r = 0, most = most_rows(K); r < M; r += most) {
        const int64_t rows = M - r < most ? M - r : most;
        hipLaunchKernelGGL(mx4_unpack_kernel<XT>, dim3((unsigned)((rows * pieces + 255) / 256)), dim3(256), 0, st,
                           codes + r * mx4_row_bytes(K), scales + r * mx4_scale_pitch(K), rows, K, pieces, magic_u32(pieces),
                           static_cast<typename XT::type*>(W) + r * K);
        const int rc = hip_status(hipGetLastError());
        if (rc != BS_OK) return rc;
    }
    return BS_OK;
}

}  // namespace

int launch_mx4_pack(const void* W, int dtype, int64_t M, int64_t K, int64_t ld, uint8_t* codes, uint8_t* scales, hipStream_t st) {
    switch (dtype) {
        case BS_F32: return pack<F32>(W, M, K, ld, codes, scales, st);
        case BS_F16: return pack<F16>(W, M, K, ld, codes, scales, st);
        default: return pack<BF16>(W, M, K, ld, codes, scales, st);
    }
}

int launch_mx4_unpack(const uint8_t* codes, const uint8_t* scales, int64_t M, int64_t K, void* W, int dtype, hipStream_t st) {
    switch (dtype) {
        case BS_F32: return unpack<F32>(codes, scales, M, K, W, st);
        case BS_F16: return unpack<F16>(codes, scales, M, K, W, st);
        default: return unpack<BF16>(codes, scales, M, K, W, st);
    }
}

}  // namespace bs

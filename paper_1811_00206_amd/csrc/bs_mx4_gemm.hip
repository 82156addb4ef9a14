// Rows of activations times an MX 4-bit matrix (bs.h: bs_mx4_gemm, bs_mx4_gemm_packed).
//
// A workgroup has 16 rows of W and 16 * NT rows of x, its wavefronts take turns with the steps of K, and their sums meet in LDS.
#include <type_traits>

#include "bs_mx4_tiles.h"

namespace bs {
namespace {

struct Args {
    const uint8_t *codes, *scales, *x_codes, *x_scales;
    int64_t M, N;
    int chunks;
    const float* bias;
    void* y;
    int64_t ldy;
};

template <typename XT, int NT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void mx4_rows_kernel(Args g) {
    __shared__ f32x4 sums[WAVES][NT][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, kb = lane >> 4;
    const int64_t m0 = (int64_t)blockIdx.x * 16, n0 = (int64_t)blockIdx.y * 16 * NT;
    const int64_t wrow = min(m0 + r, g.M - 1);
    const uint8_t* const w = g.codes + wrow * 64 * g.chunks + 16 * kb;
    const uint32_t* const ws = reinterpret_cast<const uint32_t*>(g.scales) + wrow * g.chunks;
    const uint8_t* x[NT];
    const uint32_t* xs[NT];
    f32x4 acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int64_t row = min(n0 + 16 * t + r, g.N - 1);
        x[t] = g.x_codes + row * 64 * g.chunks + 16 * kb;
        xs[t] = reinterpret_cast<const uint32_t*>(g.x_scales) + row * g.chunks;
        acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (int c = wave; c < g.chunks; c += WAVES) {
        const uint4 a = *reinterpret_cast<const uint4*>(w + (int64_t)c * 64);
        const uint32_t sa = ws[c] >> (8 * kb);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const uint4 b = *reinterpret_cast<const uint4*>(x[t] + (int64_t)c * 64);
            const uint32_t sb = xs[t][c] >> (8 * kb);
            acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx4_operand(a), mx4_operand(b), acc[t], 4, 4, 0, (int)sa, 0, (int)sb);
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) sums[wave][t][lane] = acc[t];
    __syncthreads();
    for (int i = threadIdx.x; i < NT * 64; i += 64 * WAVES) {
        const int t = i >> 6, l = i & 63;
        f32x4 s = sums[0][t][l];
        for (int v = 1; v < WAVES; ++v) s += sums[v][t][l];
        const int64_t n = n0 + 16 * t + (l & 15), m = m0 + 4 * (l >> 4);
        if (n >= g.N) continue;
        typename XT::type* const y = static_cast<typename XT::type*>(g.y) + n * g.ldy;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (m + j < g.M) y[m + j] = XT::store(g.bias ? s[j] + g.bias[m + j] : s[j]);
    }
}

// ---- tiles

template <typename XT, int TN, int TM, int WN, int WM>
int launch_tiles(Mx4Tiles g, hipStream_t st) {
    constexpr auto kernel = mx4_tiles_kernel<XT, TN, TM, WN, WM, false>;
    LdsKernel& reg = LdsKernelOf<kernel>::reg;
    const int rc = ensure_lds_limit(reg, st);
    if (rc != BS_OK) return rc;
    g.m_tiles = (int)((g.M + TM - 1) / TM);
    g.n_tiles = (int)((g.N + TN - 1) / TN);
    g.split = 1;
    g.stages = (g.chunks + 1) / 2;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(g.m_tiles * g.n_tiles)), dim3(256), (kMx4LdsBytes<TN, TM>), st, g);
    return hip_status(hipGetLastError());
}

template <typename XT>
int launch(Args g, hipStream_t st) {
    if (g.N > 16) {
        Mx4Tiles t{};
        t.codes = g.codes; t.scales = g.scales; t.x_codes = g.x_codes; t.x_scales = g.x_scales;
        t.M = g.M; t.N = g.N; t.chunks = g.chunks; t.bias = g.bias; t.y = g.y; t.ldy = g.ldy;
        if (g.N > 1024) return launch_tiles<XT, 256, 256, 2, 2>(t, st);
        return launch_tiles<XT, 128, 128, 2, 2>(t, st);
    }
    constexpr int NT = 4;
    const int64_t most = (int64_t)65535 * 16 * NT;      // tokens of a launch
    const int64_t N = g.N;
    for (int64_t n = 0; n < N; n += most) {
        Args p = g;
        p.N = N - n < most ? N - n : most;
        p.x_codes += n * 64 * g.chunks;
        p.x_scales += n * 4 * g.chunks;
        p.y = static_cast<typename XT::type*>(g.y) + n * g.ldy;
        const unsigned m = (unsigned)((g.M + 15) / 16);
        if (p.N <= 16) hipLaunchKernelGGL((mx4_rows_kernel<XT, 1, 4>), dim3(m, 1), dim3(256), 0, st, p);
        else hipLaunchKernelGGL((mx4_rows_kernel<XT, NT, 4>), dim3(m, (unsigned)((p.N + 16 * NT - 1) / (16 * NT))), dim3(256), 0, st, p);
        const int rc = hip_status(hipGetLastError());
        if (rc != BS_OK) return rc;
    }
    return BS_OK;
}

}  // namespace

size_t mx4_gemm_workspace_bytes(bool packed, int, int64_t, int64_t K, int64_t N) {
    return packed ? 0 : (size_t)(N * (mx4_row_bytes(K) + mx4_scale_pitch(K)) + 15) / 16 * 16;
}

int launch_mx4_gemm(const uint8_t* codes, const uint8_t* scales, int64_t M, int64_t K, const void* x, int64_t ldx, const uint8_t* x_codes,
                    const uint8_t* x_scales, int dtype, int64_t N, const float* bias, void* y, int64_t ldy, void* workspace,
                    size_t workspace_bytes, hipStream_t st) {
    const size_t need = mx4_gemm_workspace_bytes(!x, dtype, M, K, N);
    if (need && (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 15))) return BS_ERR_WORKSPACE;
    if (x) {
        uint8_t* const c = static_cast<uint8_t*>(workspace);
        uint8_t* const s = c + N * mx4_row_bytes(K);
        const int rc = launch_mx4_pack(x, dtype, N, K, ldx, c, s, st);
        if (rc != BS_OK) return rc;
        x_codes = c;
        x_scales = s;
    }
    const Args g{codes, scales, x_codes, x_scales, M, N, (int)mx4_chunks(K), bias, y, ldy};
    switch (dtype) {
        case BS_F32: return launch<F32>(g, st);
        case BS_F16: return launch<F16>(g, st);
        default: return launch<BF16>(g, st);
    }
}

}  // namespace bs

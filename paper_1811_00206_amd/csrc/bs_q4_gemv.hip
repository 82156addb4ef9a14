// y[n] = W . x[n] for a 4-bit matrix and one or a few vectors (bs.h: bs_q4_gemv).
//
// Bound: the codes are read once, M * K / 2 bytes.  A workgroup owns 16 * R rows; its wavefronts share K between them
// (chunk c of 128 columns goes to wavefront c % ways), so that a few thousand rows already fill the chip, and add their
// sums in LDS in the order of the wavefronts: the same bits from every call.
//
// Up to 16 virtual rows (16 vectors in 16 bits, 4 in fp32) the workgroup brings x to LDS itself, in slabs of K, split into
// its parts there.  With more, a first kernel writes the parts of every vector to the workspace, padded with zeros, and
// the product reads them from there: what a workgroup needs of x no longer fits LDS, and one split serves all workgroups.
#include "bs_q4.h"

namespace bs {
namespace {

constexpr int kU = 4;                       // chunks in flight per wavefront
constexpr size_t kSlabBytes = 48 * 1024;    // of x in LDS

struct GemvArgs {
    const uint8_t* codes;
    const uint16_t* scales;
    int64_t M, K, N, ldx, ldy;
    const void* x;      // as given, or the parts of every vector in the workspace
    void* y;
    int ways, slab;     // wavefronts that share K; columns of x in LDS at once
    bool whole;         // rows of x start on 16-byte boundaries
};

template <typename XT, int NT, int R, int GL, bool STAGED>
__global__ __launch_bounds__(STAGED ? 1024 : 512) void q4_gemv_kernel(GemvArgs g) {
    using T = typename XT::type;
    constexpr int P = XT::kParts, S = XT::kSlots, TPT = 16 / S;     // tokens per tile of virtual rows
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x & 63, kb = lane >> 4, r = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row0 = (int64_t)blockIdx.x * (16 * R);
    const int64_t n0 = (int64_t)blockIdx.y * (NT * TPT);
    const int tokens = (int)min(g.N - n0, (int64_t)(NT * TPT));
    const int chunks = (int)((g.K + kQ4Chunk - 1) / kQ4Chunk);

    Q4Walk<XT::kHalf, NT, R, GL, kU> walk;
    walk.kb = kb;
    walk.blocks = (int)((g.K + 31) / 32);
    const int64_t pitch = q4_row_bytes(g.K), groups = (g.K + (32 << GL) - 1) >> (5 + GL);
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int64_t row = min(row0 + 16 * i + r, g.M - 1);
        walk.rows(i, g.codes + row * pitch, g.scales + row * groups);
    }
    f32x4 acc[R][NT] = {};
    // the lane's virtual row of tile t, in tokens of this workgroup; rows without a token repeat the last one
    const int part = min(r % S, P - 1);

    if constexpr (STAGED) {
        static_assert(NT == 1);
        uint16_t* xs = reinterpret_cast<uint16_t*>(lds);
        const int xp = g.slab + 8;                              // row pitch: 16 bytes more, so that rows start on other banks
        const uint16_t* mine = xs + (min(r / S, tokens - 1) * P + part) * xp + 8 * kb;
        const int per_slab = g.slab / kQ4Chunk;
        for (int c0 = 0; c0 < chunks; c0 += per_slab) {
            const int end = min(chunks, c0 + per_slab);
            int c = c0 + wave;
            walk.load(c, g.ways, end);
            if (c0) __syncthreads();
            const int64_t k0 = (int64_t)c0 * kQ4Chunk;
            const int pieces = (end - c0) * (kQ4Chunk / 8);
            for (int n = 0; n < tokens; ++n) {
                const T* row = static_cast<const T*>(g.x) + (n0 + n) * g.ldx;
                for (int j = threadIdx.x; j < pieces; j += blockDim.x) {
                    uint4 p[P];
                    pieces8<XT>(row, k0 + 8 * j, g.K, g.whole, p);
#pragma unroll
                    for (int i = 0; i < P; ++i) *reinterpret_cast<uint4*>(xs + (n * P + i) * xp + 8 * j) = p[i];
                }
            }
            __syncthreads();
            const uint16_t* at = mine - k0;
            while (c < end) {
                walk.eat(c, g.ways, end, [&](int, int k) { return *reinterpret_cast<const uint4*>(at + k); }, acc);
                c += kU * g.ways;
                if (c < end) walk.load(c, g.ways, end);
            }
        }
        __syncthreads();
    } else {
        const int64_t xp = q4_padded(g.K);
        const uint16_t* at[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t)
            at[t] = static_cast<const uint16_t*>(g.x) + ((n0 + min(t * TPT + r / S, tokens - 1)) * P + part) * xp + 8 * kb;
        for (int c = wave; c < chunks; c += kU * g.ways) {
            walk.load(c, g.ways, chunks);
            walk.eat(c, g.ways, chunks, [&](int t, int k) { return *reinterpret_cast<const uint4*>(at[t] + k); }, acc);
        }
    }

    // a lane's four rows are four tokens, or the parts of one (the small parts are added first)
    constexpr int V = 4 / S;
    float* sums = reinterpret_cast<float*>(lds);            // [wave][R][NT][TPT][16]
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float sum = acc[i][t][v];
                if constexpr (S == 4) sum = acc[i][t][0] + (acc[i][t][1] + acc[i][t][2]);
                sums[(((wave * R + i) * NT + t) * TPT + kb * V + v) * 16 + r] = sum;
            }
    __syncthreads();
    constexpr int kOut = R * NT * TPT * 16;
    for (int o = threadIdx.x; o < kOut; o += blockDim.x) {
        const int i = o / (NT * TPT * 16), n = o / 16 % (NT * TPT);
        const int64_t row = row0 + 16 * i + o % 16;
        if (n >= tokens || row >= g.M) continue;
        float sum = sums[o];
        for (int w = 1; w < g.ways; ++w) sum += sums[w * kOut + o];
        static_cast<T*>(g.y)[(n0 + n) * g.ldy + row] = XT::store(sum);
    }
}

// the parts of every vector, padded with zeros to whole chunks
template <typename XT>
__global__ __launch_bounds__(256) void q4_split_kernel(const void* x, int64_t K, int64_t ldx, bool whole, uint16_t* parts) {
    using T = typename XT::type;
    constexpr int P = XT::kParts;
    const int64_t n = blockIdx.y, xp = q4_padded(K), k = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (k >= xp) return;
    uint4 p[P];
    pieces8<XT>(static_cast<const T*>(x) + n * ldx, k, K, whole, p);
#pragma unroll
    for (int i = 0; i < P; ++i) *reinterpret_cast<uint4*>(parts + (n * P + i) * xp + k) = p[i];
}

struct Plan {
    int nt, r, ways, slab;
    bool staged;
    size_t lds, workspace;
};

Plan plan_for(int dtype, int64_t M, int64_t K, int64_t N) {
    const int parts = dtype == BS_F32 ? 3 : 1, tpt = dtype == BS_F32 ? 4 : 16;
    Plan p;
    p.staged = N <= tpt;
    const int64_t tiles = (M + 15) / 16, chunks = (K + kQ4Chunk - 1) / kQ4Chunk;
    p.nt = p.staged ? 1 : N <= 2 * tpt ? 2 : 4;
    p.r = p.staged ? 1 : 2;
    p.ways = 1;
    while (p.ways < 16 && p.ways * 2 <= chunks && (p.ways * kU < chunks || tiles * p.ways < 2048)) p.ways *= 2;
    if (!p.staged && p.ways > 8) p.ways = 8;      // registers of 512 lanes
    const int rows = p.staged ? (int)N * parts : 0;
    p.slab = 0;
    if (rows) {
        const int64_t most = (int64_t)kSlabBytes / (rows * 2) / kQ4Chunk * kQ4Chunk;
        p.slab = (int)(chunks * kQ4Chunk <= most ? chunks * kQ4Chunk : most);
    }
    const size_t xs = (size_t)rows * (p.slab + 8) * 2, sums = (size_t)p.ways * p.r * p.nt * tpt * 16 * 4;
    p.lds = xs > sums ? xs : sums;
    p.workspace = p.staged ? 0 : (size_t)N * parts * q4_padded(K) * 2;
    return p;
}

template <typename XT, int NT, int R, int GL, bool STAGED>
int launch(const GemvArgs& g, const Plan& p, hipStream_t st) {
    using Reg = LdsKernelOf<q4_gemv_kernel<XT, NT, R, GL, STAGED>>;
    if (p.lds > kLdsWithoutLimit) {
        const int rc = ensure_lds_limit(Reg::reg, st);
        if (rc != BS_OK) return rc;
    }
    const int per = NT * (16 / XT::kSlots);
    const dim3 grid((unsigned)((g.M + 16 * R - 1) / (16 * R)), (unsigned)((g.N + per - 1) / per));
    hipLaunchKernelGGL((q4_gemv_kernel<XT, NT, R, GL, STAGED>), grid, dim3(64 * p.ways), p.lds, st, g);
    return hip_status(hipGetLastError());
}

template <typename XT, int GL>
int launch_tiles(const GemvArgs& g, const Plan& p, hipStream_t st) {
    if (p.staged) return launch<XT, 1, 1, GL, true>(g, p, st);
    return p.nt == 2 ? launch<XT, 2, 2, GL, false>(g, p, st) : launch<XT, 4, 2, GL, false>(g, p, st);
}

template <typename XT>
int launch_type(GemvArgs g, const Plan& p, int group, void* workspace, hipStream_t st) {
    if (!p.staged) {
        const dim3 grid((unsigned)((q4_padded(g.K) + 2047) / 2048), (unsigned)g.N);
        hipLaunchKernelGGL(q4_split_kernel<XT>, grid, dim3(256), 0, st, g.x, g.K, g.ldx, g.whole, static_cast<uint16_t*>(workspace));
        const int rc = hip_status(hipGetLastError());
        if (rc != BS_OK) return rc;
        g.x = workspace;
    }
    switch (q4_group_shift(group)) {
        case 0: return launch_tiles<XT, 0>(g, p, st);
        case 1: return launch_tiles<XT, 1>(g, p, st);
        default: return launch_tiles<XT, 2>(g, p, st);
    }
}

}  // namespace

size_t q4_gemv_workspace_bytes(int dtype, int64_t M, int64_t K, int64_t N) { return plan_for(dtype, M, K, N).workspace; }

int launch_q4_gemv(const uint8_t* codes, const uint16_t* scales, int64_t M, int64_t K, int group, const void* x, int dtype,
                   int64_t N, int64_t ldx, void* y, int64_t ldy, void* workspace, size_t workspace_bytes, hipStream_t st) {
    const Plan p = plan_for(dtype, M, K, N);
    if (p.workspace && (!workspace || workspace_bytes < p.workspace || (reinterpret_cast<uintptr_t>(workspace) & 15)))
        return BS_ERR_WORKSPACE;
    GemvArgs g{codes, scales, M, K, N, ldx, ldy, x, y, p.ways, p.slab, false};
    g.whole = (reinterpret_cast<uintptr_t>(x) & 15) == 0 && (N == 1 || ldx * dtype_bytes(dtype) % 16 == 0);
    switch (dtype) {
        case BS_F32: return launch_type<F32>(g, p, group, workspace, st);
        case BS_F16: return launch_type<F16>(g, p, group, workspace, st);
        default: return launch_type<BF16>(g, p, group, workspace, st);
    }
}

}  // namespace bs

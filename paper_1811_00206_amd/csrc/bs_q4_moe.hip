// A mixture-of-experts layer on 4-bit expert matrices for a few tokens (bs.h: bs_q4_moe), in three kernels:
//
//   route  one workgroup per token: router logits, the top_k largest, their weights; and the token's activations as
//          virtual rows (bs_q4.h), padded with zeros, for the next kernel to read in whole pieces
//   up     one workgroup per 16 hidden units of a chosen expert: gate and up rows against all tokens that chose it,
//          h = silu(g) * u, written as virtual rows of the last kernel
//   down   one workgroup per 16 outputs: its wavefronts share the chosen experts (and K, if the experts are fewer) and
//          add weight * W2 h into sums of their own in LDS, which are added in the order of the wavefronts
//
// Bound: every chosen expert's codes once.  An expert is known by the first (token, choice) pair that chose it; the
// workgroups of the other pairs end at once, so nothing is sorted or counted between the kernels.  No atomics: a result
// has the same bits from every call.  Hidden values pass to `down` in two bfloat16 parts for 16-bit activations (16
// leading bits: their rounding is not seen behind the output's) and in three (all 24 bits) for fp32.
#include "bs_q4.h"

namespace bs {
namespace {

constexpr int kU = 2;
constexpr int kDownWaves = 16;
constexpr int kMaxTokens = BS_MOE_TOKENS_MAX, kMaxExperts = BS_MOE_EXPERTS_MAX, kMaxTopK = BS_MOE_TOP_K_MAX;

// Elements between virtual rows in the workspace: whole chunks and a cache line, so that rows a power of two long do not
// meet in the same sets of the caches.
__host__ __device__ constexpr int64_t row_pitch(int64_t columns) { return q4_padded(columns) + 64; }

template <typename XT>
struct Hidden {      // virtual rows of h
    static constexpr int kParts = XT::kParts == 3 ? 3 : 2, kSlots = XT::kParts == 3 ? 4 : 2;
};

struct MoeArgs {
    const void *x, *router;
    int64_t ldx, ldy;
    int T, D, E, F, top_k, pairs;
    bool renormalise, whole_x, whole_router;
    const uint8_t *w1, *w2;
    const uint16_t *s1, *s2;
    void* y;
    int32_t* ids;
    float* weights;
    uint16_t *xp, *hp;      // [T][parts][D padded], [pairs][hidden parts][F padded]
    int ways;
};

template <typename XT>
__global__ __launch_bounds__(1024) void moe_route_kernel(MoeArgs g) {
    using T = typename XT::type;
    constexpr int P = XT::kParts, EB = 4;
    __shared__ float logits[kMaxExperts];
    const int t = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const T* x = static_cast<const T*>(g.x) + t * g.ldx;
    const int64_t columns = q4_padded(g.D), dp = row_pitch(g.D);
    for (int e = wave * EB; e < g.E; e += waves * EB) {
        float sum[EB] = {};
        for (int k = 8 * lane; k < g.D; k += 512) {
            float a[8], w[8];
            load8<XT>(x, k, g.D, g.whole_x, a);
#pragma unroll
            for (int i = 0; i < EB; ++i) {
                const T* row = static_cast<const T*>(g.router) + (int64_t)min(e + i, g.E - 1) * g.D;
                load8<XT>(row, k, g.D, g.whole_router, w);
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[i] = fmaf(a[j], w[j], sum[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < EB; ++i) {
            const float s = group_sum<64>(sum[i]);
            if (lane == 0 && e + i < g.E) logits[e + i] = s;
        }
    }
    for (int64_t k = 8 * threadIdx.x; k < columns; k += 8 * blockDim.x) {
        uint4 p[P];
        pieces8<XT>(x, k, g.D, g.whole_x, p);
#pragma unroll
        for (int i = 0; i < P; ++i) *reinterpret_cast<uint4*>(g.xp + ((int64_t)t * P + i) * dp + k) = p[i];
    }
    __syncthreads();
    if (wave) return;
    float top = 0.f, mine = 0.f, all = 0.f, chosen = 0.f;      // lane j < top_k: its choice's exp(logit - top)
    int32_t id = 0;
    uint64_t last = ~(uint64_t)0;                              // the choice before: every key below it is still free
    for (int j = 0; j < g.top_k; ++j) {
        uint64_t best = 0;
        for (int e = lane; e < g.E; e += 64) {
            const uint64_t key = order_key(logits[e], e);
            if (key < last && key > best) best = key;
        }
        best = wave_max(best);
        last = best;
        const int e = (int)index_of_key(best);
        const float l = logits[e];
        if (j == 0) top = l;
        const float w = expf(l - top);
        chosen += w;
        if (lane == j) { mine = w; id = e; }
    }
    if (!g.renormalise) {
        for (int e = lane; e < g.E; e += 64) all += expf(logits[e] - top);
        all = group_sum<64>(all);
    }
    if (lane < g.top_k) {
        g.ids[t * g.top_k + lane] = id;
        g.weights[t * g.top_k + lane] = mine / (g.renormalise ? chosen : all);
    }
}

// the pairs at or behind `first` that chose expert e, in order, by one wavefront; their number
__device__ __forceinline__ int pairs_of(const int32_t* ids, int pairs, int first, int e, int32_t* list) {
    const int lane = threadIdx.x & 63;
    int n = 0;
    for (int b = first & ~63; b < pairs; b += 64) {
        const int p = b + lane;
        const bool hit = p >= first && p < pairs && ids[p] == e;
        const uint64_t m = __ballot(hit);
        if (hit) list[n + lanes_below(m)] = p;
        n += __popcll(m);
    }
    return n;
}

template <typename XT, int NT, int GL>
__global__ __launch_bounds__(512) void moe_up_kernel(MoeArgs g) {
    constexpr int P = XT::kParts, S = XT::kSlots, TPT = 16 / S, HP = Hidden<XT>::kParts;
    extern __shared__ __align__(16) uint8_t lds[];
    float* sums = reinterpret_cast<float*>(lds);        // [wave][gate, up][NT][TPT][16]
    __shared__ int32_t list[kMaxTokens];
    __shared__ int found;
    const int lane = threadIdx.x & 63, kb = lane >> 4, r = lane & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int pair = blockIdx.y, f0 = 16 * blockIdx.x;
    const int e = g.ids[pair];
    int earlier = 0;
    for (int p = threadIdx.x; p < pair; p += blockDim.x) earlier |= g.ids[p] == e;
    if (__syncthreads_or(earlier)) return;
    if (wave == 0) {
        const int n = pairs_of(g.ids, g.pairs, pair, e, list);
        if (lane == 0) found = n;
    }
    __syncthreads();
    const int tokens = found;
    const int64_t fp = row_pitch(g.F), dp = row_pitch(g.D);
    const int chunks = (int)(q4_padded(g.D) / kQ4Chunk);
    const int64_t pitch = q4_row_bytes(g.D), groups = (g.D + (32 << GL) - 1) >> (5 + GL);
    constexpr int V = 4 / S, kOut = NT * TPT * 16;
    for (int n0 = 0; n0 < tokens; n0 += NT * TPT) {
        const int here = min(tokens - n0, NT * TPT);
        if (f0 < g.F) {
            Q4Walk<XT::kHalf, NT, 2, GL, kU> walk;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int64_t first = ((int64_t)e * 2 + i) * g.F;      // of the expert's gate or up rows
                walk.tile(i, g.w1 + first * pitch, g.s1 + first * groups, f0, g.F, g.D, lane);
            }
            RowsOfX<NT, kU> x;
            x.kb = kb;
            x.columns = chunks * kQ4Chunk;
            x.last = chunks - 1;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int token = list[n0 + min(t * TPT + r / S, here - 1)] / g.top_k;
                x.at[t] = g.xp + ((int64_t)token * P + min(r % S, P - 1)) * dp;
            }
            f32x4 acc[2][NT] = {};
            walk.template walk<kU>(wave, g.ways, chunks, x, acc);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        float sum = acc[i][t][v];
                        if constexpr (S == 4) sum = acc[i][t][0] + (acc[i][t][1] + acc[i][t][2]);
                        sums[((wave * 2 + i) * NT * TPT + t * TPT + kb * V + v) * 16 + r] = sum;
                    }
        }
        __syncthreads();
        for (int o = threadIdx.x; o < here * 16; o += blockDim.x) {
            const int f = f0 + o % 16;
            float h = 0.f;      // behind F: zeros up to whole chunks
            if (f < g.F) {
                float gate = sums[o], up = sums[kOut + o];
                for (int w = 1; w < g.ways; ++w) { gate += sums[2 * w * kOut + o]; up += sums[(2 * w + 1) * kOut + o]; }
                h = gate / (1.f + expf(-gate)) * up;
            }
            uint32_t part[3];
            split3(h, part[0], part[1], part[2]);
            if constexpr (HP == 2) {      // the second part rounded
                const float rest = __builtin_bit_cast(float, part[1]) + __builtin_bit_cast(float, part[2]);
                part[1] = (uint32_t)BF16::store(rest) << 16;
            }
            uint16_t* to = g.hp + (int64_t)list[n0 + o / 16] * HP * fp + f;
#pragma unroll
            for (int i = 0; i < HP; ++i) to[i * fp] = (uint16_t)(part[i] >> 16);
        }
        __syncthreads();
    }
}

template <typename XT, int GL>
__global__ __launch_bounds__(1024) void moe_down_kernel(MoeArgs g) {
    constexpr int P = Hidden<XT>::kParts, S = Hidden<XT>::kSlots, TPT = 16 / S, V = 4 / S;
    extern __shared__ __align__(16) uint8_t lds[];
    float* sums = reinterpret_cast<float*>(lds);                                     // [wave][T][16]
    int32_t* ids = reinterpret_cast<int32_t*>(sums + kDownWaves * g.T * 16);         // [pairs]
    int32_t* leaders = ids + g.pairs;                                                // [pairs]
    int32_t* first_of = leaders + g.pairs;                                           // [E]
    int32_t* lists = first_of + g.E;                                                 // [wave][T]
    int32_t* found = lists + kDownWaves * g.T;
    const int lane = threadIdx.x & 63, kb = lane >> 4, r = lane & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int d0 = 16 * blockIdx.x;
    for (int p = threadIdx.x; p < g.pairs; p += blockDim.x) ids[p] = g.ids[p];
    for (int i = threadIdx.x; i < kDownWaves * g.T * 16; i += blockDim.x) sums[i] = 0.f;
    for (int i = threadIdx.x; i < g.E; i += blockDim.x) first_of[i] = g.pairs;
    __syncthreads();
    for (int p = threadIdx.x; p < g.pairs; p += blockDim.x) atomicMin(first_of + ids[p], p);
    __syncthreads();
    if (wave == 0) {      // the first pair of every chosen expert
        int n = 0;
        for (int b = 0; b < g.pairs; b += 64) {
            const int p = b + lane;
            const bool first = p < g.pairs && first_of[ids[p]] == p;
            const uint64_t m = __ballot(first);
            if (first) leaders[n + lanes_below(m)] = p;
            n += __popcll(m);
        }
        if (lane == 0) *found = n;
    }
    __syncthreads();
    const int experts = __builtin_amdgcn_readfirstlane(*found);
    const int64_t fp = row_pitch(g.F);
    const int chunks = (int)(q4_padded(g.F) / kQ4Chunk);
    const int64_t pitch = q4_row_bytes(g.F), groups = (g.F + (32 << GL) - 1) >> (5 + GL);
    const int ways = experts >= kDownWaves ? 1 : min(kDownWaves / experts, (chunks + kU - 1) / kU);
    float* mine = sums + wave * g.T * 16;
    int32_t* list = lists + wave * g.T;
    for (int item = wave; item < experts * ways; item += kDownWaves) {
        const int first = __builtin_amdgcn_readfirstlane(leaders[item / ways]), c0 = item % ways;
        const int e = __builtin_amdgcn_readfirstlane(ids[first]);
        const int tokens = pairs_of(ids, g.pairs, first, e, list);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // the list is written by some lanes and read by others
        Q4Walk<false, 1, 1, GL, kU> walk;
        walk.tile(0, g.w2 + (int64_t)e * g.D * pitch, g.s2 + (int64_t)e * g.D * groups, d0, g.D, g.F, lane);
        for (int n0 = 0; n0 < tokens; n0 += TPT) {
            const int here = min(tokens - n0, TPT);
            RowsOfX<1, kU> x;
            x.kb = kb;
            x.columns = chunks * kQ4Chunk;
            x.last = chunks - 1;
            x.at[0] = g.hp + ((int64_t)list[n0 + min(r / S, here - 1)] * P + min(r % S, P - 1)) * fp;
            f32x4 acc[1][1] = {};
            walk.template walk<kU>(c0, ways, chunks, x, acc);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int n = kb * V + v;
                if (n >= here) continue;
                const int pair = list[n0 + n];
                float sum;
                if constexpr (S == 4) sum = acc[0][0][0] + (acc[0][0][1] + acc[0][0][2]);
                else sum = acc[0][0][2 * v] + acc[0][0][2 * v + 1];
                float* to = mine + pair / g.top_k * 16 + r;
                *to = fmaf(g.weights[pair], sum, *to);
            }
        }
    }
    __syncthreads();
    for (int o = threadIdx.x; o < g.T * 16; o += blockDim.x) {
        const int t = o / 16, d = d0 + o % 16;
        if (d >= g.D) continue;
        float sum = sums[o];
        for (int w = 1; w < kDownWaves; ++w) sum += sums[w * g.T * 16 + o];
        static_cast<typename XT::type*>(g.y)[t * g.ldy + d] = XT::store(sum);
    }
}

// all of it dynamic: the kernel's limit is raised to all that a compute unit has
size_t down_lds(const MoeArgs& g) { return (size_t)kDownWaves * g.T * 68 + (size_t)g.pairs * 8 + (size_t)g.E * 4 + 4; }

template <typename XT, int GL>
int launch(const MoeArgs& g, hipStream_t st) {
    constexpr int TPT = 16 / XT::kSlots;
    using Down = LdsKernelOf<moe_down_kernel<XT, GL>>;
    const size_t lds = down_lds(g);
    if (lds > kLdsWithoutLimit) {
        const int rc = ensure_lds_limit(Down::reg, st);
        if (rc != BS_OK) return rc;
    }
    const int route_waves = g.E > 32 ? 16 : g.E > 16 ? 8 : 4;
    hipLaunchKernelGGL(moe_route_kernel<XT>, dim3(g.T), dim3(64 * route_waves), 0, st, g);
    int rc = hip_status(hipGetLastError());
    if (rc != BS_OK) return rc;
    const dim3 up((unsigned)(q4_padded(g.F) / 16), (unsigned)g.pairs);
    const auto sums = [&](int nt) { return (size_t)g.ways * 2 * nt * TPT * 16 * 4; };
    if (g.T <= TPT) hipLaunchKernelGGL((moe_up_kernel<XT, 1, GL>), up, dim3(64 * g.ways), sums(1), st, g);
    else hipLaunchKernelGGL((moe_up_kernel<XT, 2, GL>), up, dim3(64 * g.ways), sums(2), st, g);
    rc = hip_status(hipGetLastError());
    if (rc != BS_OK) return rc;
    hipLaunchKernelGGL((moe_down_kernel<XT, GL>), dim3((unsigned)((g.D + 15) / 16)), dim3(64 * kDownWaves), lds, st, g);
    return hip_status(hipGetLastError());
}

template <typename XT>
int launch_group(const MoeArgs& g, int group, hipStream_t st) {
    switch (q4_group_shift(group)) {
        case 0: return launch<XT, 0>(g, st);
        case 1: return launch<XT, 1>(g, st);
        default: return launch<XT, 2>(g, st);
    }
}

size_t x_bytes(int dtype, int64_t T, int64_t D) { return (size_t)T * (dtype == BS_F32 ? 3 : 1) * row_pitch(D) * 2; }

}  // namespace

size_t q4_moe_workspace_bytes(int dtype, int64_t T, int64_t D, int64_t F, int top_k) {
    return x_bytes(dtype, T, D) + (size_t)T * top_k * (dtype == BS_F32 ? 3 : 2) * row_pitch(F) * 2;
}

int launch_q4_moe(const void* x, int dtype, int64_t T, int64_t ldx, int64_t D, const void* router, int E, const uint8_t* w1,
                  const uint16_t* s1, const uint8_t* w2, const uint16_t* s2, int64_t F, int group, int top_k, int renormalise, void* y,
                  int64_t ldy, int32_t* ids, float* weights, void* workspace, size_t workspace_bytes, hipStream_t st) {
    if (!workspace || workspace_bytes < q4_moe_workspace_bytes(dtype, T, D, F, top_k) || (reinterpret_cast<uintptr_t>(workspace) & 15))
        return BS_ERR_WORKSPACE;
    MoeArgs g{};
    g.x = x; g.router = router; g.ldx = ldx; g.ldy = ldy;
    g.T = (int)T; g.D = (int)D; g.E = E; g.F = (int)F; g.top_k = top_k; g.pairs = (int)T * top_k;
    g.renormalise = renormalise != 0;
    const int size = dtype_bytes(dtype);
    g.whole_x = (reinterpret_cast<uintptr_t>(x) & 15) == 0 && (T == 1 || ldx * size % 16 == 0);
    g.whole_router = (reinterpret_cast<uintptr_t>(router) & 15) == 0 && D * size % 16 == 0;
    g.w1 = w1; g.w2 = w2; g.s1 = s1; g.s2 = s2; g.y = y; g.ids = ids; g.weights = weights;
    g.xp = static_cast<uint16_t*>(workspace);
    g.hp = g.xp + x_bytes(dtype, T, D) / 2;
    const int64_t steps = (q4_padded(D) / kQ4Chunk + kU - 1) / kU;
    g.ways = (int)(steps < 8 ? steps : 8);
    switch (dtype) {
        case BS_F32: return launch_group<F32>(g, group, st);
        case BS_F16: return launch_group<F16>(g, group, st);
        default: return launch_group<BF16>(g, group, st);
    }
}

}  // namespace bs

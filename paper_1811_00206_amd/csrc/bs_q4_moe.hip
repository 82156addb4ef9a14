// A mixture-of-experts layer on 4-bit expert matrices for a few tokens (bs.h: bs_q4_moe), 64 at a time, in two to four kernels:
//
//   logits  a wavefront per token and expert: router logits; and the token's activations as virtual rows (bs_q4.h),
//           padded with zeros, for `up` to read in whole pieces
//   route   one workgroup: every token's top_k experts and their weights, and the pairs (token, choice) expert by expert
//   up      some tiles of 16 hidden units of a chosen expert: gate and up rows against all tokens that chose it,
//           h = silu(g) * u, written as virtual rows of the last kernel
//   down    16 outputs a tile: the wavefronts of one or a few workgroups share steps of chosen experts and add weight * W2 h
//           into sums of their own in LDS, which are added in the order of the wavefronts; of several workgroups the one that
//           is done last adds their sums, in their order
//
// Bound: every chosen expert's codes once.  What it takes above that is latency, four kernels that wait for one another, and
// the beginning and end of the workgroups of `up` and `down`.  For up to three tokens every workgroup of `up` finds its expert by
// itself, without `route` (which is 3 to 5 us; 7 tokens, 64 experts of 2048 x 1024, 6 each: 41.9 us with it, 47.6 without;
// 2 tokens, 32 experts of 1004 x 415, 8 each: kernels of 26.9 with it, 22.4 without), and where the logits are few they are made
// there too.  The order of all sums is fixed: a result has the same bits from every call.  Hidden values pass to `down` in three
// bfloat16 parts, all 24 bits, for 16-bit activations too: in two parts, 16 bits, their rounding was seen where the sum over F
// cancels.
//
// Measured: 7 tokens of 2048 x 1024 in bfloat16, 6 of 64 experts each: 40 to 42 us a call (logits 4, route 3.8, up 18 to 22 as 32 or
// more experts are chosen, down 14.8; 18.4 at the rate of reads).  16 tokens, 8 each: up 32, down 32.  One token of 1500 x 1500 in
// fp32, 2 of 8: 15.2 us, up 9.5, down 4.9.  More than 64 tokens pay for each 64 anew: 256 of those 64 experts, 6 each, 430 us.
#include "bs_q4.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace bs {
namespace {

constexpr int kDownWaves = 8;
// x (twice that, if need be) and h are brought to LDS where they take no more: h of 44 pairs and 256 columns, of which a compute unit holds
// two workgroups (7 tokens, 6 experts each: 43.9 us a call, 48.9 with h from memory)
constexpr size_t kLdsOfX = 32 * 1024, kLdsOfH = 68 * 1024;
constexpr int kTokens = 64;      // that pass together; more pass 64 by 64

// Elements between virtual rows in the workspace: whole chunks and a cache line, so that rows a power of two long do not
// meet in the same sets of the caches.
__host__ __device__ constexpr int64_t row_pitch(int64_t columns) { return q4_padded(columns) + 64; }

constexpr int kHiddenParts = 3, kHiddenSlots = 4;      // virtual rows of h, and those set aside for a token, as for fp32 activations

struct MoeArgs {
    const void *x, *router;
    int64_t ldx, ldy;
    int T, D, E, F, top_k, pairs;
    bool renormalise;
    const uint8_t *w1, *w2;
    const uint16_t *s1, *s2;
    void* y;
    int32_t* ids;
    float* weights;
    uint16_t *xp, *hp;      // [T][parts][D padded], [pairs][hidden parts][F padded]
    float* logits;          // [T][E]
    float* parts;           // [down workgroups of a tile][D padded to tiles][T], if there are several
    uint32_t* done;         // [tile]: those of them that are done
    int4* groups;           // x of the first: number of chosen experts; then of each: expert, first place in `order`, pairs
    int32_t* order;         // [pairs]: the pairs, expert by expert
    bool routed;            // groups are known before `up`
    uint32_t magic_x, magic_h;   // of the pieces of a row in LDS
    int split, part_chunks;      // workgroups of a tile in `down`, and the chunks of F of each
    int ways, tiles, rows;       // rows: tokens whose sums a wavefront of `up` keeps
};

// one wavefront: a router row times a token's activations
template <typename XT>
__device__ __forceinline__ void router_row(const MoeArgs& g, const typename XT::type* x, int e, float* logit) {
    const int lane = threadIdx.x & 63;
    const typename XT::type* row = static_cast<const typename XT::type*>(g.router) + (int64_t)e * g.D;
    float sum = 0.f;
#pragma unroll 4
    for (int k0 = 0; k0 < g.D; k0 += 512) {
        float a[8], w[8];
        load8<XT>(x, k0 + 8 * lane, g.D, a);
        load8<XT>(row, k0 + 8 * lane, g.D, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = fmaf(a[j], w[j], sum);
    }
    sum = sum_of_wave(sum);
    if (lane == 0) *logit = sum;
}

// Of up to 64 experts, a lane's each, the next choice among the free ones, by one wavefront: the largest logit, and of lanes that have it
// the first.  A logit that is no number comes last, behind -inf too: `own` is -inf there, and the lane is not in `numbers`.
__device__ __forceinline__ int next_choice(float own, uint64_t numbers, uint64_t free, float& most) {
    most = max_of_wave(free >> (threadIdx.x & 63) & 1 ? own : -__builtin_inff());
    const uint64_t m = __ballot(own == most) & free, n = m & numbers;
    return __ffsll((unsigned long long)(n ? n : m)) - 1;
}

// One wavefront: a token's top_k experts and their weights.
__device__ __forceinline__ void choose(const MoeArgs& g, const float* logits, int32_t* ids, float* weights) {
    const int lane = threadIdx.x & 63;
    if (g.E <= 64) {
        float l = lane < g.E ? logits[lane] : 0.f;
        const bool nan = l != l;
        const float own = nan ? -__builtin_inff() : l;
        const uint64_t numbers = __ballot(!nan);
        uint64_t free = g.E == 64 ? ~(uint64_t)0 : ((uint64_t)1 << g.E) - 1;
        int rank = -1;
        float top = 0.f;
        for (int j = 0; j < g.top_k; ++j) {
            float most;
            const int first = next_choice(own, numbers, free, most);
            if (lane == first) rank = j;
            free &= ~((uint64_t)1 << first);
            if (j == 0) top = most;
        }
        const float w = nan ? l : expf(own - top);
        const float sum = sum_of_wave(lane < g.E && (!g.renormalise || rank >= 0) ? w : 0.f);
        if (rank >= 0) {
            ids[rank] = lane;
            weights[rank] = w / sum;
        }
        return;
    }
    float top = 0.f, mine = 0.f, all = 0.f, chosen = 0.f;      // lane j < top_k: its choice's exp(logit - top)
    int32_t id = 0;
    uint64_t last = ~(uint64_t)0;                              // the choice before: every key below it is still free
    for (int j = 0; j < g.top_k; ++j) {
        uint64_t best = 0;
        for (int e = lane; e < g.E; e += 64) {
            const uint64_t key = order_key(logits[e], e);
            if (key < last && key > best) best = key;
        }
        last = wave_max(best);
        const float l = value_of_key(last);
        if (j == 0) top = l;
        const float w = expf(l - top);
        chosen += w;
        if (lane == j) { mine = w; id = (int32_t)index_of_key(last); }
    }
    if (!g.renormalise) {
        for (int e = lane; e < g.E; e += 64) all += expf(logits[e] - top);
        all = sum_of_wave(all);
    }
    if (lane < g.top_k) {
        ids[lane] = id;
        weights[lane] = mine / (g.renormalise ? chosen : all);
    }
}

// How many experts are chosen before expert e, whose logit is le, by one wavefront: what choose() goes by.
__device__ __forceinline__ int experts_before(const MoeArgs& g, const float* logits, int e, float le) {
    const int lane = threadIdx.x & 63;
    if (g.E <= 64) {
        const float l = lane < g.E ? logits[lane] : 0.f;
        const bool nan = l != l, other_nan = le != le;
        const float own = nan ? -__builtin_inff() : l, other = other_nan ? -__builtin_inff() : le;
        return __popcll(__ballot(lane < g.E && (own > other || (own == other && (nan == other_nan ? lane < e : other_nan)))));
    }
    const uint64_t key = order_key(le, e);
    int n = 0;
    for (int i = lane; i < (g.E + 63) / 64 * 64; i += 64) n += __popcll(__ballot(i < g.E && order_key(logits[min(i, g.E - 1)], i) > key));
    return n;
}

// Choice j of a token, by one wavefront
__device__ __forceinline__ int expert_of(const MoeArgs& g, const float* logits, int j) {
    const int lane = threadIdx.x & 63;
    if (g.E <= 64) {
        const float l = lane < g.E ? logits[lane] : 0.f;
        const float own = l != l ? -__builtin_inff() : l;
        const uint64_t numbers = __ballot(l == l);
        uint64_t free = g.E == 64 ? ~(uint64_t)0 : ((uint64_t)1 << g.E) - 1;
        for (;;) {
            float most;
            const int first = next_choice(own, numbers, free, most);
            if (j-- == 0) return __builtin_amdgcn_readfirstlane(first);
            free &= ~((uint64_t)1 << first);
        }
    }
    uint64_t last = ~(uint64_t)0;
    for (; j >= 0; --j) {
        uint64_t best = 0;
        for (int e = lane; e < g.E; e += 64) {
            const uint64_t key = order_key(logits[e], e);
            if (key < last && key > best) best = key;
        }
        last = wave_max(best);
    }
    return __builtin_amdgcn_readfirstlane((int)index_of_key(last));
}

// blockIdx: token, four experts, a wavefront's each; and the first workgroup of a token has its virtual rows.  (Four experts a
// wavefront read less of x and are slower: 7 tokens, 64 experts of 2048 columns 6.6 us instead of 4.8, 64 tokens of 1024 experts of
// 512 19.4 instead of 16.)
template <typename XT>
__global__ __launch_bounds__(256) void moe_logits_kernel(MoeArgs g) {
    constexpr int P = XT::kParts;
    const int t = blockIdx.x, e = blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const typename XT::type* x = static_cast<const typename XT::type*>(g.x) + t * g.ldx;
    if (e < g.E) router_row<XT>(g, x, e, g.logits + t * g.E + e);
    if (blockIdx.y) return;
    const int64_t columns = q4_padded(g.D), dp = row_pitch(g.D);
    for (int64_t k = 8 * threadIdx.x; k < columns; k += 8 * 256) {
        uint4 p[P];
        pieces8<XT>(x, k, g.D, p);
#pragma unroll
        for (int i = 0; i < P; ++i) *reinterpret_cast<uint4*>(g.xp + ((int64_t)t * P + i) * dp + k) = p[i];
    }
}

// `rows` rows of `pieces` 16-byte pieces to LDS, `have` of which there are; from(row): where one is
template <typename From>
__device__ __forceinline__ void rows_to_lds(uint16_t* to, int to_pitch, From&& from, int rows, int pieces, uint32_t magic, int have) {
    const int all = rows * pieces, stride = blockDim.x;
    const auto load = [&](int j, int& at) {      // (what is not there is read as what is, and not stored)
        const int row = (int)div_magic_any(min(j, all - 1), pieces, magic), k = min(j, all - 1) - row * pieces;
        at = j < all && k < have ? row * to_pitch + 8 * k : -1;
        return *reinterpret_cast<const uint4*>(from(row) + 8 * min(k, have - 1));
    };
    for (int j = threadIdx.x; j < all; j += 4 * stride) {      // four on their way together
        int a0, a1, a2, a3;
        const uint4 v0 = load(j, a0), v1 = load(j + stride, a1), v2 = load(j + 2 * stride, a2), v3 = load(j + 3 * stride, a3);
        if (a0 >= 0) *reinterpret_cast<uint4*>(to + a0) = v0;
        if (a1 >= 0) *reinterpret_cast<uint4*>(to + a1) = v1;
        if (a2 >= 0) *reinterpret_cast<uint4*>(to + a2) = v2;
        if (a3 >= 0) *reinterpret_cast<uint4*>(to + a3) = v3;
    }
}

// All threads of a workgroup: every token's choices and what follows from them, written for the other kernels and the caller.
// LDS: for every expert the tokens that chose it, as bits, [E]; its place in `order`, [E]; [pairs] ids, [pairs] weights.
__device__ __forceinline__ void route(const MoeArgs& g, const float* logits, uint8_t* lds) {
    static_assert(kTokens == 64);
    unsigned long long* chose = reinterpret_cast<unsigned long long*>(lds);
    int32_t* place = reinterpret_cast<int32_t*>(chose + g.E);
    int32_t* ids = place + g.E;
    float* weights = reinterpret_cast<float*>(ids + g.pairs);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    for (int t = wave; t < g.T; t += waves) choose(g, logits + t * g.E, ids + t * g.top_k, weights + t * g.top_k);
    for (int i = threadIdx.x; i < g.E; i += blockDim.x) chose[i] = 0;
    if (g.split > 1)
        for (int i = threadIdx.x; i < (g.D + 15) / 16; i += blockDim.x) g.done[i] = 0;
    __syncthreads();
    for (int p = threadIdx.x; p < g.pairs; p += blockDim.x) {
        g.ids[p] = ids[p];
        g.weights[p] = weights[p];
        atomicOr(chose + ids[p], 1ull << (p / g.top_k));
    }
    __syncthreads();
    const auto earlier = [&](int p, uint64_t m) { return __popcll(m & ((1ull << (p / g.top_k)) - 1)); };
    if (wave == 0) {      // experts in the order of their first pairs
        int n = 0, places = 0;
        for (int b = 0; b < g.pairs; b += 64) {
            const int p = b + lane, e = ids[min(p, g.pairs - 1)];
            const uint64_t of = chose[e];
            const bool leads = p < g.pairs && earlier(p, of) == 0;
            const int count = leads ? __popcll(of) : 0, before = group_prefix_i<64>(count, lane);
            const uint64_t m = __ballot(leads);
            if (leads) {
                g.groups[1 + n + lanes_below(m)] = int4{e, places + before, count, 0};
                place[e] = places + before;
            }
            n += __popcll(m);
            places += __builtin_amdgcn_readlane(before + count, 63);
        }
        if (lane == 0) g.groups[0] = int4{n, 0, 0, 0};
    }
    __syncthreads();
    for (int p = threadIdx.x; p < g.pairs; p += blockDim.x) g.order[place[ids[p]] + earlier(p, chose[ids[p]])] = p;
}

__host__ __device__ constexpr int route_bytes(int pairs, int E) { return (pairs * 8 + E * 12 + 15) / 16 * 16; }

// One workgroup: the choices, where there are many workgroups of `up` that would each have to find its expert
__global__ __launch_bounds__(1024) void moe_route_kernel(MoeArgs g) {
    extern __shared__ __align__(16) uint8_t lds[];
    route(g, g.logits, lds);
}

// LDS of `down` before h.  (All LDS here is dynamic: the kernels' limits are raised to all that a compute unit has.)
__host__ __device__ constexpr int down_small(int T, int pairs) { return (kDownWaves * T * 64 + pairs * 28 + 4 + 15) / 16 * 16; }
// LDS of `up` before its sums
__host__ __device__ constexpr int up_small(int T, int pairs, int E, bool alone) {
    return route_bytes(pairs, E) + (T * 4 + (alone ? T * E * 4 : 0) + 15) / 16 * 16;
}

// 16 * tiles hidden units of a chosen expert.  Half of the wavefronts have the gate rows, half the up rows; each half shares
// D, and a wavefront walks its columns of one tile after the other, the next one's codes on their way.  IN_LDS: the tokens' x
// is brought to LDS, else read from memory.  ALONE: without the kernel of the logits, they are made here, by every workgroup.
template <typename XT, int NT, int GL, bool IN_LDS, bool ALONE>
__global__ __launch_bounds__(512) void moe_up_kernel(MoeArgs g) {
    constexpr int P = XT::kParts, S = XT::kSlots, TPT = 16 / S, HP = kHiddenParts, U = IN_LDS ? 4 : 2;
    extern __shared__ __align__(16) uint8_t lds[];
    int32_t* list = reinterpret_cast<int32_t*>(lds + route_bytes(g.pairs, g.E));                   // [T]
    float* sums = reinterpret_cast<float*>(lds + up_small(g.T, g.pairs, g.E, ALONE));      // [way][gate, up][tile][rows][16]
    uint16_t* xs = reinterpret_cast<uint16_t*>(sums + 2 * g.ways * g.tiles * g.rows * 16);         // [rows * parts][D padded + 8]
    const int lane = threadIdx.x & 63, kb = lane >> 4, r = lane & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int f0 = 16 * g.tiles * blockIdx.x, half = wave & 1, way = wave >> 1;
    const int64_t fp = row_pitch(g.F), dp = row_pitch(g.D);
    const int chunks = (int)(q4_padded(g.D) / kQ4Chunk);
    const int xp = chunks * kQ4Chunk + 8;
    const float* logits = g.logits;
    if constexpr (ALONE) {
        float* made = reinterpret_cast<float*>(list + g.T);      // [T][E]
        logits = made;
        for (int i = wave; i < g.T * g.E; i += 2 * g.ways)
            router_row<XT>(g, static_cast<const typename XT::type*>(g.x) + i / g.E * g.ldx, i % g.E, made + i);
        for (int t = 0; t < g.T; ++t)
            for (int j = threadIdx.x; j < chunks * (kQ4Chunk / 8); j += blockDim.x) {
                uint4 p[P];
                pieces8<XT>(static_cast<const typename XT::type*>(g.x) + t * g.ldx, 8 * j, g.D, p);
#pragma unroll
                for (int i = 0; i < P; ++i) *reinterpret_cast<uint4*>(xs + (t * P + i) * xp + 8 * j) = p[i];
            }
        __syncthreads();
    }
    // Every wavefront for itself (all write the same list): an expert, and the pairs that chose it
    int e, tokens = 0;
    if (!ALONE && g.routed) {
        const int4 group = g.groups[1 + blockIdx.y];      // (behind the last one: of an earlier call or none, and not looked at)
        if ((int)blockIdx.y >= g.groups[0].x) return;
        e = __builtin_amdgcn_readfirstlane(group.x);
        tokens = __builtin_amdgcn_readfirstlane(group.z);
        for (int i = lane; i < tokens; i += 64) list[i] = g.order[group.y + i];
    } else {
        // that of pair blockIdx.y; if one of the pairs comes before it, its workgroups have the expert
        const int pair = blockIdx.y, token = pair / g.top_k;
        e = expert_of(g, logits + token * g.E, pair - token * g.top_k);
#pragma unroll 4
        for (int t = 0; t < g.T; ++t) {
            const int before = experts_before(g, logits + t * g.E, e, logits[t * g.E + e]);
            if (before >= g.top_k) continue;
            if (t < token) return;
            if (lane == 0) list[tokens] = t * g.top_k + before;
            ++tokens;
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int64_t pitch = q4_row_bytes(g.D), groups = (g.D + (32 << GL) - 1) >> (5 + GL);
    const int64_t first = ((int64_t)e * 2 + half) * g.F;      // of the expert's gate or up rows
    Q4Walk<XT::kHalf, NT, 1, GL, U> walk;
    const auto start = [&](int tile) {
        walk.tile(0, g.w1 + first * pitch, g.s1 + first * groups, f0 + 16 * tile, g.F, g.D, lane);
        walk.load(way * U);
    };
    start(0);
    constexpr int V = 4 / S;
    const int out = g.tiles * g.rows * 16;      // sums of a wavefront
    for (int n0 = 0; n0 < tokens; n0 += g.rows) {
        const int here = min(tokens - n0, g.rows);
        if constexpr (IN_LDS && !ALONE) {      // x of the tokens while the first codes are on their way
            const auto from = [&](int row) {
                const int n = row / P;
                return g.xp + ((int64_t)(list[n0 + n] / g.top_k) * P + (row - n * P)) * dp;
            };
            rows_to_lds(xs, xp, from, here * P, chunks * (kQ4Chunk / 8), g.magic_x, chunks * (kQ4Chunk / 8));
            __syncthreads();
        }
        std::conditional_t<IN_LDS, LdsRowsOfX<NT>, RowsOfX<NT, U, false>> x;
        if constexpr (IN_LDS) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {      // rows without a token repeat the last one
                const int n = min(t * TPT + r / S, here - 1);
                x.at[t] = xs + ((ALONE ? list[n0 + n] / g.top_k : n) * P + min(r % S, P - 1)) * xp + 8 * kb;
            }
        } else {
            x.kb = kb;
            x.columns = chunks * kQ4Chunk;
            x.last = chunks - 1;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int n = t * TPT + r / S;
                const bool row = n < here && r % S < P;
                x.at[t] = row ? g.xp + ((int64_t)(list[n0 + n] / g.top_k) * P + r % S) * dp : nullptr;
            }
        }
        if (n0) start(0);
        for (int tile = 0; tile < g.tiles; ++tile) {
            f32x4 acc[1][NT] = {};
            for (int c = way * U; c < chunks;) {
                const int now = c;
                walk.take();
                c += g.ways * U;
#pragma unroll
                for (int u = 0; u < U; ++u) x.fetch(now, u);
                if (c < chunks) walk.load(c);
                else if (tile + 1 < g.tiles) start(tile + 1);
                uint32_t sc[1][decltype(walk)::kWords][4];
                walk.spread(sc);
                walk.template eat<0, U>(now, chunks, x, sc, acc);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const f32x4& a = acc[0][t];
                    float sum = a[v];
                    if constexpr (S == 4) sum = a[0] + (a[1] + a[2]);
                    const int n = t * TPT + kb * V + v;
                    if (n < here) sums[wave * out + (tile * g.rows + n) * 16 + r] = sum;
                }
        }
        __syncthreads();
        for (int o = threadIdx.x; o < g.tiles * here * 16; o += blockDim.x) {
            const int tile = o / (here * 16), n = o / 16 % here, f = f0 + 16 * tile + o % 16;
            if (f >= fp) continue;
            float h = 0.f;      // behind F: zeros up to whole chunks
            if (f < g.F) {
                const float* from = sums + (tile * g.rows + n) * 16 + o % 16;
                float gate = from[0], up = from[out];
                for (int w = 1; w < g.ways; ++w) { gate += from[2 * w * out]; up += from[(2 * w + 1) * out]; }
                gate *= kQ4Unit<XT::kHalf>;
                up *= kQ4Unit<XT::kHalf>;
                h = gate / (1.f + expf(-gate)) * up;
            }
            uint32_t part[HP];
            split3(h, part[0], part[1], part[2]);
            uint16_t* to = g.hp + (int64_t)list[n0 + n] * HP * fp + f;
#pragma unroll
            for (int i = 0; i < HP; ++i) to[i * fp] = (uint16_t)(part[i] >> 16);
        }
        __syncthreads();
    }
    if (blockIdx.x || blockIdx.y || (!ALONE && g.routed)) return;
    route(g, logits, lds);      // the first workgroup says what was chosen
}

// Workgroup z of a tile has a part of F, two chunks at least; a wavefront's work is one step of one chosen expert after the
// other: (expert, two chunks).  While a step is multiplied the codes of its next one, of whatever expert, are on their way.
// IN_LDS: the part's h of all pairs is brought to LDS, else read from memory.
template <typename XT, int GL, bool IN_LDS>
__global__ __launch_bounds__(512) void moe_down_kernel(MoeArgs g) {
    constexpr int P = kHiddenParts, S = kHiddenSlots, TPT = 16 / S, U = 2;
    extern __shared__ __align__(16) uint8_t lds[];
    float* sums = reinterpret_cast<float*>(lds);                                     // [wave][T][16]
    int4* groups = reinterpret_cast<int4*>(sums + kDownWaves * g.T * 16);            // [pairs at most]
    int32_t* order = reinterpret_cast<int32_t*>(groups + g.pairs);                   // [pairs]
    int32_t* places = order + g.pairs;                                               // [pairs], in that order: of the token's sums
    float* weights = reinterpret_cast<float*>(places + g.pairs);                     // [pairs], in that order
    int32_t* found = reinterpret_cast<int32_t*>(weights + g.pairs);
    uint16_t* xs = reinterpret_cast<uint16_t*>(lds + down_small(g.T, g.pairs));      // [pairs * parts][columns + 8]
    const int lane = threadIdx.x & 63, kb = lane >> 4, r = lane & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int d0 = 16 * blockIdx.x;
    const int64_t fp = row_pitch(g.F);
    const int chunks = (int)(q4_padded(g.F) / kQ4Chunk), first_chunk = blockIdx.y * g.part_chunks;
    const int end = min(chunks, first_chunk + g.part_chunks), steps = (end - first_chunk + U - 1) / U;
    const int xp = g.part_chunks * kQ4Chunk + 8;
    const int experts = __builtin_amdgcn_readfirstlane(g.groups[0].x), items = experts * steps;
    const int64_t pitch = q4_row_bytes(g.F), row_groups = (g.F + (32 << GL) - 1) >> (5 + GL);
    float* mine = sums + wave * g.T * 16;
    Q4Walk<false, 1, 1, GL, U> walk;
    const auto load = [&](int step, int4 group) {
        const int64_t e = __builtin_amdgcn_readfirstlane(group.x);
        walk.tile(0, g.w2 + e * g.D * pitch, g.s2 + e * g.D * row_groups, d0, g.D, g.F, lane);
        walk.load(first_chunk + step * U);
    };
    // (the next item of a wavefront is found by counting: divisions are 25 instructions each)
    int expert = wave / steps, step = wave - expert * steps;
    if (wave < items) load(step, g.groups[1 + expert]);
    if constexpr (IN_LDS)
        rows_to_lds(xs, xp, [&](int row) { return g.hp + first_chunk * kQ4Chunk + row * fp; }, g.pairs * P, g.part_chunks * (kQ4Chunk / 8),
                    g.magic_h, (end - first_chunk) * (kQ4Chunk / 8));
    for (int p = threadIdx.x; p < g.pairs; p += blockDim.x) {
        const int pair = g.order[p];
        order[p] = pair;
        places[p] = pair / g.top_k * 16;
        weights[p] = g.weights[pair];
        if (p < experts) groups[p] = g.groups[1 + p];
    }
    for (int i = threadIdx.x; i < kDownWaves * g.T * 16; i += blockDim.x) sums[i] = 0.f;
    __syncthreads();
    for (int item = wave; item < items; item += kDownWaves) {
        const int c = first_chunk + step * U;
        const int4 group = groups[expert];
        const int32_t *list = order + group.y, *place = places + group.y;
        const float* share = weights + group.y;
        for (step += kDownWaves; step >= steps; step -= steps) ++expert;
        const int tokens = __builtin_amdgcn_readfirstlane(group.z);
        walk.take();
        uint32_t sc[1][decltype(walk)::kWords][4];
        walk.spread(sc);
        for (int n0 = 0; n0 < tokens; n0 += TPT) {
            const int here = min(tokens - n0, TPT);
            std::conditional_t<IN_LDS, LdsRowsOfX<1>, RowsOfX<1, U, false>> x;
            if constexpr (IN_LDS) {
                x.at[0] = xs + (list[n0 + min(r / S, here - 1)] * P + min(r % S, P - 1)) * xp + 8 * kb - first_chunk * kQ4Chunk;
            } else {
                x.kb = kb;
                x.columns = chunks * kQ4Chunk;
                x.last = chunks - 1;
                x.at[0] = r / S < here && r % S < P ? g.hp + ((int64_t)list[n0 + r / S] * P + r % S) * fp : nullptr;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) x.fetch(c, u);
            if (n0 + TPT >= tokens && item + kDownWaves < items) load(step, groups[expert]);
            f32x4 acc[1][1] = {};
            walk.template eat<0, U>(c, end, x, sc, acc);
            if (kb < here) {      // a lane's four rows are the parts of token kb
                const float sum = acc[0][0][0] + (acc[0][0][1] + acc[0][0][2]);
                float* to = mine + place[n0 + kb] + r;
                *to = fmaf(share[n0 + kb], sum, *to);
            }
        }
    }
    __syncthreads();
    const int all = g.T * 16;
    float* parts = g.parts + (int64_t)blockIdx.x * g.split * all;      // of this tile
    for (int o = threadIdx.x; o < all; o += blockDim.x) {
        float sum = sums[o];
        for (int w = 1; w < kDownWaves; ++w) sum += sums[w * all + o];
        if (g.split == 1) {
            if (d0 + o % 16 < g.D) static_cast<typename XT::type*>(g.y)[o / 16 * g.ldy + d0 + o % 16] = XT::store(sum * kQ4Unit<false>);
        } else {
            __hip_atomic_store(parts + blockIdx.y * all + o, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    if (g.split == 1 || !last_of(g.done + blockIdx.x, g.split, found)) return;
    for (int o = threadIdx.x; o < all; o += blockDim.x) {
        float sum = __hip_atomic_load(parts + o, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        for (int z = 1; z < g.split; ++z) sum += __hip_atomic_load(parts + z * all + o, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (d0 + o % 16 < g.D) static_cast<typename XT::type*>(g.y)[o / 16 * g.ldy + d0 + o % 16] = XT::store(sum * kQ4Unit<false>);
    }
}

template <typename XT, int GL, int NT, bool IN_LDS, bool ALONE>
int launch_up_rows(const MoeArgs& g, size_t lds, hipStream_t st) {
    using Reg = LdsKernelOf<moe_up_kernel<XT, NT, GL, IN_LDS, ALONE>>;
    if (lds > kLdsWithoutLimit) {
        const int rc = ensure_lds_limit(Reg::reg, st);
        if (rc != BS_OK) return rc;
    }
    const dim3 grid((unsigned)((q4_padded(g.F) + 16 * g.tiles - 1) / (16 * g.tiles)), (unsigned)(g.routed && g.E < g.pairs ? g.E : g.pairs));
    hipLaunchKernelGGL((moe_up_kernel<XT, NT, GL, IN_LDS, ALONE>), grid, dim3(128 * g.ways), lds, st, g);
    return hip_status(hipGetLastError());
}

// Tiles of 16 hidden units for a workgroup of `up`, two of which share a compute unit.  What the busiest one does: its bytes at
// the rate of reads, 4 us to begin and end each round of 512 workgroups, 3 where it has one only.  How many experts several tokens
// choose is not known here: `experts`, their expected number, or, at a weight of 0.3, a tenth more (the same launch takes 28.7 us with
// 46 chosen experts and 42.5 with 47, where those need a second round).  64 experts of 2048 x 1024, 32 of them chosen: 23.3 / 20.2 /
// 17.6 / 20.1 / 17.2 us with 1 / 2 / 4 / 5 / 8; 8 of 944 x 4094: 31 / 20.6 / 14.9 / 17 / 18.8.
int tiles_for(double experts, bool known, int64_t tiles, double bytes, int lds) {
    int best = 1;
    double least = 0;
    for (int t = 1; t <= 16 && (t == 1 || t * lds <= 32 * 1024); ++t) {
        const auto time = [&](double chosen) {
            const double wgs = chosen * ((tiles + t - 1) / t);
            return std::ceil(wgs / 256) * t * bytes / 21.5e3 + 4 * std::ceil(wgs / 512) + (wgs <= 256 ? 3 : 0);
        };
        const double cost = known ? time(experts) : 0.7 * time(experts) + 0.3 * time(1.1 * experts);
        if (t == 1 || cost < least) { best = t; least = cost; }
    }
    return best;
}

template <typename XT, int GL>
int launch_up(MoeArgs g, hipStream_t st) {
    constexpr int TPT = 16 / XT::kSlots;
    const size_t row = (size_t)XT::kParts * (q4_padded(g.D) + 8) * 2;      // of x in LDS
    const double experts = g.E * (1 - std::pow(1 - (double)g.top_k / g.E, g.T));
    g.tiles = tiles_for(experts, g.T == 1, q4_padded(g.F) / 16, 32.0 * (q4_row_bytes(g.D) + 2 * q4_groups(g.D, 32 << GL)), 2 * g.ways * std::min(g.T, TPT) * 64);
    const auto sizes = [&](int rows, bool alone, size_t& small, size_t& sums) {
        g.rows = g.T < rows ? g.T : rows;
        small = up_small(g.T, g.pairs, g.E, alone);
        sums = (size_t)2 * g.ways * g.tiles * g.rows * 64;
    };
    size_t small, sums;
    sizes(TPT, true, small, sums);
    // The logits by every workgroup itself where they are few (1 token, 8 experts, 1500 columns: 15.0 us in two kernels against
    // 17.4 in three); 64 experts of 2048 columns would have each read 256 KB.
    if (g.T <= TPT && g.T * row <= 40 * 1024 && g.T * g.E <= 4 * g.ways && (int64_t)g.T * g.E * g.D <= 32768)
        return launch_up_rows<XT, GL, 1, true, true>(g, small + sums + g.T * row, st);
    g.routed = g.T >= 4;
    hipLaunchKernelGGL(moe_logits_kernel<XT>, dim3(g.T, (g.E + 3) / 4), dim3(256), 0, st, g);
    int rc = hip_status(hipGetLastError());
    if (rc != BS_OK) return rc;
    if (g.routed) {
        const int lds = route_bytes(g.pairs, g.E);
        hipLaunchKernelGGL(moe_route_kernel, dim3(1), dim3(g.T < 16 ? 64 * g.T : 1024), lds, st, g);
        rc = hip_status(hipGetLastError());
        if (rc != BS_OK) return rc;
    }
    // x in LDS where most experts' tokens fit there at once, or in three passes over the expert's codes: 12 tokens of 2322 x 2716 in
    // fp32, 7 of 8 experts each, 45 us in three passes, 75 with x from memory in two
    for (const size_t room : {kLdsOfX, 2 * kLdsOfX}) {
        const int fit = (int)(room / row < TPT ? room / row : TPT);
        const int pairs = room == kLdsOfX ? 2 * g.pairs : g.pairs / 3;
        if (fit < 1 || (fit < g.T && pairs > g.E * fit)) continue;
        sizes(fit, false, small, sums);
        return launch_up_rows<XT, GL, 1, true, false>(g, small + sums + g.rows * row, st);
    }
    if (g.T > TPT) {
        sizes(2 * TPT, false, small, sums);
        return launch_up_rows<XT, GL, 2, false, false>(g, small + sums, st);
    }
    sizes(TPT, false, small, sums);
    return launch_up_rows<XT, GL, 1, false, false>(g, small + sums, st);
}

template <typename XT, int GL, bool IN_LDS>
int launch_down(const MoeArgs& g, size_t lds, hipStream_t st) {
    using Reg = LdsKernelOf<moe_down_kernel<XT, GL, IN_LDS>>;
    if (lds > kLdsWithoutLimit) {
        const int rc = ensure_lds_limit(Reg::reg, st);
        if (rc != BS_OK) return rc;
    }
    const dim3 grid((unsigned)((g.D + 15) / 16), (unsigned)g.split);
    hipLaunchKernelGGL((moe_down_kernel<XT, GL, IN_LDS>), grid, dim3(64 * kDownWaves), lds, st, g);
    return hip_status(hipGetLastError());
}

template <typename XT, int GL>
int launch(const MoeArgs& g, hipStream_t st) {
    const int rc = launch_up<XT, GL>(g, st);
    if (rc != BS_OK) return rc;
    const size_t small = down_small(g.T, g.pairs), h = (size_t)g.pairs * kHiddenParts * (g.part_chunks * kQ4Chunk + 8) * 2;
    return h <= kLdsOfH ? launch_down<XT, GL, true>(g, small + h, st) : launch_down<XT, GL, false>(g, small, st);
}

template <typename XT>
int launch_group(const MoeArgs& g, int group, hipStream_t st) {
    switch (q4_group_shift(group)) {
        case 0: return launch<XT, 0>(g, st);
        case 1: return launch<XT, 1>(g, st);
        default: return launch<XT, 2>(g, st);
    }
}

// the workspace: x's rows, h's rows, logits, sums of down's workgroups, their counts
struct Space {
    size_t h, logits, groups, order, parts, done, all;
    int split, part_chunks;
};

Space space_for(int dtype, int64_t T, int64_t D, int64_t F, int E, int top_k) {
    Space s;
    // Workgroups of a tile of outputs: as many as let h of a part of F fit LDS, and then as many as give every compute unit two
    // (more where their wavefronts have four steps each).  7 tokens of 2048 x 1024, 64 experts, 6 of them each: `down` 14.8 us with
    // four workgroups a tile, 34 with one.
    const int64_t tiles = (D + 15) / 16, chunks = q4_padded(F) / kQ4Chunk, pairs = T * top_k, experts = pairs < E ? pairs : E;
    s.split = 1;
    s.part_chunks = (int)chunks;
    while (s.split < 16 && s.part_chunks > 2) {
        const auto room = [&](int64_t n) { return pairs * kHiddenParts * (n * kQ4Chunk + 8) * 2; };
        const bool fits = room(s.part_chunks) <= (int64_t)kLdsOfH || room(2) > (int64_t)kLdsOfH;      // or no split would make it fit
        const int64_t steps = (s.part_chunks + 1) / 2 * experts;
        if (fits && (tiles * s.split >= 512 || steps < 4 * kDownWaves)) break;
        s.split *= 2;
        s.part_chunks = (int)((chunks + s.split - 1) / s.split + 1) / 2 * 2;
    }
    s.split = (int)((chunks + s.part_chunks - 1) / s.part_chunks);
    const auto up16 = [](size_t n) { return (n + 15) / 16 * 16; };
    s.h = (size_t)T * (dtype == BS_F32 ? 3 : 1) * row_pitch(D) * 2;
    s.logits = s.h + (size_t)pairs * kHiddenParts * row_pitch(F) * 2;
    s.groups = s.logits + up16((size_t)T * E * 4);
    s.order = s.groups + (size_t)(pairs + 1) * 16;
    s.parts = s.order + up16((size_t)pairs * 4);
    s.done = s.parts + (s.split > 1 ? (size_t)tiles * s.split * T * 64 : 0);
    s.all = s.done + (s.split > 1 ? (size_t)tiles * 4 : 0);
    return s;
}

}  // namespace

size_t q4_moe_workspace_bytes(int dtype, int64_t T, int64_t D, int64_t F, int E, int top_k) {
    const size_t rest = T % kTokens ? space_for(dtype, T % kTokens, D, F, E, top_k).all : 0;
    if (T < kTokens) return rest;
    const size_t whole = space_for(dtype, kTokens, D, F, E, top_k).all;
    return whole > rest ? whole : rest;
}

namespace {

int launch_tokens(const void* x, int dtype, int64_t T, int64_t ldx, int64_t D, const void* router, int E, const uint8_t* w1,
                  const uint16_t* s1, const uint8_t* w2, const uint16_t* s2, int64_t F, int group, int top_k, int renormalise, void* y,
                  int64_t ldy, int32_t* ids, float* weights, void* workspace, hipStream_t st) {
    const Space s = space_for(dtype, T, D, F, E, top_k);
    MoeArgs g{};
    g.x = x; g.router = router; g.ldx = ldx; g.ldy = ldy;
    g.T = (int)T; g.D = (int)D; g.E = E; g.F = (int)F; g.top_k = top_k; g.pairs = (int)T * top_k;
    g.renormalise = renormalise != 0;
    g.w1 = w1; g.w2 = w2; g.s1 = s1; g.s2 = s2; g.y = y; g.ids = ids; g.weights = weights;
    char* const base = static_cast<char*>(workspace);
    g.xp = reinterpret_cast<uint16_t*>(base);
    g.hp = reinterpret_cast<uint16_t*>(base + s.h);
    g.logits = reinterpret_cast<float*>(base + s.logits);
    g.parts = reinterpret_cast<float*>(base + s.parts);
    g.done = reinterpret_cast<uint32_t*>(base + s.done);
    g.split = s.split;
    g.part_chunks = s.part_chunks;
    g.groups = reinterpret_cast<int4*>(base + s.groups);
    g.order = reinterpret_cast<int32_t*>(base + s.order);
    g.magic_x = magic_u32((uint32_t)(q4_padded(D) / 8));
    g.magic_h = magic_u32((uint32_t)(s.part_chunks * (kQ4Chunk / 8)));
    const int64_t steps = (q4_padded(D) / kQ4Chunk + 1) / 2;
    g.ways = (int)(steps < 4 ? steps : 4);
    switch (dtype) {
        case BS_F32: return launch_group<F32>(g, group, st);
        case BS_F16: return launch_group<F16>(g, group, st);
        default: return launch_group<BF16>(g, group, st);
    }
}

}  // namespace

int launch_q4_moe(const void* x, int dtype, int64_t T, int64_t ldx, int64_t D, const void* router, int E, const uint8_t* w1,
                  const uint16_t* s1, const uint8_t* w2, const uint16_t* s2, int64_t F, int group, int top_k, int renormalise, void* y,
                  int64_t ldy, int32_t* ids, float* weights, void* workspace, size_t workspace_bytes, hipStream_t st) {
    if (!workspace || workspace_bytes < q4_moe_workspace_bytes(dtype, T, D, F, E, top_k) || (reinterpret_cast<uintptr_t>(workspace) & 15))
        return BS_ERR_WORKSPACE;
    const int64_t size = dtype_bytes(dtype);
    for (int64_t t = 0; t < T; t += kTokens) {
        const int rc = launch_tokens(static_cast<const char*>(x) + t * ldx * size, dtype, T - t < kTokens ? T - t : kTokens, ldx, D, router,
                                     E, w1, s1, w2, s2, F, group, top_k, renormalise, static_cast<char*>(y) + t * ldy * size, ldy,
                                     ids + t * top_k, weights + t * top_k, workspace, st);
        if (rc != BS_OK) return rc;
    }
    return BS_OK;
}

}  // namespace bs

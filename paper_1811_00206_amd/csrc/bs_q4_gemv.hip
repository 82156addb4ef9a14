// y[n] = W . x[n] for a 4-bit matrix and one or a few vectors (bs.h: bs_q4_gemv).
//
// Bound: the codes are read once, M * K / 2 bytes.  A wavefront owns 16 * R rows; the wavefronts of a workgroup share K
// (step i of U chunks goes to wavefront i % ways), so that a few thousand rows already fill the chip, and add their sums in
// LDS in the order of the wavefronts: the same bits from every call.
//
// x comes to the matrix unit in three ways.  A few virtual rows (4: one fp32 vector, four in 16 bits) are brought to LDS and split
// into parts there: by a workgroup, in slabs of K, where `tiles` groups of 16 rows share them, or by every wavefront for its own
// columns, a step ahead, where a workgroup has one group of rows.  More are read from memory by every
// wavefront, 64 bytes of 16 rows at a time, which the caches hold: rows of 16-bit vectors as they are, or tiles of parts that a
// first kernel puts into the workspace.
#include "bs_q4.h"

namespace bs {
namespace {

constexpr size_t kSlabBytes = 64 * 1024;    // of x in LDS
constexpr int kStagedRows = 4;              // virtual rows that are brought to LDS
constexpr int kSplitMost = 16;              // workgroups that share K

struct GemvArgs {
    const uint8_t* codes;
    const uint16_t* scales;
    int64_t M, K, N, ldx, ldy;
    const void* x;      // as given, or the parts of every vector in the workspace
    void* y;
    int ways, tiles;    // wavefronts that share K; groups of wavefronts that share x in LDS
    int slab;           // columns of x in LDS at once
    int split, part_chunks;      // workgroups that share K, and the chunks of each
    float* parts;       // [tile of rows and tokens][split][its sums], if there are several
    uint32_t* done;     // [tile]: those of them that are done
};

// a wavefront's sums to LDS: [wave][R][NT][TPT][16]
template <int S, int R, int NT>
__device__ __forceinline__ void put_sums(float* sums, int wave, int lane, const f32x4 (&acc)[R][NT]) {
    constexpr int TPT = 16 / S, V = 4 / S;
    const int kb = lane >> 4, r = lane & 15;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                // a lane's four rows are four tokens, or the parts of one (the small parts are added first)
                float sum = acc[i][t][v];
                if constexpr (S == 4) sum = acc[i][t][0] + (acc[i][t][1] + acc[i][t][2]);
                sums[(((wave * R + i) * NT + t) * TPT + kb * V + v) * 16 + r] = sum;
            }
}

template <typename XT, int GL, int U>
__global__ __launch_bounds__(1024) void q4_gemv_kernel(GemvArgs g) {
    using T = typename XT::type;
    constexpr int P = XT::kParts, S = XT::kSlots;
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x & 63, kb = lane >> 4, r = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), way = wave % g.ways, tile = wave / g.ways;
    const int64_t row0 = (int64_t)blockIdx.x * (16 * g.tiles);
    const int chunks = (int)((g.K + kQ4Chunk - 1) / kQ4Chunk), tokens = (int)g.N;
    Q4Walk<XT::kHalf, 1, 1, GL, U> walk;
    walk.tile(0, g.codes, g.scales, row0 + 16 * tile, g.M, g.K, lane);
    f32x4 acc[1][1] = {};
    uint16_t* xs = reinterpret_cast<uint16_t*>(lds);
    const int xp = g.slab + 8;                              // row pitch: 16 bytes more, so that rows start on other banks
    // the lane's virtual row; rows without a token repeat the last one
    const uint16_t* mine = xs + (min(r / S, tokens - 1) * P + min(r % S, P - 1)) * xp + 8 * kb;
    const int per_slab = g.slab / kQ4Chunk;
    for (int c0 = 0; c0 < chunks; c0 += per_slab) {
        const int end = min(chunks, c0 + per_slab), c = c0 + U * way;
        walk.load(c);
        if (c0) __syncthreads();
        const int64_t k0 = (int64_t)c0 * kQ4Chunk;
        const int pieces = (end - c0) * (kQ4Chunk / 8);
        for (int n = 0; n < tokens; ++n) {
            const T* row = static_cast<const T*>(g.x) + n * g.ldx;
            for (int j = threadIdx.x; j < pieces; j += blockDim.x) {
                uint4 p[P];
                pieces8<XT>(row, k0 + 8 * j, g.K, p);
#pragma unroll
                for (int i = 0; i < P; ++i) *reinterpret_cast<uint4*>(xs + (n * P + i) * xp + 8 * j) = p[i];
            }
        }
        __syncthreads();
        LdsRowsOfX<1> staged{{mine - k0}};
        walk.template rest<U>(c, g.ways, end, staged, acc);
    }
    __syncthreads();
    float* sums = reinterpret_cast<float*>(lds);
    put_sums<S>(sums, wave, lane, acc);
    __syncthreads();
    constexpr int kOut = 256 / S;      // of a tile
    for (int o = threadIdx.x; o < kOut * g.tiles; o += blockDim.x) {
        const int i = o / kOut, n = o % kOut / 16;
        const int64_t row = row0 + 16 * i + o % 16;
        if (n >= tokens || row >= g.M) continue;
        const float* from = sums + i * g.ways * kOut + o % kOut;
        float sum = from[0];
        for (int w = 1; w < g.ways; ++w) sum += from[w * kOut];
        static_cast<T*>(g.y)[n * g.ldy + row] = XT::store(sum * kQ4Unit<XT::kHalf>);
    }
}

// x of a wavefront's step, 128 * U columns of a few virtual rows, in LDS of its own: asked for a step ahead, split and put there
// when the step begins.  K >= 8.
template <typename XT, int U>
struct OwnX {
    using T = typename XT::type;
    static constexpr int P = XT::kParts, kMost = P == 3 ? 1 : kStagedRows, kPitch = U * kQ4Chunk + 8;
    const T* x;
    int64_t K, ldx;
    int tokens, lane;
    uint16_t* own;            // [tokens * P][kPitch]
    const uint16_t* mine;     // the lane's row, from its column 8 * kb on
    uint4 raw[kMost][sizeof(T) / 2];
    __device__ __forceinline__ int64_t column(int c) const { return (int64_t)c * kQ4Chunk + 8 * (U == 4 ? lane : lane & 31); }
    __device__ __forceinline__ void fetch(int c) {
        const int64_t from = min(column(c), K - 8);
#pragma unroll
        for (int n = 0; n < kMost; ++n)
            if (n < tokens) __builtin_memcpy(raw[n], x + n * ldx + from, sizeof(raw[n]));
    }
    __device__ __forceinline__ void put(int c) {
        const int64_t k = column(c), from = min(k, K - 8);
#pragma unroll
        for (int n = 0; n < kMost; ++n) {
            if (n >= tokens) break;
            uint4 p[P];
            if constexpr (P == 3) {
                float v[8];
                __builtin_memcpy(v, raw[n], 32);
                moved8(v, k, from);
                split8(v, p);
            } else {
                p[0] = moved8(raw[n][0], k, from, K);
            }
#pragma unroll
            for (int i = 0; i < P; ++i) *reinterpret_cast<uint4*>(own + (n * P + i) * kPitch + (k - (int64_t)c * kQ4Chunk)) = p[i];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // some lanes write what others read
    }
    __device__ __forceinline__ uint4 operator()(int, int, int u, int i) const {
        return *reinterpret_cast<const uint4*>(mine + u * kQ4Chunk + 32 * i);
    }
};

// The same for few rows: a workgroup has one tile, so no two wavefronts want the same columns of x, and each brings its own.
template <typename XT, int GL, int U>
__global__ __launch_bounds__(1024) void q4_gemv_own_kernel(GemvArgs g) {
    using T = typename XT::type;
    constexpr int P = XT::kParts, S = XT::kSlots, kOut = 256 / S;
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x & 63, kb = lane >> 4, r = lane & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row0 = (int64_t)blockIdx.x * 16;
    const int chunks = (int)((g.K + kQ4Chunk - 1) / kQ4Chunk), tokens = (int)g.N;
    Q4Walk<XT::kHalf, 1, 1, GL, U> walk;
    walk.tile(0, g.codes, g.scales, row0, g.M, g.K, lane);
    OwnX<XT, U> x;
    x.x = static_cast<const T*>(g.x);
    x.K = g.K;
    x.ldx = g.ldx;
    x.tokens = tokens;
    x.lane = lane;
    x.own = reinterpret_cast<uint16_t*>(lds) + wave * tokens * P * x.kPitch;
    x.mine = x.own + (min(r / S, tokens - 1) * P + min(r % S, P - 1)) * x.kPitch + 8 * kb;
    f32x4 acc[1][1] = {};
    int c = wave * U;
    walk.load(c);
    x.fetch(c);
    while (c < chunks) {
        const int now = c;
        walk.take();
        x.put(now);
        c += g.ways * U;
        if (c < chunks) {
            walk.load(c);
            x.fetch(c);
        }
        uint32_t sc[1][decltype(walk)::kWords][4];
        walk.spread(sc);
        walk.template eat<0, U>(now, chunks, x, sc, acc);
    }
    __syncthreads();
    float* sums = reinterpret_cast<float*>(lds);
    put_sums<S>(sums, wave, lane, acc);
    __syncthreads();
    for (int o = threadIdx.x; o < kOut; o += blockDim.x) {
        const int64_t row = row0 + o % 16;
        if (o / 16 >= tokens || row >= g.M) continue;
        float sum = sums[o];
        for (int w = 1; w < g.ways; ++w) sum += sums[w * kOut + o];
        static_cast<T*>(g.y)[o / 16 * g.ldy + row] = XT::store(sum * kQ4Unit<XT::kHalf>);
    }
}

template <typename XT, int NT, int R, int GL, bool TILED>
__global__ __launch_bounds__(NT * R == 1 ? 1024 : 512) void q4_gemv_many_kernel(GemvArgs g) {
    using T = typename XT::type;
    constexpr int S = XT::kSlots, TPT = 16 / S, U = 2;     // TPT: tokens per tile of virtual rows
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x & 63, kb = lane >> 4, r = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row0 = (int64_t)blockIdx.x * (16 * R), n0 = (int64_t)blockIdx.y * (NT * TPT);
    const int tokens = (int)min(g.N - n0, (int64_t)(NT * TPT));
    const int chunks = (int)((g.K + kQ4Chunk - 1) / kQ4Chunk);
    const int first = TILED ? blockIdx.z * g.part_chunks : 0, end = TILED ? min(chunks, first + g.part_chunks) : chunks;
    Q4Walk<XT::kHalf, NT, R, GL, U> walk;
#pragma unroll
    for (int i = 0; i < R; ++i) walk.tile(i, g.codes, g.scales, row0 + 16 * i, g.M, g.K, lane);
    f32x4 acc[R][NT] = {};
    constexpr int kFetch = NT <= 2 ? U : 1;
    if constexpr (TILED) {
        TilesOfX<NT, kFetch> x;
        // (tiles of 16 virtual rows that no vector is in were not made: the last one is read instead, for rows that nobody stores)
        const int last = (int)((g.N + TPT - 1) / TPT) - 1;
#pragma unroll
        for (int t = 0; t < NT; ++t)
            x.at[t] = static_cast<const uint16_t*>(g.x) + (int64_t)min((int)blockIdx.y * NT + t, last) * chunks * 2048 + 8 * lane;
        x.last = chunks - 1;
        walk.load(first + wave * U);
        walk.template rest<kFetch>(first + wave * U, g.ways, end, x, acc);
    } else {
        static_assert(S == 1);
        RowsOfX<NT, kFetch, true> x;
        x.kb = kb;
        x.columns = (int)g.K;
        x.last = chunks - 1;
#pragma unroll
        for (int t = 0; t < NT; ++t)
            x.at[t] = t * TPT + r < tokens ? static_cast<const uint16_t*>(g.x) + (n0 + t * TPT + r) * g.ldx : nullptr;
        walk.load(wave * U);
        walk.template rest<kFetch>(wave * U, g.ways, end, x, acc);
    }
    float* sums = reinterpret_cast<float*>(lds);
    put_sums<S>(sums, wave, lane, acc);
    __syncthreads();
    constexpr int kOut = R * NT * TPT * 16;
    const auto store = [&](int o, float sum) {
        const int64_t row = row0 + o / (NT * TPT * 16) * 16 + o % 16;
        static_cast<T*>(g.y)[(n0 + o / 16 % (NT * TPT)) * g.ldy + row] = XT::store(sum * kQ4Unit<XT::kHalf>);
    };
    const auto wanted = [&](int o) { return o / 16 % (NT * TPT) < tokens && row0 + o / (NT * TPT * 16) * 16 + o % 16 < g.M; };
    const int64_t tile = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    float* parts = TILED ? g.parts + tile * g.split * kOut : nullptr;
    for (int o = threadIdx.x; o < kOut; o += blockDim.x) {
        if (!wanted(o)) continue;
        float sum = sums[o];
        for (int w = 1; w < g.ways; ++w) sum += sums[w * kOut + o];
        if (!TILED || g.split == 1) store(o, sum);
        else __hip_atomic_store(parts + blockIdx.z * kOut + o, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if constexpr (TILED) {
        if (g.split == 1 || !last_of(g.done + tile, g.split, reinterpret_cast<int*>(lds))) return;
        for (int o = threadIdx.x; o < kOut; o += blockDim.x) {
            if (!wanted(o)) continue;
            float sum = __hip_atomic_load(parts + o, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            for (int z = 1; z < g.split; ++z) sum += __hip_atomic_load(parts + z * kOut + o, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            store(o, sum);
        }
    }
}

// x as the matrix unit takes it (TilesOfX): a workgroup writes a chunk of a tile, 4 KB.  Columns behind K are zero, rows
// without a token stay as they are.
template <typename XT>
__global__ __launch_bounds__(256) void q4_tiles_kernel(const void* x, int64_t K, int64_t N, int64_t ldx, uint16_t* tiles, uint32_t* done,
                                                       int64_t counts) {
    using T = typename XT::type;
    constexpr int P = XT::kParts, S = XT::kSlots, TPT = 16 / S;
    for (int64_t i = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * blockDim.x + threadIdx.x; i < counts;
         i += (int64_t)gridDim.x * gridDim.y * blockDim.x)
        done[i] = 0;
    const int token = threadIdx.x % TPT, piece = threadIdx.x / TPT;
    const int64_t n = (int64_t)blockIdx.y * TPT + token, k = (int64_t)blockIdx.x * kQ4Chunk + 8 * piece;
    if (n >= N) return;
    uint4 p[P];
    pieces8<XT>(static_cast<const T*>(x) + n * ldx, k, K, p);
    uint16_t* to = tiles + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 2048 + 128 * piece + 8 * S * token;
#pragma unroll
    for (int i = 0; i < P; ++i) *reinterpret_cast<uint4*>(to + 8 * i) = p[i];
}

struct Plan {
    bool staged, own;
    bool tiled;
    int nt, r, u, ways, tiles, slab, split, part_chunks;
    int64_t counts;
    size_t lds, parts, done, workspace;
};

Plan plan_for(int dtype, int64_t M, int64_t K, int64_t N) {
    const int parts = dtype == BS_F32 ? 3 : 1, tpt = dtype == BS_F32 ? 4 : 16;
    const int64_t tiles = (M + 15) / 16, chunks = (K + kQ4Chunk - 1) / kQ4Chunk;
    Plan p{};
    p.staged = N * parts <= kStagedRows;
    if (p.staged) {
        // Wavefronts that share K: as many as give the chip 2048 (eight for a compute unit), or what K has steps for.  Where
        // two are enough, four groups share x.  16384 x 8192: 14.9 us with 2 x 4, 16.6 with 2 x 1, 15.4 with 4 x 1, 17.2 with
        // 8 x 1.
        const int64_t steps = (chunks + 1) / 2;
        p.ways = 1;
        while (p.ways < 16 && tiles * p.ways < 2048 && p.ways < steps) p.ways *= 2;
        p.tiles = 4;
        // four chunks a step where every wavefront has many: 16384 x 8192 14.1 us against 14.9
        p.u = chunks >= 16 * p.ways ? 4 : 2;
        const int rows = (int)N * parts;
        // A workgroup of one tile has nobody to share x with: 4096 x 25088 for an fp32 vector 17 us with all of x in LDS first, 13.2
        // with x step by step; for four binary16 ones 24 and 14.7; 2000 x 1000 3.9 and 3.5.  Steps of four chunks where a wavefront has
        // more than three: 1269 x 13037 7.7 us instead of 8.1, 2000 x 1000 4.1 instead of 3.5.
        p.own = p.ways > 2;
        if (p.own) {
            p.u = chunks > 3 * p.ways ? 4 : 2;
            const size_t xs = (size_t)p.ways * rows * (p.u * kQ4Chunk + 8) * 2, sums = (size_t)p.ways * tpt * 16 * 4;
            p.lds = xs > sums ? xs : sums;
            return p;
        }
        const int64_t whole = p.u * kQ4Chunk, most = (int64_t)kSlabBytes / (rows * 2) / whole * whole, all = (K + whole - 1) / whole * whole;
        p.slab = (int)(all < most ? all : most);
        const size_t xs = (size_t)rows * (p.slab + 8) * 2, sums = (size_t)p.ways * p.tiles * tpt * 16 * 4;
        p.lds = xs > sums ? xs : sums;
        return p;
    }
    // A wavefront loads as much of x as R rows' worth of codes, so R is as large as leaves a workgroup for every compute unit:
    // 16384 x 8192 for 16 vectors 24.1 / 19.9 / 19.0 us with R = 1 / 2 / 4, 4096 x 25088 17.3 / 23.0 / 38.
    p.nt = N <= tpt ? 1 : N <= 2 * tpt ? 2 : 4;
    p.r = p.nt == 4 || tiles < 320 ? 1 : tiles < 1024 ? 2 : 4;
    const int most = p.r == 4 ? 4 : 8;
    // Workgroups that share K, where they are few or leave most of the chip without one at the end: what the busiest compute unit
    // does, a step of a wavefront being about 1 us and 0.5 for every 16 rows by 16 virtual rows, 2 us to begin and end, and 2 to join the
    // sums.
    // 698 x 7877 for 21 bfloat16 vectors 10.1 us alone, 8.0 / 6.6 / 9.9 with 2 / 4 / 8; 9409 x 22330 for 6 in fp32 67, 54.5 / 53 /
    // 62; 5000 x 5000 for 4 in fp32 8.0, 8.9 / 8.8 / 11.6; 4096 x 25088 for 13 in binary16 17.4, 19.5 / 18.9 / 20.5.
    const int64_t groups = (tiles + p.r - 1) / p.r * ((N + p.nt * tpt - 1) / (p.nt * tpt));
    double least = 0;
    for (int split = 1; split <= kSplitMost && split <= (chunks + 1) / 2; ++split) {
        const int part = (int)((chunks + split - 1) / split + 1) / 2 * 2, parts = (int)((chunks + part - 1) / part);
        const int steps = part / 2, ways = steps < most ? steps : most;
        const double cost = (double)((groups * parts + 255) / 256) * ((steps + ways - 1) / ways * (1 + 0.5 * p.r * p.nt) + 2) + (parts > 1 ? 2 : 0);
        if (split > 1 && cost >= least) continue;
        least = cost;
        p.ways = ways;
        p.split = parts;
        p.part_chunks = part;
    }
    // 16-bit vectors as they are, unless the matrix is large: every 16 * R rows of it read all of x, in pieces of 16 rows of half a line
    // each, which then costs more than a kernel that lays x out once.  A call for 7 / 16 / 32 bfloat16 vectors, as they are and as tiles:
    // 6000 x 3000 6.2 / 6.5 / 9.2 and 7.6 / 7.6 / 8.8 us, 4096 x 8192 9.8 / 12.9 / 20.5 and 10.4 / 10.5 / 13.0, 8192 x 8192 12.9 / 16.7 / 23.8
    // and 13.9 / 14.1 / 16.9, 8192 x 8200 12.1 / 13.5 / 19.2 and 13.8 / 14.0 / 17.0, 4096 x 25088 21 / 31 / 53 and 20 / 20 / 27.  (The size alone does
    // not tell all: more vectors, and rows a power of two apart, favour tiles sooner.)
    p.tiled = dtype == BS_F32 || p.nt == 4 || p.split > 1 || M * K >= ((int64_t)1 << 26);
    p.lds = (size_t)p.ways * p.r * p.nt * tpt * 16 * 4;
    p.parts = (size_t)((N + tpt - 1) / tpt) * 32 * q4_padded(K);
    p.counts = p.split > 1 ? groups : 0;
    p.done = p.parts + (size_t)p.counts * p.split * p.r * p.nt * tpt * 64;
    p.workspace = p.done + (size_t)p.counts * 4;
    return p;
}

template <typename XT, int GL, int U>
int launch_staged(const GemvArgs& g, const Plan& p, hipStream_t st) {
    using Reg = LdsKernelOf<q4_gemv_kernel<XT, GL, U>>;
    using Own = LdsKernelOf<q4_gemv_own_kernel<XT, GL, U>>;
    if (p.lds > kLdsWithoutLimit) {
        const int rc = p.own ? ensure_lds_limit(Own::reg, st) : ensure_lds_limit(Reg::reg, st);
        if (rc != BS_OK) return rc;
    }
    if (p.own) {
        hipLaunchKernelGGL((q4_gemv_own_kernel<XT, GL, U>), dim3((unsigned)((g.M + 15) / 16)), dim3(64 * p.ways), p.lds, st, g);
        return hip_status(hipGetLastError());
    }
    const dim3 grid((unsigned)((g.M + 16 * p.tiles - 1) / (16 * p.tiles)));
    hipLaunchKernelGGL((q4_gemv_kernel<XT, GL, U>), grid, dim3(64 * p.ways * p.tiles), p.lds, st, g);
    return hip_status(hipGetLastError());
}

template <typename XT, int NT, int R, int GL, bool TILED>
int launch_many(const GemvArgs& g, const Plan& p, hipStream_t st) {
    using Reg = LdsKernelOf<q4_gemv_many_kernel<XT, NT, R, GL, TILED>>;
    if (p.lds > kLdsWithoutLimit) {
        const int rc = ensure_lds_limit(Reg::reg, st);
        if (rc != BS_OK) return rc;
    }
    const int per = NT * (16 / XT::kSlots);
    const dim3 grid((unsigned)((g.M + 16 * R - 1) / (16 * R)), (unsigned)((g.N + per - 1) / per), (unsigned)g.split);
    hipLaunchKernelGGL((q4_gemv_many_kernel<XT, NT, R, GL, TILED>), grid, dim3(64 * p.ways), p.lds, st, g);
    return hip_status(hipGetLastError());
}

template <typename XT, int NT, int GL>
int launch_rows(const GemvArgs& g, const Plan& p, bool tiled, hipStream_t st) {
    if constexpr (XT::kParts == 1 && NT <= 2) {
        if (!tiled)
            return p.r == 1 ? launch_many<XT, NT, 1, GL, false>(g, p, st) : p.r == 2 ? launch_many<XT, NT, 2, GL, false>(g, p, st)
                                                                                     : launch_many<XT, NT, 4, GL, false>(g, p, st);
    }
    if constexpr (NT <= 2) {
        if (p.r == 2) return launch_many<XT, NT, 2, GL, true>(g, p, st);
        if (p.r == 4) return launch_many<XT, NT, 4, GL, true>(g, p, st);
    }
    return launch_many<XT, NT, 1, GL, true>(g, p, st);
}

template <typename XT, int GL>
int launch_group(const GemvArgs& g, const Plan& p, bool tiled, hipStream_t st) {
    if (p.staged) return p.u == 2 ? launch_staged<XT, GL, 2>(g, p, st) : launch_staged<XT, GL, 4>(g, p, st);
    return p.nt == 1   ? launch_rows<XT, 1, GL>(g, p, tiled, st)
           : p.nt == 2 ? launch_rows<XT, 2, GL>(g, p, tiled, st)
                       : launch_rows<XT, 4, GL>(g, p, tiled, st);
}

template <typename XT>
int launch_type(GemvArgs g, const Plan& p, int group, void* workspace, hipStream_t st) {
    bool tiled = false;
    if (!p.staged) {
        // rows that do not start where a load does: 698 x 7877 for 21 vectors 30 us as they are, 10 + 2.5 as tiles
        tiled = p.tiled || g.ldx % 8 || (reinterpret_cast<uintptr_t>(g.x) & 15);
        if (tiled) {
            constexpr int TPT = 16 / XT::kSlots;
            const dim3 grid((unsigned)(q4_padded(g.K) / kQ4Chunk), (unsigned)((g.N + TPT - 1) / TPT));
            hipLaunchKernelGGL(q4_tiles_kernel<XT>, grid, dim3(16 * TPT), 0, st, g.x, g.K, g.N, g.ldx,
                               static_cast<uint16_t*>(workspace), g.done, p.counts);
            const int rc = hip_status(hipGetLastError());
            if (rc != BS_OK) return rc;
            g.x = workspace;
        }
    }
    switch (q4_group_shift(group)) {
        case 0: return launch_group<XT, 0>(g, p, tiled, st);
        case 1: return launch_group<XT, 1>(g, p, tiled, st);
        default: return launch_group<XT, 2>(g, p, tiled, st);
    }
}

}  // namespace

size_t q4_gemv_workspace_bytes(int dtype, int64_t M, int64_t K, int64_t N) { return plan_for(dtype, M, K, N).workspace; }

int launch_q4_gemv(const uint8_t* codes, const uint16_t* scales, int64_t M, int64_t K, int group, const void* x, int dtype,
                   int64_t N, int64_t ldx, void* y, int64_t ldy, void* workspace, size_t workspace_bytes, hipStream_t st) {
    const Plan p = plan_for(dtype, M, K, N);
    if (p.workspace && (!workspace || workspace_bytes < p.workspace || (reinterpret_cast<uintptr_t>(workspace) & 15)))
        return BS_ERR_WORKSPACE;
    char* const base = static_cast<char*>(workspace);
    const GemvArgs g{codes, scales, M, K, N, ldx, ldy, x, y, p.ways, p.tiles, p.slab, p.split, p.part_chunks,
                     reinterpret_cast<float*>(base + p.parts), reinterpret_cast<uint32_t*>(base + p.done)};
    switch (dtype) {
        case BS_F32: return launch_type<F32>(g, p, group, workspace, st);
        case BS_F16: return launch_type<F16>(g, p, group, workspace, st);
        default: return launch_type<BF16>(g, p, group, workspace, st);
    }
}

}  // namespace bs

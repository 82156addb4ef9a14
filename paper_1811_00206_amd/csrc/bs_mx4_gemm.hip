// Rows of activations times an MX 4-bit matrix (bs.h: bs_mx4_gemm, bs_mx4_gemm_packed).
//
// Few rows: a wavefront has 16 rows of W, which go from memory to the matrix unit, and reads x beside them.  Many: tiles that pass
// through LDS (bs_mx4_tiles.h), with K split between workgroups where there are few of them; a second kernel then adds their sums up,
// in order.  Dense x is rounded by a kernel of its own first, or, where that is little work, by every workgroup for itself.
// Bound: HBM for few rows (16384 x 8192 for one row 14.2 us, 71 MB at 5 TB/s; 10000 x 1500 5.0, latency), the matrix unit for many.
#include <type_traits>

#include "bs_mx4_tiles.h"

namespace bs {
namespace {

struct Args {
    const uint8_t *codes, *scales, *x_codes, *x_scales;
    const void* x;              // dense
    int64_t ldx;
    int64_t M, K, N;
    uint32_t pieces_magic;      // division by 16 chunks
    int chunks, ways, tiles;    // chunks of 128 columns; wavefronts that share K, and groups of them
    const float* bias;
    void* y;
    int64_t ldy;
};

constexpr int kStep = 4;      // chunks of 128 columns that a wavefront takes at a time: 256 bytes of a row
constexpr int kFusedRows = 2, kFusedBytes = 48 * 1024;

typedef uint32_t Words __attribute__((ext_vector_type(4), aligned(4)));

// What a wavefront brings for a step: R pieces of 16 rows, a lane 16 bytes of its row for each chunk and the chunks' scale bytes.
template <int R>
struct Piece {
    uint4 q[R][kStep], s[R];
};

// 16 * R rows of W by 16 * NT of x for each wavefront.  Of a workgroup's wavefronts `ways` take turns with the steps of K and add their
// sums up in LDS, in order; `tiles` groups of them have different rows of W and the same of x.  x comes from memory in MX form, or
// (FUSED, for few rows) dense: then the workgroup first rounds it into LDS, while its first pieces of W are on their way.
template <typename XT, int R, int NT, bool FUSED>
__global__ __launch_bounds__(R * NT == 1 ? 1024 : 512) void mx4_rows_kernel(Args g) {
    static_assert(!FUSED || NT == 1);
    extern __shared__ __align__(16) uint8_t lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 15, kb = lane >> 4;
    const int way = wave % g.ways, tile = wave / g.ways;
    const int64_t m0 = ((int64_t)blockIdx.x * g.tiles + tile) * 16 * R, n0 = (int64_t)blockIdx.y * 16 * NT;
    const int chunks = g.chunks, whole = chunks / kStep;      // steps of four chunks
    const uint8_t* w[R];
    const uint32_t* ws[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int64_t row = min(m0 + 16 * i + r, g.M - 1);
        w[i] = g.codes + row * 64 * chunks + 16 * kb;
        ws[i] = reinterpret_cast<const uint32_t*>(g.scales) + row * chunks;
    }
    const auto load = [&](Piece<R>& p, int step) {
        const uint32_t at = (uint32_t)step * (64 * kStep);
#pragma unroll
        for (int i = 0; i < R; ++i) {
#pragma unroll
            for (int u = 0; u < kStep; ++u) p.q[i][u] = *reinterpret_cast<const uint4*>(w[i] + at + 64 * u);
            const Words v = *reinterpret_cast<const Words*>(reinterpret_cast<const uint8_t*>(ws[i]) + (at >> 4));
            p.s[i] = uint4{v[0], v[1], v[2], v[3]};
        }
    };
    // FUSED: all rows' pieces of 8 elements, one after the other; the next of a thread is on its way while one is rounded
    const uint32_t pieces = 16 * chunks, all = (uint32_t)g.N * pieces;
    const auto row_of = [&](uint32_t e) { return g.N == 1 ? 0 : div_magic_any(e, pieces, g.pieces_magic); };
    const auto bring = [&](uint32_t e, float (&v)[8]) {
        const uint32_t n = row_of(e), k = (e - n * pieces) * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
        if (e < all && k < g.K) load8<XT>(static_cast<const typename XT::type*>(g.x) + n * g.ldx, (int64_t)k, g.K, v);
    };
    // A thread's first piece of x goes before those of W: loads come back in order.
    float u[8], v[8];
    if constexpr (FUSED) bring(threadIdx.x, u);
    // Two pieces are on their way while one is multiplied.  (Where there is no whole step nothing is loaded here.)
    Piece<R> a, b;
    if (way < whole) load(a, way);
    if (way + g.ways < whole) load(b, way + g.ways);
    const uint8_t* x[NT];
    const uint32_t* xs[NT];
    if constexpr (FUSED) {
        const int pitch = (chunks + 3) & ~3;
        uint32_t* const scales = reinterpret_cast<uint32_t*>(lds + g.N * 64 * chunks);
        const auto round = [&](uint32_t e, const float (&v)[8]) {
            const uint32_t s = mx4_scale(max_of_4(mx4_most(v)));
            const uint32_t word = mx4_codes(v, mx4_factor(s));
            uint32_t bytes = s << (e / 4 % 4 * 8);
            bytes |= (uint32_t)dpp_move_i<0x141>((int)bytes);
            bytes |= (uint32_t)dpp_move_i<0x140>((int)bytes);
            if (e >= all) return;
            const uint32_t n = row_of(e);
            reinterpret_cast<uint32_t*>(lds)[e] = word;
            if (e % 16 == 0) scales[n * pitch + (e - n * pieces) / 16] = bytes;
        };
        for (uint32_t e = 0; e < all; e += 2 * blockDim.x) {
            const uint32_t next = e + blockDim.x;
            if (next < all) bring(next + threadIdx.x, v);
            round(e + threadIdx.x, u);
            if (next + blockDim.x < all) bring(next + blockDim.x + threadIdx.x, u);
            if (next < all) round(next + threadIdx.x, v);
        }
        const int row = min(r, (int)g.N - 1);
        x[0] = lds + row * 64 * chunks + 16 * kb;
        xs[0] = scales + row * pitch;
        __syncthreads();
    } else {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int64_t row = min(n0 + 16 * t + r, g.N - 1);
            x[t] = g.x_codes + row * 64 * chunks + 16 * kb;
            xs[t] = reinterpret_cast<const uint32_t*>(g.x_scales) + row * chunks;
        }
    }
    f32x4 acc[R][NT];
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[i][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    const auto multiply = [&](const Piece<R>& p, int u, int t, uint4 xv, uint32_t xsv) {
#pragma unroll
        for (int i = 0; i < R; ++i)
            acc[i][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx4_operand(p.q[i][u]), mx4_operand(xv), acc[i][t], 4, 4, 0,
                                                                         (int)(word_of(p.s[i], u) >> (8 * kb)), 0, (int)(xsv >> (8 * kb)));
    };
    const auto eat = [&](const Piece<R>& p, int step) {
        const uint32_t at = (uint32_t)step * (64 * kStep);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            uint4 xv[kStep];
#pragma unroll
            for (int u = 0; u < kStep; ++u) xv[u] = *reinterpret_cast<const uint4*>(x[t] + at + 64 * u);
            const Words sv = *reinterpret_cast<const Words*>(reinterpret_cast<const uint8_t*>(xs[t]) + (at >> 4));
#pragma unroll
            for (int u = 0; u < kStep; ++u) multiply(p, u, t, xv[u], sv[u]);
        }
    };
    for (int step = way; step < whole; step += 2 * g.ways) {
        eat(a, step);
        if (step + 2 * g.ways < whole) load(a, step + 2 * g.ways);
        if (step + g.ways >= whole) break;
        eat(b, step + g.ways);
        if (step + 3 * g.ways < whole) load(b, step + 3 * g.ways);
    }
    if (whole % g.ways == way)      // the rest, one to three chunks
        for (int c = whole * kStep; c < chunks; ++c) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                a.q[i][0] = *reinterpret_cast<const uint4*>(w[i] + (int64_t)c * 64);
                a.s[i].x = ws[i][c];
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) multiply(a, 0, t, *reinterpret_cast<const uint4*>(x[t] + (int64_t)c * 64), xs[t][c]);
        }
    if constexpr (FUSED) __syncthreads();
    f32x4* const sums = reinterpret_cast<f32x4*>(lds);      // [tile][way][R * NT][lane]
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) sums[(wave * R * NT + i * NT + t) * 64 + lane] = acc[i][t];
    __syncthreads();
    for (int e = threadIdx.x; e < g.tiles * R * NT * 64; e += blockDim.x) {
        const int l = e & 63, in = e >> 6, part = in % (R * NT), group = in / (R * NT);
        f32x4 s = sums[(group * g.ways * R * NT + part) * 64 + l];
        for (int v = 1; v < g.ways; ++v) s += sums[((group * g.ways + v) * R * NT + part) * 64 + l];
        const int64_t n = n0 + 16 * (part % NT) + (l & 15), m = (((int64_t)blockIdx.x * g.tiles + group) * R + part / NT) * 16 + 4 * (l >> 4);
        if (n >= g.N) continue;
        typename XT::type* const y = static_cast<typename XT::type*>(g.y) + n * g.ldy;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (m + j < g.M) y[m + j] = XT::store(g.bias ? s[j] + g.bias[m + j] : s[j]);
    }
}

template <typename XT, int R, int NT, bool FUSED>
int launch_rows(Args g, hipStream_t st) {
    const size_t sums = (size_t)g.ways * g.tiles * R * NT * 1024, x = FUSED ? (size_t)g.N * (64 * g.chunks + 4 * ((g.chunks + 3) & ~3)) : 0;
    const int64_t rows = 16 * R * g.tiles;
    const dim3 grid((unsigned)((g.M + rows - 1) / rows), (unsigned)((g.N + 16 * NT - 1) / (16 * NT)));
    hipLaunchKernelGGL((mx4_rows_kernel<XT, R, NT, FUSED>), grid, dim3(64 * g.ways * g.tiles), sums > x ? sums : x, st, g);
    return hip_status(hipGetLastError());
}

// ---- tiles

// sums of the shares of K, in order
template <typename XT>
__global__ __launch_bounds__(256) void mx4_join_kernel(Mx4Tiles g, int64_t n0) {
    typedef float Floats __attribute__((ext_vector_type(4), aligned(4)));
    const int64_t m = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, n = n0 + blockIdx.y, all = g.N * g.M;
    if (m >= g.M) return;
    const float* const from = g.sums + n * g.M + m;
    typename XT::type* const to = static_cast<typename XT::type*>(g.y) + n * g.ldy + m;
    if (m + 4 <= g.M) {
        Floats s = *reinterpret_cast<const Floats*>(from);
        for (int i = 1; i < g.split; i += 4) {      // four on their way together; those behind the last are the last one again
            Floats v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = *reinterpret_cast<const Floats*>(from + min(i + u, g.split - 1) * all);
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i + u < g.split) s += v[u];
        }
        if (g.bias) s += *reinterpret_cast<const Floats*>(g.bias + m);
#pragma unroll
        for (int e = 0; e < 4; ++e) to[e] = XT::store(s[e]);
    } else {
        for (int e = 0; m + e < g.M; ++e) {
            float s = from[e];
            for (int i = 1; i < g.split; ++i) s += from[e + i * all];
            to[e] = XT::store(g.bias ? s + g.bias[m + e] : s);
        }
    }
}

constexpr int kTileGroup = 400;      // these kernels' LDS limits are raised together: which one a product takes is a matter of its sizes

template <typename XT, int TN, int TM, int WN, int WM, int NB, bool SPLIT>
int launch_tiles(const Mx4Tiles& g, hipStream_t st) {
    constexpr auto kernel = mx4_tiles_kernel<XT, TN, TM, WN, WM, NB, SPLIT>;
    const int rc = ensure_lds_limit(LdsKernelOf<kernel, kTileGroup>::reg, st, nullptr, kTileGroup);
    if (rc != BS_OK) return rc;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(g.m_tiles * g.n_tiles * g.split)), dim3(256), (kMx4LdsBytes<TN, TM, NB>), st, g);
    return hip_status(hipGetLastError());
}

template <typename XT, int TN, int TM, int WN, int WM, int NB>
int launch_tiles(Mx4Tiles g, hipStream_t st) {
    g.m_tiles = (int)((g.M + TM - 1) / TM);
    g.n_tiles = (int)((g.N + TN - 1) / TN);
    if (g.split == 1) return launch_tiles<XT, TN, TM, WN, WM, NB, false>(g, st);
    const int rc = launch_tiles<F32, TN, TM, WN, WM, NB, true>(g, st);
    if (rc != BS_OK) return rc;
    const int64_t most = 65535;      // rows of a launch
    for (int64_t n = 0; n < g.N; n += most) {
        const dim3 grid((unsigned)((g.M + 1023) / 1024), (unsigned)(g.N - n < most ? g.N - n : most));
        hipLaunchKernelGGL(mx4_join_kernel<XT>, grid, dim3(256), 0, st, g, n);
        const int code = hip_status(hipGetLastError());
        if (code != BS_OK) return code;
    }
    return BS_OK;
}

// Kinds of tiles go by their rows of y, but for the second one of 128 x 128, which has four stages in LDS.
constexpr int kFourStages = 127;

template <typename XT>
int launch_tiles(const Mx4Tiles& t, int kind, hipStream_t st) {
    switch (kind) {
        case 32: return launch_tiles<XT, 32, 128, 1, 4, 4>(t, st);
        case 64: return launch_tiles<XT, 64, 128, 1, 4, 4>(t, st);
        case 96: return launch_tiles<XT, 96, 128, 1, 4, 4>(t, st);
        case kFourStages: return launch_tiles<XT, 128, 128, 2, 2, 4>(t, st);
        case 128: return launch_tiles<XT, 128, 128, 2, 2, 2>(t, st);
        default: return launch_tiles<XT, 256, 256, 2, 2, 2>(t, st);
    }
}

// ---- which

struct Plan {
    int tile;                      // kind of tiles; 0: none
    int split, stages;             // workgroups that share K, and the stages of 256 columns of each
    int r, nt, ways, groups;       // without tiles
};

// What a product takes, in microseconds, as far as it takes to choose.  A round of tiles, `fit` for a compute unit, takes `begin` and for
// each stage `full`, or `alone` where a compute unit has one; fitted to 300 x 600, 1024 x 1024, 4096 x 4096, 10000 x 1500, 32003 x 1500,
// 4096 x 25088 and 16384 x 8192 for 16 to 4096 rows of x, which it meets within a quarter.  Large tiles read least for each product;
// small ones leave room for four stages in LDS, and so has a second kind of 128 x 128, which two tiles of a compute unit are better than
// where results count for more than the way to them (32003 x 1500 for 256 rows 13.9 us against 17.7, 16384 x 8192 28.0 against 24.3).
struct Tile {
    int kind, n, m, fit;
    double alone, full, begin;
};
constexpr Tile kTiles[] = {{32, 32, 128, 1, 0.45, 0.45, 2.2}, {64, 64, 128, 1, 0.5, 0.5, 2.8}, {96, 96, 128, 1, 0.56, 0.56, 3.2},
                           {kFourStages, 128, 128, 1, 0.64, 0.64, 3.5}, {128, 128, 128, 2, 0.77, 1.1, 3.0}, {256, 256, 256, 1, 1.75, 1.75, 7.0}};

double matrix_us(int64_t M, int chunks) { return (double)M * chunks * 68 / 4.6e6; }

double tiles_us(const Tile& t, int64_t M, int64_t N, int chunks, int stages, int split) {
    const double groups = (double)((M + t.m - 1) / t.m) * ((N + t.n - 1) / t.n) * split, sums = (double)M * N * 4;
    const double rounds = groups <= 256 ? 1 : (double)(int64_t)((groups + 256 * t.fit - 1) / (256 * t.fit));
    const double work = rounds * (stages * (groups <= 256 ? t.alone : t.full) + t.begin), least = matrix_us(M, chunks);
    return 2 + (work > least ? work : least) + (split > 1 ? 2 + (2 * split + 0.5) * sums / 8e6 : 0);
}

// the same for W straight from memory: every wavefront's steps one after the other, 2048 of them at a time
double rows_us(const Plan& p, int64_t M, int chunks, int steps) {
    const double waves = (double)((M + 16 * p.r - 1) / (16 * p.r)) * p.ways, rounds = waves < 2048 ? 1 : waves / 2048;
    const double work = (steps + p.ways - 1) / p.ways * (1.3 + 0.65 * p.nt) * rounds, least = matrix_us(M, chunks);
    return 2.5 + (work > least ? work : least);
}

// Whether every workgroup rounds x for itself, which spares a kernel of 3 us: a piece of a thread takes .8 us, in every round of
// workgroups (10000 x 1500 for 4 rows, 3 pieces, 6.1 us instead of 8.2, for 8 rows, 6 pieces, 8.4 and 8.5, for 16 13.0 and 8.1;
// 32306 x 651 for 12 rows 6.9 and 9.0, 200000 x 500 for 5 17.3 and 16.6).
bool fused(const Plan& p, int64_t M, int64_t K, int64_t N) {
    if (p.tile || p.r * p.nt > 1 || N * 68 * (mx4_chunks(K) + 3) > kFusedBytes) return false;
    const int64_t threads = 64 * p.ways * p.groups, pieces = (N * 16 * mx4_chunks(K) + threads - 1) / threads;
    return N <= kFusedRows || (pieces <= 5 && pieces * ((M + 16 * p.groups - 1) / (16 * p.groups)) <= 3200);
}

Plan plan_for(int64_t M, int64_t K, int64_t N) {
    const int chunks = (int)mx4_chunks(K), steps = (chunks + kStep - 1) / kStep, stages = (chunks + 1) / 2;
    const int64_t tiles = (M + 15) / 16;
    Plan p{};
    double least = 0;
    if (N <= 64) {
        p.nt = N <= 16 ? 1 : N <= 32 ? 2 : 4;
        // Wavefronts that share K: as many as give the chip 2048 (eight for a compute unit), or what K has steps for; where two are
        // enough, four groups of them share x in LDS.  16384 x 8192 for one row: 17.1 us with 2 x 4, 18.9 with 1 x 4, 17.8 with
        // 4 x 2, 18.3 with 8 x 1.  With more rows x is what counts: twice as many rows of W for each of its pieces, 14.5 us instead
        // of 16.0 for 4 rows and 17.0 instead of 20.9 for 16.
        p.r = N > kFusedRows && N <= 16 && tiles >= 1024 && steps >= 8 ? 2 : 1;
        p.ways = 1;
        const int most = p.nt * p.r > 1 ? 8 : 16;      // wavefronts of a workgroup
        while (p.ways < most && tiles * p.ways < 2048 * p.r && p.ways < steps) p.ways *= 2;
        p.groups = p.ways <= 2 ? 4 : p.r == 2 ? 2 : 1;
        least = rows_us(p, M, chunks, steps);
        if (N <= kFusedRows || fused(p, M, K, N)) return p;
    }
    for (const Tile& t : kTiles)
        for (int split = 1; split <= 16 && split <= stages; ++split) {
            const int each = (stages + split - 1) / split;
            if ((stages + each - 1) / each != split) continue;
            if (split > 1 && ((M + t.m - 1) / t.m) * ((N + t.n - 1) / t.n) * split > 1024) break;      // enough for the chip before
            const double cost = tiles_us(t, M, N, chunks, each, split);
            if (least && cost >= least) continue;
            least = cost;
            p.tile = t.kind;
            p.split = split;
            p.stages = each;
        }
    return p;
}

size_t packed_bytes(int64_t K, int64_t N) { return (size_t)(N * (mx4_row_bytes(K) + mx4_scale_pitch(K)) + 15) / 16 * 16; }

template <typename XT>
int launch(Args g, const Plan& p, float* sums, hipStream_t st) {
    if (p.tile) {
        Mx4Tiles t{};
        t.codes = g.codes; t.scales = g.scales; t.x_codes = g.x_codes; t.x_scales = g.x_scales;
        t.M = g.M; t.N = g.N; t.chunks = g.chunks; t.bias = g.bias; t.y = g.y; t.ldy = g.ldy;
        t.split = p.split; t.stages = p.stages; t.sums = sums;
        return launch_tiles<XT>(t, p.tile, st);
    }
    g.ways = p.ways;
    g.tiles = p.groups;
    if (g.x) return launch_rows<XT, 1, 1, true>(g, st);
    if (p.r == 2) return launch_rows<XT, 2, 1, false>(g, st);
    return p.nt == 1 ? launch_rows<XT, 1, 1, false>(g, st) : p.nt == 2 ? launch_rows<XT, 1, 2, false>(g, st) : launch_rows<XT, 1, 4, false>(g, st);
}

}  // namespace

void mx4_gemm_plan_describe(int64_t M, int64_t K, int64_t N, int64_t* out, int n_out) {
    const Plan p = plan_for(M, K, N);
    int64_t v[11] = {};
    if (p.tile) {
        for (const Tile& t : kTiles) {
            if (t.kind != p.tile) continue;
            v[0] = t.n, v[1] = t.m, v[2] = t.fit == 1 && t.n < 256 ? 4 : 2;
            v[9] = ((M + t.m - 1) / t.m) * ((N + t.n - 1) / t.n) * p.split;
            v[10] = (t.n + t.m) * (128 * v[2] + 2 * 8 * kMx4Group);
        }
        v[3] = p.split, v[4] = p.stages;
    } else {
        v[5] = p.r, v[6] = p.nt, v[7] = p.ways, v[8] = p.groups;
        const int64_t rows = 16 * p.r * p.groups, sums = (int64_t)p.ways * p.groups * p.r * p.nt * 1024,
                      x = fused(p, M, K, N) ? N * (64 * mx4_chunks(K) + 4 * ((mx4_chunks(K) + 3) & ~(int64_t)3)) : 0;
        v[9] = (M + rows - 1) / rows;
        v[10] = sums > x ? sums : x;
    }
    for (int i = 0; i < n_out && i < 11; ++i) out[i] = v[i];
}

static size_t workspace_of(const Plan& p, bool packed, int64_t M, int64_t K, int64_t N) {
    return (packed || fused(p, M, K, N) ? 0 : packed_bytes(K, N)) + (p.split > 1 ? (size_t)p.split * M * N * 4 : 0);
}
size_t mx4_gemm_workspace_bytes(bool packed, int64_t M, int64_t K, int64_t N) {
    return workspace_of(plan_for(M, K, N), packed, M, K, N);
}

int launch_mx4_gemm(const uint8_t* codes, const uint8_t* scales, int64_t M, int64_t K, const void* x, int64_t ldx, const uint8_t* x_codes,
                    const uint8_t* x_scales, int dtype, int64_t N, const float* bias, void* y, int64_t ldy, void* workspace,
                    size_t workspace_bytes, hipStream_t st) {
    const Plan p = plan_for(M, K, N);
    const size_t need = workspace_of(p, !x, M, K, N);
    if (need && (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 15))) return BS_ERR_WORKSPACE;
    // y over what workgroups read while others store
    const Rows out(y, N, M, ldy, dtype_bytes(dtype));
    if (rows_meet(mx4_codes_place(codes, M, K), out) || rows_meet(mx4_scales_place(scales, M, K), out) ||
        (bias && rows_meet(Rows(bias, 1, M, 0, 4), out)) ||
        (!x && (rows_meet(mx4_codes_place(x_codes, N, K), out) || rows_meet(mx4_scales_place(x_scales, N, K), out))))
        return BS_ERR_UNSUPPORTED;
    uint8_t* at = static_cast<uint8_t*>(workspace);
    const bool dense = x && fused(p, M, K, N);
    if (x && !dense) {
        uint8_t* const s = at + N * mx4_row_bytes(K);
        const int rc = launch_mx4_pack(x, dtype, N, K, ldx, at, s, st);
        if (rc != BS_OK) return rc;
        x_codes = at;
        x_scales = s;
        at += packed_bytes(K, N);
    }
    float* const sums = reinterpret_cast<float*>(at);
    const Args g{codes, scales, x_codes, x_scales, dense ? x : nullptr, ldx, M, K, N, magic_u32((uint32_t)(16 * mx4_chunks(K))),
                 (int)mx4_chunks(K), 1, 1, bias, y, ldy};
    switch (dtype) {
        case BS_F32: return launch<F32>(g, p, sums, st);
        case BS_F16: return launch<F16>(g, p, sums, st);
        default: return launch<BF16>(g, p, sums, st);
    }
}

}  // namespace bs

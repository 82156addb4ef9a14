// One step of beam search, and the states that follow it (bs.h: bs_beam_step, bs_beam_reorder).
//
// The step.  Bound: HBM, the logits of the beams that go on once.  What orders the words of one beam are its logits; what orders those
// of different beams is a difference of two sums, which must not depend on how either was rounded, so sums are made in 64 bits: with
// u = (x - m) log2(e), the sum of 2^u by a polynomial of degree 7 between -1/2 and 1/2 (off by 5e-11, and exact at 0: a word that is
// certain has log probability 0), its exponent added to the number's own.  64-bit operations run at the rate of 32-bit ones here, and one exponential is about as many as a 32-bit one takes
// with the transcendental unit's four.  Elements come to threads by their index, wherever a row starts in memory: beams with the same
// logits have the same sums to the last bit, and tie.  A row's n largest are found as bs_logprobs finds them.
// A second kernel joins the rows of a sequence: a candidate's total is scores + ((x - m) - log s); of the lists that are full each
// answers for its share of the n, the least of those totals is a bound, and what reaches it is ordered by counting what comes before.
#include "bs_logits.h"

namespace bs {
namespace {

constexpr int kThreads = kRowThreads, kWaves = kThreads / 64;
constexpr int kBatch = 32;                     // elements of a thread
constexpr int kSlices = 16;                    // of a row, at most
constexpr int kPlaces = 8;                     // in LDS for a thread's batches' largest; more batches share them
constexpr int kParts = kBatch / 8;
constexpr int kWidth = BS_BEAM_WIDTH_MAX;
constexpr int kCandidates = kWidth * kWidth;   // of a sequence, all its lists
constexpr double kLog2e = 1.4426950408889634074;
static_assert(kWidth <= kTopMax);

// 2^u for -1000 < u < 1000, 1 for 0
__device__ __forceinline__ double exp2_wide(double u) {
    constexpr double kMagic = 0x1.8p52;      // the whole part, in the low bits
    const double t = u + kMagic, f = u - (t - kMagic);
    double p = 0x1.fde5fe3497e78p-17;
    p = fma(p, f, 0x1.445c8421d1ed2p-13);
    p = fma(p, f, 0x1.5d8a85ff048c0p-10);
    p = fma(p, f, 0x1.3b29f39d29c2ap-7);
    p = fma(p, f, 0x1.c6b08ac06b2ccp-5);
    p = fma(p, f, 0x1.ebfbe07787485p-3);
    p = fma(p, f, 0x1.62e42ff0e1927p-1);
    p = fma(p, f, 1.0);
    const uint64_t b = __builtin_bit_cast(uint64_t, p);
    const uint32_t high = (uint32_t)(b >> 32) + ((uint32_t)__builtin_bit_cast(uint64_t, t) << 20);
    return __builtin_bit_cast(double, (uint64_t)high << 32 | (uint32_t)b);
}

// the sum of exp(x - m) over some of a row; m is -inf before anything was seen
struct Sum {
    double s;
    float m;
};
__device__ __forceinline__ void raise(Sum& a, float m) {
    if (a.m == m) return;
    const double d = a.m == -__builtin_inff() ? -900.0 : fmax(((double)a.m - (double)m) * kLog2e, -900.0);
    a.s = m == __builtin_inff() ? __builtin_nan("") : a.s * exp2_wide(d);
    a.m = m;
}
__device__ __forceinline__ double moved(double v, int by) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__shfl_xor((int)(uint32_t)b, by, 64), hi = (uint32_t)__shfl_xor((int)(b >> 32), by, 64);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ Sum join_wave(Sum a) {
    raise(a, max_of_wave(a.m));
#pragma unroll
    for (int by = 1; by < 64; by *= 2) a.s += moved(a.s, by);
    return a;
}
__device__ __forceinline__ Sum join(Sum a, Sum b) {
    const float m = fmaxf(a.m, b.m);
    raise(a, m);
    raise(b, m);
    return {a.s + b.s, m};
}

// A row as 16-byte pieces from its first element on, wherever that is in memory
template <typename XT>
struct BeamRow {
    using T = typename XT::type;
    static constexpr int E = 16 / sizeof(T), head = 0;
    const T* p;
    int64_t V;
    __device__ BeamRow(const void* base, int64_t row, int64_t ld, int64_t V_) : p(static_cast<const T*>(base) + row * ld), V(V_) {}
    __device__ __forceinline__ int64_t vectors() const { return (V + E - 1) / E; }
    static __device__ __forceinline__ void values(uint4 a, float* out) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if constexpr (sizeof(T) == 4) out[i] = __builtin_bit_cast(float, word_of(a, i));
            else out[i] = XT::load((uint16_t)(word_of(a, i >> 1) >> (16 * (i & 1))));
        }
    }
    __device__ __forceinline__ void load(int64_t v, float* out) const {
        const int64_t e = v * E;
        if (e + E <= V) {
            uint4 a;
            __builtin_memcpy(&a, p + e, 16);
            values(a, out);
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) out[i] = e + i < V ? XT::load(p[e + i]) : -__builtin_inff();
        }
    }
};

struct Args {
    const void* logits;
    int64_t B, V, ld, rows, end;
    int W, n, slices;
    int64_t slice_vectors;      // 16-byte pieces of a row in a slice
    int sharing, places;        // batches of a place, places of a thread
    const float* scores;
    const uint8_t* finished;
    float* out_scores;
    int32_t *out_tokens, *out_parents;
    uint8_t* out_finished;
    Sum* sums;                  // [rows][slices]
    uint64_t* keys;             // [rows][slices][n]
};

__device__ __forceinline__ bool finite(float v) { return fabsf(v) < __builtin_inff(); }

// THREADS: a workgroup for a row (or a slice of one), or a wavefront
template <typename XT, int THREADS>
__global__ __launch_bounds__(kThreads) void beam_rows_kernel(Args g) {
    using G = Group<THREADS>;
    using R = BeamRow<XT>;
    constexpr int E = R::E, U = kBatch / E, V8 = 8 / E, kRows = kThreads / THREADS;      // pieces of a thread, and of eight elements
    extern __shared__ __align__(16) f32x4 all_largest[];           // [row][place][thread]: of the batches' four eights
    __shared__ TopList lists[kRows];
    __shared__ Sum all_sums[kWaves];
    const int mine = __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS), me = G::thread(), wave = G::wave(), lane = threadIdx.x & 63;
    const int64_t r = kRows > 1 ? (int64_t)blockIdx.x * kRows + mine : blockIdx.x / g.slices, slice = kRows > 1 ? 0 : blockIdx.x % g.slices;
    if (kRows > 1 && r >= g.rows) return;
    if ((g.finished && g.finished[r]) || !finite(g.scores[r])) return;      // all threads of the row; the join looks itself
    TopList& l = lists[mine];
    Sum* const sums = all_sums + mine * G::kWaves;
    f32x4* const largest = all_largest + mine * g.places * THREADS;
    const R row(g.logits, r, g.ld, g.V);
    const int64_t v0 = slice * g.slice_vectors, v1 = min(row.vectors(), v0 + g.slice_vectors);
    if (me == 0) l.count = l.eight_count = 0;
    Sum st{0.0, -__builtin_inff()};
    int batches = 0;
    for (int64_t b = v0; b < v1; b += THREADS * U, ++batches) {
        float x[kBatch];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t v = b + u * THREADS + me;
            if (v < v1) row.load(v, x + u * E);
            else
#pragma unroll
                for (int i = 0; i < E; ++i) x[u * E + i] = -__builtin_inff();
        }
        float part[kParts], most = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            part[i] = x[8 * i];
#pragma unroll
            for (int j = 1; j < 8; ++j) part[i] = fmaxf(part[i], x[8 * i + j]);
            most = fmaxf(most, part[i]);
        }
        f32x4& place = largest[batches / g.sharing * THREADS + me];
        if (batches % g.sharing) {
#pragma unroll
            for (int i = 0; i < kParts; ++i) part[i] = fmaxf(part[i], place[i]);
        }
        place = f32x4{part[0], part[1], part[2], part[3]};
        if (most > st.m) raise(st, most);
        // Differences are at least -600, where the exponential counts for nothing.  Far from 0 they are taken in fp32, where they are
        // exact or beyond that; else in 64 bits.
        const bool none = st.m == -__builtin_inff(), far = !(fabsf(st.m) <= 0x1p20f);
        const double m = none || far ? 0.0 : (double)st.m;
        if (far && !none) {
#pragma unroll
            for (int i = 0; i < kBatch; ++i) x[i] -= st.m;
        }
        const float least = none || far ? -600.f : st.m - 600.f;
        double s0 = 0.0, s1 = 0.0;
#pragma unroll
        for (int j = 0; j < kParts; ++j) {
            if (b + j * V8 * THREADS >= v1) break;      // no thread has more
#pragma unroll
            for (int i = 8 * j; i < 8 * j + 8; i += 2) {
                s0 += exp2_wide(((double)__builtin_elementwise_maximum(x[i], least) - m) * kLog2e);
                s1 += exp2_wide(((double)__builtin_elementwise_maximum(x[i + 1], least) - m) * kLog2e);
            }
        }
        st.s += s0 + s1;
    }
    G::sync();
    const int with_words = __popcll(__ballot(st.m > -__builtin_inff()));
    if (lane == 0) l.wave_count[wave] = with_words;
    G::sync();
    // of the n, every wavefront answers for its share of the lanes that have words
    int here = l.wave_count[wave], lanes = 0;
    for (int w = 0; w < G::kWaves; ++w) lanes += l.wave_count[w];
    const int k = lanes < g.n ? -1 : (g.n * here + lanes - 1) / lanes;
    const float bound_here = k < 0 ? -__builtin_inff() : k ? kth_largest(st.m, k) : __builtin_inff();
    if (lane == 0) l.bound[wave] = bound_here;
    st = join_wave(st);
    if (lane == 0) sums[wave] = st;
    G::sync();
    float bound = l.bound[0];
    for (int w = 1; w < G::kWaves; ++w) bound = fminf(bound, l.bound[w]);
    for (int b = 0; b * g.sharing < batches; ++b) {
        const f32x4 part = largest[b * THREADS + me];
#pragma unroll
        for (int i = 0; i < kParts; ++i)
            if (part[i] >= bound && part[i] > -__builtin_inff()) {
                const int at = atomicAdd(&l.eight_count, 1);
                if (at < kEights) l.eights[at] = (uint32_t)(b * kParts + i) * THREADS + me;
            }
    }
    G::sync();
    const int eights = l.eight_count;
    const int64_t pieces = (int64_t)min(eights, kEights) * V8 * g.sharing;
    for (int64_t j = me; j < pieces; j += THREADS) {
        const uint32_t eight = l.eights[j / (V8 * g.sharing)], place = eight / THREADS;
        const int64_t batch = place / kParts * (int64_t)g.sharing + j / V8 % g.sharing;
        const int64_t v = v0 + (batch * U + place % kParts * V8 + j % V8) * THREADS + eight % THREADS;
        float x[E];
        if (v < v1) row.load(v, x);
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (v < v1 && x[i] >= bound && x[i] > -__builtin_inff()) {
                const int at = atomicAdd(&l.count, 1);
                if (at < kList) l.keys[at] = order_key(x[i], (uint32_t)(v * E + i));
            }
    }
    if (me == THREADS - 64) {      // meanwhile
        Sum all = sums[0];
        for (int w = 1; w < G::kWaves; ++w) all = join(all, sums[w]);
        g.sums[r * g.slices + slice] = all;
    }
    G::sync();
    const int count = l.count;
    if (eights > kEights || count > kList)
        flooded<THREADS>(l, row, v0, v1, bound, g.n, reinterpret_cast<uint64_t*>(largest), (batches + g.sharing - 1) / g.sharing * (THREADS * 2));
    else order_list<THREADS>(l, count, g.n);
    // a slice can have fewer words than n that are larger than its bound
    if (bound > -__builtin_inff() && !l.sorted[g.n - 1]) fill<THREADS>(l, row, v0, v1, bound, g.n);
    for (int i = me; i < g.n; i += THREADS) g.keys[(r * g.slices + slice) * g.n + i] = l.sorted[i];
}

// a sequence's n best of what its lists (one for each beam and slice) offer
__global__ __launch_bounds__(kThreads) void beam_join_kernel(Args g) {
    __shared__ double totals[kCandidates], bounds[kWidth * kSlices];
    __shared__ uint16_t from[kCandidates];
    __shared__ double log_s[kWidth];
    __shared__ float most[kWidth];
    __shared__ int kind[kWidth], kept, full;      // kind of a beam: 0 offers nothing, 1 goes on, 2 is finished
    const int64_t b = blockIdx.x;
    const int lists = g.W * g.slices, all = lists * g.n;
    const uint64_t* const keys = g.keys + b * all;
    if (threadIdx.x == 0) kept = full = 0;
    if ((int)threadIdx.x < g.W) {
        const int64_t r = b * g.W + threadIdx.x;
        int is = finite(g.scores[r]) ? g.finished && g.finished[r] ? 2 : 1 : 0;
        if (is == 1) {
            Sum st = g.sums[r * g.slices];
            for (int i = 1; i < g.slices; ++i) st = join(st, g.sums[r * g.slices + i]);
            log_s[threadIdx.x] = log(st.s);
            most[threadIdx.x] = st.m;
            if (!(st.s > 0.0)) is = 0;      // no words, or a logit that is NaN or +inf
        }
        kind[threadIdx.x] = is;
    }
    __syncthreads();
    // the total of candidate i, the one of place i % n in list i / n; -inf for what is none
    const auto total_of = [&](int i) {
        const int list = i / g.n, beam = list / g.slices, rank = i - list * g.n;
        const double score = (double)g.scores[b * g.W + beam];
        if (kind[beam] == 2) return rank == 0 && list % g.slices == 0 ? score : -(double)__builtin_inff();
        if (kind[beam] == 0) return -(double)__builtin_inff();
        const uint64_t key = keys[i];
        const float x = value_of_key(key);
        if (!key || x == -__builtin_inff()) return -(double)__builtin_inff();
        return score + (((double)x - (double)most[beam]) - log_s[beam]);
    };
    for (int i = threadIdx.x; i < lists; i += kThreads)
        if (total_of(i * g.n + g.n - 1) > -(double)__builtin_inff()) atomicAdd(&full, 1);
    __syncthreads();
    // every full list answers for its share of the n
    const int share = full ? (g.n + full - 1) / full : 0;
    for (int i = threadIdx.x; i < lists; i += kThreads)
        bounds[i] = full && total_of(i * g.n + g.n - 1) > -(double)__builtin_inff() ? total_of(i * g.n + share - 1) : (double)__builtin_inff();
    __syncthreads();
    double bound = (double)__builtin_inff();
    for (int i = 0; i < lists; ++i) bound = fmin(bound, bounds[i]);
    if (!full) bound = -(double)__builtin_inff();
    for (int i = threadIdx.x; i < all; i += kThreads) {
        const double t = total_of(i);
        if (t >= bound && t > -(double)__builtin_inff()) {
            const int at = atomicAdd(&kept, 1);
            totals[at] = t;
            from[at] = (uint16_t)i;
        }
    }
    __syncthreads();
    const int count = kept;
    for (int c = threadIdx.x; c < count; c += kThreads) {
        const double t = totals[c];
        const int i = from[c], list = i / g.n, beam = list / g.slices;
        int before = 0;
        for (int j = 0; j < count; ++j) {
            if (totals[j] != t) {
                before += totals[j] > t;
                continue;
            }
            // equals: the lower beam, then the beam's own order
            const int other = from[j], other_list = other / g.n;
            if (other_list == list || other_list / g.slices != beam) before += other < i;
            else before += keys[other] > keys[i];
        }
        if (before >= g.n) continue;
        const bool done = kind[beam] == 2;
        const int64_t token = done ? (g.end < 0 ? 0 : g.end) : (int64_t)index_of_key(keys[i]);
        const int64_t to = b * g.n + before;
        g.out_scores[to] = (float)t;
        g.out_tokens[to] = (int32_t)token;
        g.out_parents[to] = beam;
        g.out_finished[to] = done || token == g.end;
    }
    for (int j = count + threadIdx.x; j < g.n; j += kThreads) {
        const int64_t to = b * g.n + j;
        g.out_scores[to] = -__builtin_inff();
        g.out_tokens[to] = (int32_t)(g.end < 0 ? 0 : g.end);
        g.out_parents[to] = min(j, g.W - 1);
        g.out_finished[to] = 1;
    }
}

struct Plan {
    bool waves;
    int slices;
    int64_t slice_vectors;
};

Plan plan_for(int dtype, int64_t rows, int W, int64_t V, int n) {
    const int E = 16 / dtype_bytes(dtype);
    const int64_t vectors = (V + E - 1) / E, batch = (int64_t)kThreads * (kBatch / E);
    if (V <= 16384 && rows >= (V <= 2048 ? 1024 : 2048)) return {true, 1, vectors};
    // all lists of a sequence are joined by one workgroup, kCandidates at most
    const int64_t most = kCandidates / ((int64_t)W * n) < kSlices ? kCandidates / ((int64_t)W * n) : kSlices;
    int64_t slices = 1;
    if (vectors >= 2 * batch)
        while (slices * 2 <= most && rows * slices < 512 && vectors / (slices * 2) >= kThreads) slices *= 2;
    Plan p{false, 1, (vectors + slices - 1) / slices};
    p.slices = (int)((vectors + p.slice_vectors - 1) / p.slice_vectors);
    return p;
}

size_t sums_bytes(int64_t rows, const Plan& p) { return (size_t)rows * p.slices * sizeof(Sum); }

template <typename XT, int THREADS>
int launch_rows(Args g, hipStream_t st) {
    constexpr int kRows = kThreads / THREADS, per = THREADS * (kBatch / BeamRow<XT>::E);
    const int64_t batches = (g.slice_vectors + per - 1) / per;
    g.sharing = (int)((batches + kPlaces - 1) / kPlaces);
    g.places = (int)((batches + g.sharing - 1) / g.sharing);
    hipLaunchKernelGGL((beam_rows_kernel<XT, THREADS>), dim3((unsigned)((g.rows * g.slices + kRows - 1) / kRows)), dim3(kThreads),
                       (size_t)g.places * kThreads * sizeof(f32x4), st, g);
    return hip_status(hipGetLastError());
}

template <typename XT>
int launch(Args all, bool waves, hipStream_t st) {
    // sequences of a launch: a grid has fewer than 2^32 lanes
    const int64_t most = ((int64_t)1 << 23) / (all.W * all.slices);
    for (int64_t b = 0; b < all.B; b += most) {
        Args g = all;
        g.B = all.B - b < most ? all.B - b : most;
        g.rows = g.B * g.W;
        const int64_t row = b * g.W, out = b * g.n;
        g.logits = static_cast<const typename XT::type*>(all.logits) + row * g.ld;
        g.scores += row;
        if (g.finished) g.finished += row;
        g.sums += row * g.slices;
        g.keys += row * g.slices * g.n;
        g.out_scores += out; g.out_tokens += out; g.out_parents += out; g.out_finished += out;
        int rc = waves ? launch_rows<XT, 64>(g, st) : launch_rows<XT, kThreads>(g, st);
        if (rc != BS_OK) return rc;
        hipLaunchKernelGGL(beam_join_kernel, dim3((unsigned)g.B), dim3(kThreads), 0, st, g);
        rc = hip_status(hipGetLastError());
        if (rc != BS_OK) return rc;
    }
    return BS_OK;
}

// ---- states

constexpr int kStates = BS_REORDER_STATES_MAX;
struct State {
    const char* in;
    char* out;
    int64_t pitch, out_pitch;
    int32_t bytes, word;        // of a row; of a move: 16, 4 or 1, all rows being that much apart and as aligned
    uint32_t first;             // workgroup, of those of a sequence
};
struct States {
    State s[kStates];
    int count;
    uint32_t groups;            // workgroups of a sequence
};

// A workgroup has some columns of all of a sequence's rows: every lane reads a word of each row before any is written, so a row may be
// overwritten by another's.
template <typename T, int ROWS>
__device__ __forceinline__ void move_rows(const State& s, int64_t row0, int W, uint32_t at, const int* parents) {
    T v[ROWS];
    const bool mine = at < (uint32_t)s.bytes;
#pragma unroll
    for (int j = 0; j < ROWS; ++j)
        if (mine && j < W) v[j] = *reinterpret_cast<const T*>(s.in + (row0 + parents[j]) * s.pitch + at);
#pragma unroll
    for (int j = 0; j < ROWS; ++j)
        if (mine && j < W && !(parents[j] == j && s.in == s.out)) *reinterpret_cast<T*>(s.out + (row0 + j) * s.out_pitch + at) = v[j];
}

template <int ROWS>
__global__ __launch_bounds__(256) void beam_reorder_kernel(States all, int W, const int32_t* parents) {
    __shared__ int parent[kWidth];
    const uint32_t b = blockIdx.x / all.groups, group = blockIdx.x % all.groups;
    if ((int)threadIdx.x < ROWS) {
        const int p = (int)threadIdx.x < W ? parents[(int64_t)b * W + threadIdx.x] : 0;
        parent[threadIdx.x] = p >= 0 && p < W ? p : (int)threadIdx.x;
    }
    int i = 0;
    while (i + 1 < all.count && group >= all.s[i + 1].first) ++i;
    const State& s = all.s[i];
    __syncthreads();
    const int64_t row0 = (int64_t)b * W;
    const uint32_t at = ((group - s.first) * 256 + threadIdx.x) * (uint32_t)s.word;
    if (s.word == 16) move_rows<uint4, ROWS>(s, row0, W, at, parent);
    else if (s.word == 4) move_rows<uint32_t, ROWS>(s, row0, W, at, parent);
    else move_rows<uint8_t, ROWS>(s, row0, W, at, parent);
}

}  // namespace

size_t beam_step_workspace_bytes(int dtype, int64_t B, int W, int64_t V, int n) {
    const Plan p = plan_for(dtype, B * W, W, V, n);
    return sums_bytes(B * W, p) + (size_t)B * W * p.slices * n * 8;
}

int launch_beam_step(const void* logits, int dtype, int64_t B, int W, int64_t V, int64_t ld, const float* scores, const uint8_t* finished,
                     int64_t end, int n, float* out_scores, int32_t* out_tokens, int32_t* out_parents, uint8_t* out_finished,
                     void* workspace, size_t workspace_bytes, hipStream_t st) {
    const size_t need = beam_step_workspace_bytes(dtype, B, W, V, n);
    if (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 15)) return BS_ERR_WORKSPACE;
    const Plan p = plan_for(dtype, B * W, W, V, n);
    Args g{};
    g.logits = logits; g.B = B; g.V = V; g.ld = ld; g.end = end; g.W = W; g.n = n;
    g.slices = p.slices; g.slice_vectors = p.slice_vectors;
    g.scores = scores; g.finished = finished;
    g.out_scores = out_scores; g.out_tokens = out_tokens; g.out_parents = out_parents; g.out_finished = out_finished;
    g.sums = static_cast<Sum*>(workspace);
    g.keys = reinterpret_cast<uint64_t*>(static_cast<char*>(workspace) + sums_bytes(B * W, p));
    switch (dtype) {
        case BS_F32: return launch<F32>(g, p.waves, st);
        case BS_F16: return launch<F16>(g, p.waves, st);
        default: return launch<BF16>(g, p.waves, st);
    }
}

int launch_beam_reorder(int count, const void* const* states, void* const* outs, const int64_t* row_bytes, const int64_t* pitch,
                        const int64_t* out_pitch, int64_t B, int W, const int32_t* parents, hipStream_t st) {
    States all{};
    all.count = count;
    uint64_t groups = 0;
    for (int i = 0; i < count; ++i) {
        State& s = all.s[i];
        s.in = static_cast<const char*>(states[i]);
        s.out = static_cast<char*>(outs[i]);
        s.pitch = pitch[i];
        s.out_pitch = out_pitch[i];
        s.bytes = (int32_t)row_bytes[i];
        const uint64_t bits = reinterpret_cast<uintptr_t>(states[i]) | reinterpret_cast<uintptr_t>(outs[i]) | (uint64_t)pitch[i] |
                              (uint64_t)out_pitch[i] | (uint64_t)row_bytes[i];
        s.word = bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : 1;
        s.first = (uint32_t)groups;
        groups += ((uint64_t)row_bytes[i] + 256 * s.word - 1) / (256 * s.word);
    }
    all.groups = (uint32_t)groups;
    // sequences of a launch: a grid has fewer than 2^32 lanes
    const int64_t most = ((int64_t)1 << 23) / (int64_t)groups > 1 ? ((int64_t)1 << 23) / (int64_t)groups : 1;
    for (int64_t b = 0; b < B; b += most) {
        const unsigned grid = (unsigned)((B - b < most ? B - b : most) * (int64_t)groups);
        if (W <= 4) hipLaunchKernelGGL(beam_reorder_kernel<4>, dim3(grid), dim3(256), 0, st, all, W, parents + b * W);
        else if (W <= 16) hipLaunchKernelGGL(beam_reorder_kernel<16>, dim3(grid), dim3(256), 0, st, all, W, parents + b * W);
        else hipLaunchKernelGGL(beam_reorder_kernel<64>, dim3(grid), dim3(256), 0, st, all, W, parents + b * W);
        const int rc = hip_status(hipGetLastError());
        if (rc != BS_OK) return rc;
        for (int i = 0; i < count; ++i) {
            all.s[i].in += most * W * all.s[i].pitch;
            all.s[i].out += most * W * all.s[i].out_pitch;
        }
    }
    return BS_OK;
}

}  // namespace bs

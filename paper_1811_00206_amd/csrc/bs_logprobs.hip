// Log probabilities of given tokens, entropy and most likely alternatives of rows of logits, and their gradient
// (bs.h: bs_logprobs, bs_logprobs_backward).  Bound: HBM, the logits once (the gradient: once in, once out).
//
// Softmax statistics in one pass: a thread keeps the largest logit m it has seen and, with L = log2(e) and u = x L - c,
// c = m L rounded,
//     s = sum 2^u,   t = sum u 2^u,   so that  lse = ln2 (c + log2 s)  and  entropy = ln2 (log2 s - t / s):
// c's rounding is no error, since c itself goes into the result.  A batch of 32 elements moves m once.  u is cut off at
// -200, where 2^u is 0: a banned word, x = -inf, adds nothing to either sum (and no 0 * inf), and what is no number stays
// so.  Where c's rounding would be a large exponent (masks of -1e9 or of the type's lowest value that leave nothing, where m L
// could overflow too) u = (x - m) L and lse = m + log s.
//
// The n largest: each of the four wavefronts finds the k-th largest of its lanes' largest, k being its share of n (a quarter,
// where all lanes have words), and at least n elements reach the least of those, the bound; few others do.  While the
// statistics are made a thread only keeps, in LDS, the largest of every eight elements; the eights that reach the bound are
// listed and loaded once more, each by a thread of its own, and their elements that reach it are ordered by counting, for every
// one, those before it.  They are 64-bit keys (value, then index), all different, so the order in which threads reach a list
// does not matter.  Rows that flood the lists (masks that leave fewer than n words, equal logits) are gone over once more with
// the strict bound, or n times, which is slow and right.
//
// Measured: 4096 rows of 32003 bfloat16 logits with the 5 largest in 59 us (4.4 TB/s; 45 at the rate of reads), 56 without
// alternatives.  The vector ALU is busy about 40 us of it (conversion, maximum, two for u, an exponential of four, two sums, and two
// of loads and copies, an element); eight wavefronts a SIMD instead of seven, and no checks of edges inside a row, changed
// nothing.  One row of 131072 fp32 logits, a batch for every thread of 16 workgroups: 4.8 us, and 2.2 to join them; with the 20
// largest 8.1 and 4.8.  The gradient of 4096 x 32003: 106 us, 102 at the rate of a copy.
#include "bs_q4.h"

namespace bs {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kBatch = 32;                     // elements of a thread
constexpr int kSlices = 16;                    // of a row, at most
constexpr int kList = 256;                     // keys in LDS
constexpr int kEights = 256;                   // listed eights
constexpr int kPlaces = 8;                     // in LDS for a thread's batches' largest; more batches share them
constexpr int kParts = kBatch / 8;
constexpr int kTopMax = BS_LOGPROBS_TOP_MAX;
constexpr float kLog2e = 1.44269504088896340736f;

struct Stats {
    float m, s, t;      // m: -inf before anything was seen
};

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
// u, at least `least`; NaN where u is
__device__ __forceinline__ float at_least(float u, float least) { return __builtin_elementwise_maximum(u, least); }
// m so large that the rounding of m * log2(e) counts, 1/16 here (or no number): differences are taken first then
__device__ __forceinline__ bool extreme(float m) { return !(fabsf(m) <= 0x1p20f); }

// the power of two by which sums made with `from` are multiplied to go with `to` >= from, as an exponent
__device__ __forceinline__ float exponent(float from, float to) {
#pragma clang fp contract(off)      // products rounded where the sums are made with rounded ones
    const float f = from * kLog2e, t = to * kLog2e;
    const bool exact = extreme(to);
    const float d = extreme(from) ? (exact ? (from - to) * kLog2e : fmaf(from, kLog2e, -t)) : exact ? -fmaf(to, kLog2e, -f) : f - t;
    return from == to ? 0.f : at_least(d, -200.f);
}
__device__ __forceinline__ void raise(Stats& a, float m) {
    const float d = exponent(a.m, m), f = exp2_hw(d);
    a.t = fmaf(a.s, d, a.t) * f;
    a.s *= f;
    a.m = m;
}

__device__ __forceinline__ Stats join(Stats a, Stats b) {
    const float m = fmaxf(a.m, b.m);
    raise(a, m);
    raise(b, m);
    return {m, a.s + b.s, a.t + b.t};
}
__device__ __forceinline__ Stats join_wave(Stats a) {
    raise(a, max_of_wave(a.m));
    return {a.m, sum_of_wave(a.s), sum_of_wave(a.t)};
}

struct Args {
    const void* logits;
    int64_t T, V, ld, first_row;
    const int64_t* targets;
    int n, slices;
    int64_t slice_vectors;      // 16-byte pieces of a row in a slice
    int sharing, places;        // batches of a place, places of a thread
    float *logprob, *entropy, *lse, *top_values;
    int32_t* top_ids;
    Stats* part_stats;          // [rows][slices]
    uint64_t* part_keys;        // [rows][slices][n]
};

// A row as 16-byte pieces on 16-byte boundaries: piece v has the elements v * E - head .. + E - 1 of the row; those
// before or behind the row are -inf here and nowhere looked at.
template <typename XT>
struct Row {
    using T = typename XT::type;
    static constexpr int E = 16 / sizeof(T);
    const T* p;
    int64_t V;
    int head;
    __device__ Row(const void* base, int64_t row, int64_t ld, int64_t V_) : p(static_cast<const T*>(base) + row * ld), V(V_) {
        head = (int)((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
    }
    __device__ __forceinline__ int64_t vectors() const { return (V + head + E - 1) / E; }
    // Piece v as it lies in memory, if it is one of the whole ones, first .. last; else one of those
    __device__ __forceinline__ int first() const { return head ? 1 : 0; }
    __device__ __forceinline__ int last() const { return (int)((V + head) / E) - 1; }
    __device__ __forceinline__ uint4 raw(int v) const { return reinterpret_cast<const uint4*>(p - head)[min(max(v, first()), last())]; }
    // a piece that is not whole, -inf where it has no elements
    __device__ __forceinline__ uint4 edge(int64_t v) const {
        const int64_t e = v * E - head;
        T out[E];
#pragma unroll
        for (int i = 0; i < E; ++i) out[i] = e + i >= 0 && e + i < V ? p[e + i] : XT::store(-__builtin_inff());
        uint4 a;
        __builtin_memcpy(&a, out, 16);
        return a;
    }
    static __device__ __forceinline__ void values(uint4 a, float* out) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            if constexpr (sizeof(T) == 4) out[i] = __builtin_bit_cast(float, word_of(a, i));
            else out[i] = XT::load((uint16_t)(word_of(a, i >> 1) >> (16 * (i & 1))));
        }
    }
    __device__ __forceinline__ void load(int64_t v, float* out) const {
        const int64_t e = v * E - head;
        if (e >= 0 && e + E <= V) {
            values(*reinterpret_cast<const uint4*>(p + e), out);
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) out[i] = e + i >= 0 && e + i < V ? XT::load(p[e + i]) : -__builtin_inff();
        }
    }
};

// The threads of a row: a workgroup, or a wavefront of one
template <int THREADS>
struct Group {
    static constexpr int kWaves = THREADS / 64;
    static __device__ __forceinline__ int thread() { return threadIdx.x % THREADS; }
    static __device__ __forceinline__ int wave() { return thread() >> 6; }
    static __device__ __forceinline__ void sync() {
        if constexpr (THREADS == kThreads) __syncthreads();
        else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // LDS serves a wavefront in order
    }
};

template <int LIST>
struct KeyList {
    alignas(16) uint64_t keys[LIST + 8];
    uint64_t sorted[kTopMax];
    int count;
};
struct TopList : KeyList<kList> {
    uint32_t eights[kEights];      // first piece of the eight elements
    float bound[kWaves];
    int eight_count, wave_count[kWaves];
    uint64_t wave_best[kWaves];
};

// how many of the first `count` keys, a multiple of eight, are larger
__device__ __forceinline__ int keys_before(const uint64_t* keys, int count, uint64_t key) {
    int before = 0;
    for (int j = 0; j < count; j += 8) {
        uint64_t k[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) k[i] = keys[j + i];
#pragma unroll
        for (int i = 0; i < 8; ++i) before += k[i] > key;
    }
    return before;
}

// the n largest keys of the list, in order; entries behind the list's end become 0.  All threads, barriers inside.
template <int THREADS, int LIST>
__device__ __forceinline__ void order_list(KeyList<LIST>& l, int count, int n) {
    using G = Group<THREADS>;
    const int me = G::thread();
    for (int i = me; i < n; i += THREADS)
        if (i >= count) l.sorted[i] = 0;
    const int padded = (count + 7) & ~7;       // the walk below takes eight at a time
    if (me < 8 && count + me < padded) l.keys[count + me] = 0;
    G::sync();
    for (int i = me; i < count; i += THREADS) {
        const uint64_t key = l.keys[i];
        const int before = keys_before(l.keys, padded, key);
        if (before < n) l.sorted[before] = key;
    }
    G::sync();
}

// the k-th largest of the lanes' values.  One after the other is about 100 cycles each, all ranks at once 800.
__device__ __forceinline__ float kth_largest(float v, int k) {
    float most = v;
    if (k > 8) {
        const int lane = threadIdx.x & 63;
        int rank = 0;
#pragma unroll
        for (int j = 0; j < 64; ++j) {
            const float other = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), j));
            rank += other > v || (other == v && j < lane);
        }
        const int at = __ffsll((unsigned long long)__ballot(rank == k - 1)) - 1;
        return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), __builtin_amdgcn_readfirstlane(at)));
    }
    for (int j = 0; j < k; ++j) {
        most = max_of_wave(v);
        const uint64_t m = __ballot(v == most);
        if ((int)(threadIdx.x & 63) == __ffsll((unsigned long long)m) - 1) v = -__builtin_inff();
    }
    return most;
}

// how many of the list's keys are not below `least`; all threads
template <int THREADS>
__device__ __forceinline__ int keys_from(TopList& l, const uint64_t* keys, int count, uint64_t least) {
    const int me = Group<THREADS>::thread();
    int n = 0;
    for (int i = me; i < (count + 63) / 64 * 64; i += THREADS) n += __popcll(__ballot(i < count && keys[i] >= least));
    if ((me & 63) == 0) l.wave_count[me >> 6] = n;
    Group<THREADS>::sync();
    n = 0;
    for (int w = 0; w < Group<THREADS>::kWaves; ++w) n += l.wave_count[w];
    Group<THREADS>::sync();
    return n;
}

// The list flooded.  First what is larger than the bound, into the room of the eights' largest (`most` keys), out of which the
// n-th largest key is found bit by bit; if that is too many too, the n largest one after the other.
template <typename XT, int THREADS>
__device__ void flooded(TopList& l, const Row<XT>& row, int64_t v0, int64_t v1, float bound, int n, uint64_t* keys, int most) {
    constexpr int E = Row<XT>::E;
    const int me = Group<THREADS>::thread();
    Group<THREADS>::sync();
    if (me == 0) l.count = 0;
    Group<THREADS>::sync();
    for (int64_t v = v0 + me; v < v1; v += THREADS) {
        float x[E];
        row.load(v, x);
        for (int i = 0; i < E; ++i)
            if (x[i] > bound) {
                const int at = atomicAdd(&l.count, 1);
                if (at < most) keys[at] = order_key(x[i], (uint32_t)(v * E - row.head + i));
            }
    }
    Group<THREADS>::sync();
    const int count = l.count;
    if (count <= most) {
        uint64_t least = 0;
        if (count > n)
            for (int bit = 63; bit >= 0; --bit)
                if (keys_from<THREADS>(l, keys, count, least | (uint64_t)1 << bit) >= n) least |= (uint64_t)1 << bit;
        Group<THREADS>::sync();
        if (me == 0) l.count = 0;
        Group<THREADS>::sync();
        for (int i = me; i < count; i += THREADS)
            if (keys[i] >= least) l.keys[atomicAdd(&l.count, 1)] = keys[i];      // n at most: keys are different
        Group<THREADS>::sync();
        order_list<THREADS>(l, min(count, n), n);
        return;
    }
    uint64_t last = ~(uint64_t)0;
    for (int j = 0; j < n; ++j) {
        uint64_t best = 0;
        for (int64_t v = v0 + me; v < v1; v += THREADS) {
            float x[E];
            row.load(v, x);
            for (int i = 0; i < E; ++i) {
                const int64_t e = v * E - row.head + i;
                const uint64_t key = order_key(x[i], (uint32_t)e);
                if (e >= 0 && e < row.V && key < last && key > best) best = key;
            }
        }
        best = wave_max(best);
        if ((me & 63) == 0) l.wave_best[me >> 6] = best;
        Group<THREADS>::sync();
        for (int w = 0; w < Group<THREADS>::kWaves; ++w) best = l.wave_best[w] > best ? l.wave_best[w] : best;
        last = best;
        if (me == 0) l.sorted[j] = best;
        Group<THREADS>::sync();
    }
}

// Entries of sorted[] that are still 0: the first elements of the slice that are not larger than `bound` (all that are
// larger are there already)
template <typename XT, int THREADS>
__device__ void fill(TopList& l, const Row<XT>& row, int64_t v0, int64_t v1, float bound, int n) {
    constexpr int E = Row<XT>::E;
    const int me = Group<THREADS>::thread();
    int have = 0;
    while (have < n && l.sorted[have]) ++have;
    const int lane = me & 63, wave = me >> 6;
    // the equals of the bound, in order of their index; then, lower than any number, what is none
    for (int pass = 0; pass < 2 && have < n; ++pass) {
        for (int64_t b = v0; b < v1 && have < n; b += THREADS) {
            const int64_t v = b + me;
            float x[E];
            uint32_t mine = 0;
            if (v < v1) {
                row.load(v, x);
                for (int i = 0; i < E; ++i) {
                    const int64_t e = v * E - row.head + i;
                    if (e >= 0 && e < row.V && (pass ? x[i] != x[i] : x[i] == bound)) mine |= 1u << i;
                }
            }
            const int c = __popc(mine);
            const int before = group_prefix_i<64>(c, lane);
            if (lane == 63) l.wave_count[wave] = before + c;
            Group<THREADS>::sync();
            int at = have + before, all = 0;
            for (int w = 0; w < Group<THREADS>::kWaves; ++w) {
                if (w < wave) at += l.wave_count[w];
                all += l.wave_count[w];
            }
            for (int i = 0; i < E; ++i)
                if (mine >> i & 1) {
                    if (at < n) l.sorted[at] = order_key(x[i], (uint32_t)(v * E - row.head + i));
                    ++at;
                }
            have += all;
            Group<THREADS>::sync();
        }
    }
    Group<THREADS>::sync();
}

// what a log probability is made of
struct Norm {
    float m;
    double log2_s;
};

__device__ __forceinline__ float logprob_of(float x, Norm z) {
    if (z.log2_s != z.log2_s) return __builtin_nanf("");
    if (x == -__builtin_inff()) return x;      // a row without words: all are impossible
    const double d = extreme(z.m) ? ((double)x - (double)z.m) * (double)kLog2e : fma((double)x, (double)kLog2e, -(double)(z.m * kLog2e));
    return (float)((d - z.log2_s) * 0.69314718055994530942);
}

// a row's target and its logit, which are asked for long before they are needed
struct Target {
    int64_t at;
    float x;
};
template <typename XT>
__device__ __forceinline__ Target target_of(const Args& g, int64_t row) {
    const int64_t at = g.targets[row];
    return {at, at >= 0 && at < g.V ? XT::load(static_cast<const typename XT::type*>(g.logits)[row * g.ld + at]) : 0.f};
}

// a row's results, by one lane
__device__ __forceinline__ Norm finish(const Args& g, int64_t row, Stats st, Target target) {
    constexpr double kLn2 = 0.69314718055994530942;
    const double log2_s = log2((double)st.s);
    const Norm z{st.m, log2_s};
    const bool words = st.s != 0.f;
    const double lse = extreme(st.m) ? (double)st.m + log2_s * kLn2 : ((double)(st.m * kLog2e) + log2_s) * kLn2;
    g.lse[row] = words ? (float)lse : -__builtin_inff();
    g.entropy[row] = words ? (float)((log2_s - (double)st.t / (double)st.s) * kLn2) : 0.f;
    float p = 0.f;
    if (target.at >= g.V) p = __builtin_nanf("");
    else if (target.at >= 0) p = logprob_of(target.x, z);
    g.logprob[row] = p;
    return z;
}

template <int THREADS>
__device__ __forceinline__ void write_top(const Args& g, int64_t row, const uint64_t* sorted, Norm z) {
    for (int i = Group<THREADS>::thread(); i < g.n; i += THREADS) {
        g.top_values[row * g.n + i] = logprob_of(value_of_key(sorted[i]), z);
        g.top_ids[row * g.n + i] = (int32_t)index_of_key(sorted[i]);
    }
}

// THREADS: a workgroup for a row (or a slice of one), or a wavefront
template <typename XT, bool TOP, int THREADS>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(sizeof(typename XT::type) == 2 ? 7 : 8))) void logprobs_kernel(Args g) {
    using G = Group<THREADS>;
    using R = Row<XT>;
    constexpr int E = R::E, U = kBatch / E, V8 = 8 / E, kRows = kThreads / THREADS;      // pieces of a thread, and of eight elements
    extern __shared__ __align__(16) f32x4 all_largest[];           // [row][place][thread]: of the batches' four eights
    __shared__ TopList lists[kRows];
    __shared__ Stats all_stats[kWaves];
    __shared__ Norm norms[kRows];
    const int mine = __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS), me = G::thread(), wave = G::wave(), lane = threadIdx.x & 63;
    const int64_t r = kRows > 1 ? (int64_t)blockIdx.x * kRows + mine : blockIdx.x / g.slices, slice = kRows > 1 ? 0 : blockIdx.x % g.slices;
    const int64_t row_no = g.first_row + r;
    if (kRows > 1 && row_no >= g.T) return;
    TopList& l = lists[mine];
    Stats* const stats = all_stats + mine * G::kWaves;
    f32x4* const largest = all_largest + mine * g.places * THREADS;
    const R row(g.logits, row_no, g.ld, g.V);
    const int64_t v0 = slice * g.slice_vectors, v1 = min(row.vectors(), v0 + g.slice_vectors);
    if (TOP && me == 0) l.count = l.eight_count = 0;
    const Target target = g.slices == 1 ? target_of<XT>(g, row_no) : Target{-1, 0.f};
    Stats st{-__builtin_inff(), 0.f, 0.f};
    int batches = 0;
    // 16-bit rows: the next batch's pieces are held while one is added up (16 registers; fp32's would be 32)
    constexpr bool kAhead = E == 8;
    const int first = row.first(), last = (int)min(v1, (int64_t)row.last() + 1) - 1;      // whole pieces
    const bool any = row.last() >= first;
    uint4 next[kAhead ? U : 1];
    const auto load = [&](int64_t b) {
#pragma unroll
        for (int u = 0; u < U; ++u) next[u] = row.raw((int)b + u * THREADS + me);
    };
    if constexpr (kAhead) {
        if (any) load(v0);
    }
    for (int64_t b = v0; b < v1; b += THREADS * U, ++batches) {
        float x[kBatch];
        if constexpr (kAhead) {
            uint4 now[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                now[u] = next[u];
                asm volatile("" : "+v"(now[u].x), "+v"(now[u].y), "+v"(now[u].z), "+v"(now[u].w));
            }
            if (b + THREADS * U < v1 && any) load(b + THREADS * U);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int v = (int)b + u * THREADS + me;
                if (v < first || v > last) now[u] = row.edge(v < v1 ? v : row.vectors());
                R::values(now[u], x + u * E);
            }
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t v = b + u * THREADS + me;
                if (v < v1) row.load(v, x + u * E);
                else
#pragma unroll
                    for (int i = 0; i < E; ++i) x[u * E + i] = -__builtin_inff();
            }
        }
        float part[kParts], most = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            part[i] = x[8 * i];
#pragma unroll
            for (int j = 1; j < 8; ++j) part[i] = fmaxf(part[i], x[8 * i + j]);
            most = fmaxf(most, part[i]);
        }
        if constexpr (TOP) {
            f32x4& place = largest[batches / g.sharing * THREADS + me];
            if (batches % g.sharing) {
#pragma unroll
                for (int i = 0; i < kParts; ++i) part[i] = fmaxf(part[i], place[i]);
            }
            place = f32x4{part[0], part[1], part[2], part[3]};
        }
        if (most > st.m) raise(st, most);
        float s0 = 0.f, s1 = 0.f, t0 = 0.f, t1 = 0.f;
        const bool none = st.m == -__builtin_inff();      // so far
        float c = none ? 0.f : st.m * kLog2e;
        if (!none && extreme(st.m)) {
            c = 0.f;
#pragma unroll
            for (int i = 0; i < kBatch; ++i) x[i] -= st.m;
        }
#pragma unroll
        for (int j = 0; j < kParts; ++j) {
            if (b + j * V8 * THREADS >= v1) break;      // no thread has more
#pragma unroll
            for (int i = 8 * j; i < 8 * j + 8; i += 2) {
                const float u0 = at_least(fmaf(x[i], kLog2e, -c), -200.f), u1 = at_least(fmaf(x[i + 1], kLog2e, -c), -200.f);
                const float p0 = exp2_hw(u0), p1 = exp2_hw(u1);
                s0 += p0; s1 += p1;
                t0 = fmaf(p0, u0, t0); t1 = fmaf(p1, u1, t1);
            }
        }
        st.s += s0 + s1;
        st.t += t0 + t1;
    }
    float bound = 0.f;
    if constexpr (TOP) {
        const int with_words = __popcll(__ballot(st.m > -__builtin_inff()));
        if (lane == 0) l.wave_count[wave] = with_words;
        G::sync();
        // of the n, every wavefront answers for its share of the lanes that have words
        int here = l.wave_count[wave], lanes = 0;
        for (int w = 0; w < G::kWaves; ++w) lanes += l.wave_count[w];
        const int k = lanes < g.n ? -1 : (g.n * here + lanes - 1) / lanes;
        const float bound_here = k < 0 ? -__builtin_inff() : k ? kth_largest(st.m, k) : __builtin_inff();
        if (lane == 0) l.bound[wave] = bound_here;
    }
    st = join_wave(st);
    if (lane == 0) stats[wave] = st;
    G::sync();
    if constexpr (TOP) {
        bound = l.bound[0];
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
                    if (at < kList) l.keys[at] = order_key(x[i], (uint32_t)(v * E - row.head + i));
                }
        }
        // meanwhile
        if (me == THREADS - 64) {
            for (int w = 0; w < G::kWaves - 1; ++w) st = join(st, stats[w]);
            if (g.slices == 1) norms[mine] = finish(g, row_no, st, target);
            else g.part_stats[blockIdx.x] = st;
        }
        G::sync();
        const int count = l.count;
        if (eights > kEights || count > kList)
            flooded<XT, THREADS>(l, row, v0, v1, bound, g.n, reinterpret_cast<uint64_t*>(largest),
                                 (batches + g.sharing - 1) / g.sharing * (THREADS * 2));
        else order_list<THREADS>(l, count, g.n);
        // a slice can have fewer words than n that are larger than its bound
        if (!l.sorted[g.n - 1]) fill<XT, THREADS>(l, row, v0, v1, bound, g.n);
        if (g.slices == 1) write_top<THREADS>(g, row_no, l.sorted, norms[mine]);
        else
            for (int i = me; i < g.n; i += THREADS) g.part_keys[(int64_t)blockIdx.x * g.n + i] = l.sorted[i];
    } else if (me == 0) {
        for (int w = 1; w < G::kWaves; ++w) st = join(st, stats[w]);
        if (g.slices == 1) finish(g, row_no, st, target);
        else g.part_stats[blockIdx.x] = st;
    }
}

// joins the slices of a row: the bound is the least of the slices' ceil(n / slices)-th largest
template <typename XT>
__global__ __launch_bounds__(kThreads) void logprobs_join_kernel(Args g) {
    __shared__ KeyList<kSlices * kTopMax> l;
    __shared__ Norm norm;
    const int64_t row = g.first_row + blockIdx.x;
    const int all = g.slices * g.n, lane = threadIdx.x & 63;
    const uint64_t* keys = g.part_keys + (int64_t)blockIdx.x * all;
    if (threadIdx.x == 0) l.count = 0;
    const Target target = target_of<XT>(g, row);
    uint64_t bound = lane < g.slices && g.n ? keys[lane * g.n + (g.n + g.slices - 1) / g.slices - 1] : ~(uint64_t)0;
    bound = ~wave_max(~bound);
    __syncthreads();
    for (int i = threadIdx.x; i < all; i += kThreads) {
        const uint64_t key = keys[i];
        if (key && key >= bound) l.keys[atomicAdd(&l.count, 1)] = key;
    }
    if (threadIdx.x < 64) {
        Stats st{-__builtin_inff(), 0.f, 0.f};
        if (lane < g.slices) st = g.part_stats[(int64_t)blockIdx.x * g.slices + lane];
        st = join_wave(st);
        if (threadIdx.x == 0) norm = finish(g, row, st, target);
    }
    __syncthreads();
    order_list<kThreads>(l, l.count, g.n);
    write_top<kThreads>(g, row, l.sorted, norm);
}

struct BackArgs {
    const void* logits;
    void* grad;
    int64_t V, ld, ldg, first_row;
    const int64_t* targets;
    const float *lse, *entropy, *g_logprob, *g_entropy;
    int slices;
};

// log p = (x - m) - log_s for all of a row, by all threads.  These sums are of 2^((x - m) L), differences first, and go with another m by a
// difference too: raise() and join() are for sums made with m L rounded by itself, whose rounding is theirs as well.
struct Shift {
    float m, log_s;
};
__device__ __forceinline__ float moved_sum(float s, float from, float to) {
    return from == to ? s : s * exp2_hw(at_least((from - to) * kLog2e, -200.f));
}
template <typename XT, int U>
__device__ __forceinline__ Shift shift_of(const Row<XT>& row) {
    constexpr int E = Row<XT>::E;
    __shared__ float largest[kWaves], sums[kWaves];
    float m = -__builtin_inff(), s = 0.f;
    const int64_t pieces = row.vectors();
    for (int64_t b = threadIdx.x; b < pieces; b += kThreads * U) {
        float x[U][E], most = -__builtin_inff();
#pragma unroll
        for (int u = 0; u < U; ++u) row.load(min(b + u * kThreads, pieces), x[u]);      // (behind the last piece: -inf)
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < E; ++i) most = fmaxf(most, x[u][i]);
        if (most > m) {
            s = moved_sum(s, m, most);
            m = most;
        }
        if (m == -__builtin_inff()) continue;
        float part = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < E; ++i) part += exp2_hw(at_least((x[u][i] - m) * kLog2e, -200.f));
        s += part;
    }
    const float most = max_of_wave(m);
    s = sum_of_wave(moved_sum(s, m, most));
    if ((threadIdx.x & 63) == 0) {
        largest[threadIdx.x >> 6] = most;
        sums[threadIdx.x >> 6] = s;
    }
    __syncthreads();
    m = largest[0];
    for (int w = 1; w < kWaves; ++w) m = fmaxf(m, largest[w]);
    s = 0.f;
    for (int w = 0; w < kWaves; ++w) s += moved_sum(sums[w], largest[w], m);
    return {m, logf(s)};
}

// exp(x).  EXACT: with what x log2(e) loses as one rounded product (2^-18 of the result at x = -80), by a first-order factor.
template <bool EXACT>
__device__ __forceinline__ float exp_of(float x) {
    const float u = x * kLog2e, p = exp2_hw(u);
    if constexpr (!EXACT) return p;
    constexpr float kLow = 1.92596299112662e-8f, kLn2 = 0.693147180559945f;      // log2(e) - kLog2e
    return fmaf(p, fmaf(x, kLow, fmaf(x, kLog2e, -u)) * kLn2, p);
}

// |lse| up to which the gradient goes by it.  It is rounded, and what it lost is a factor of all of the row's p: up to 2^-17 below 256, less
// than a row's sums are off by; 2^-15 below 1024 and 2^-13 below 4096, a sixteenth of a binary16 result's rounding and less of a
// bfloat16 one's.
template <typename XT>
constexpr float kLseMost = sizeof(typename XT::type) == 4 ? 256.f : XT::kHalf ? 1024.f : 4096.f;

// d = p * -(g_lp + g_H (log p + H)), and g_lp at the target.  A large lse has lost what a difference of logits needs (1000 words that a mask of
// -1e9 leaves alike would have a probability of 1 each): such rows are summed up once more, by one of the row's workgroups, which then
// has all of it.  Not the first of each row: with eight workgroups a row those all run on the same XCD, and 4096 x 32003 in bfloat16 take 669
// us instead of 363 (107 where lse serves).  700 x 10000 in fp32 19.5 us instead of 10.4, one row of 131072 64 instead of 4.5.
template <typename XT>
__global__ __launch_bounds__(kThreads) void logprobs_backward_kernel(BackArgs g) {
    using T = typename XT::type;
    constexpr int E = Row<XT>::E, U = 16 / E;
    const int64_t r = blockIdx.x / g.slices, slice = blockIdx.x % g.slices, row_no = g.first_row + r;
    const Row<XT> row(g.logits, row_no, g.ld, g.V);
    T* const out = static_cast<T*>(g.grad) + row_no * g.ldg;
    const bool together = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(row.p)) & 15) == 0;
    const float lse = g.lse[row_no];
    // A row in which a mask has left nothing has no gradient: its lse is -inf, or so near the lowest fp32 number that the
    // differences from it are lost.
    const bool empty = lse <= -1e30f;
    int64_t target = g.targets[row_no];
    const float gl = target < 0 ? 0.f : target < g.V ? g.g_logprob[row_no] : __builtin_nanf("");
    const float gh = g.g_entropy ? g.g_entropy[row_no] : 0.f;
    const float at0 = -fmaf(gh, gh != 0.f ? g.entropy[row_no] : 0.f, gl);
    if (empty) target = -1;
    const int64_t v0 = slice * (kThreads * U), v1 = min(row.vectors(), v0 + kThreads * U);
    const auto gradient = [&](float logp, bool hit) {
        if (empty) logp = -1e4f;
        logp = at_least(logp, -1e4f);      // exp of which is 0
        const float v = exp_of<sizeof(T) == 4>(logp) * fmaf(-gh, logp, at0);
        return XT::store(hit ? v + gl : v);
    };
    const auto write = [&](int64_t v, const float (&x)[E], auto&& logp) {
        const int64_t e = v * E - row.head, mine = target - e;
        T d[E];
#pragma unroll
        for (int i = 0; i < E; ++i) d[i] = gradient(logp(x[i]), mine == i);
        if (together && e >= 0 && e + E <= g.V) {
            uint4 w;
            __builtin_memcpy(&w, d, 16);
            *reinterpret_cast<uint4*>(out + e) = w;
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (e + i >= 0 && e + i < g.V) out[e + i] = d[i];
        }
    };
    float x[U][E];
    if (!empty && fabsf(lse) > kLseMost<XT>) {
        if (slice != r % g.slices) return;
        const Shift z = shift_of<XT, U>(row);      // every thread has read the row now, which may be overwritten
        const int64_t pieces = row.vectors();
        for (int64_t b = threadIdx.x; b < pieces; b += kThreads * U) {
#pragma unroll
            for (int u = 0; u < U; ++u) row.load(min(b + u * kThreads, pieces), x[u]);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (b + u * kThreads < pieces) write(b + u * kThreads, x[u], [&](float a) { return (a - z.m) - z.log_s; });
        }
        return;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t v = v0 + u * kThreads + threadIdx.x;
        if (v < v1) row.load(v, x[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t v = v0 + u * kThreads + threadIdx.x;
        if (v >= v1) break;
        write(v, x[u], [&](float a) { return a - lse; });
    }
}

struct Plan {
    bool waves;      // a wavefront for a row
    int slices;
    int64_t slice_vectors;
};

Plan plan_for(int dtype, int64_t T, int64_t V) {
    const int e = 16 / dtype_bytes(dtype), batch = kThreads * (kBatch / e);
    const int64_t vectors = (V + e - 1) / e + 1;      // one more for a row that starts between boundaries
    // A wavefront for a row where there are many that are not long: no thread without words, no barriers.  4096 rows of 2100 fp32
    // words with the 5 largest 14.9 us instead of 19.7, of 8200 bfloat16 words 23.9 instead of 34.1; 4096 x 32003 69 instead of
    // 62, 1024 x 4100 equal, 1024 x 1100 8.4 instead of 10.7, 256 x 1100 7.8 instead of 6.4.
    if (V <= 16384 && T >= (V <= 2048 ? 1024 : 2048)) return {true, 1, vectors};
    // Several workgroups for a row only where it is long, since their sums take a second kernel to join (4 us and the launch):
    // 206 rows of 12635 fp32 words 9.6 us alone, 8.3 + 4.2 halved; one of 131072 8.2 + 4.6 in 16 slices, 13.4 + 4 in 4.
    int64_t slices = 1;
    if (vectors >= 6 * batch)
        while (slices < kSlices && T * slices < 512 && vectors / (slices * 2) >= 2 * kThreads) slices *= 2;
    while (slices < kSlices && slices * kPlaces * batch < vectors) ++slices;      // (longer slices share places)
    Plan p{false, 1, (vectors + slices - 1) / slices};
    p.slices = (int)((vectors + p.slice_vectors - 1) / p.slice_vectors);
    return p;
}

size_t stats_bytes(int64_t T, const Plan& p) { return ((size_t)T * p.slices * sizeof(Stats) + 15) / 16 * 16; }

template <typename XT, int THREADS>
int launch_rows(Args g, int64_t rows, hipStream_t st) {
    constexpr int kRows = kThreads / THREADS, per = THREADS * (kBatch / Row<XT>::E);
    const dim3 grid((unsigned)((rows * g.slices + kRows - 1) / kRows));
    if (g.n) {
        const int64_t batches = (g.slice_vectors + per - 1) / per;
        g.sharing = (int)((batches + kPlaces - 1) / kPlaces);
        g.places = (int)((batches + g.sharing - 1) / g.sharing);
        hipLaunchKernelGGL((logprobs_kernel<XT, true, THREADS>), grid, dim3(kThreads), (size_t)g.places * kThreads * sizeof(f32x4), st, g);
    } else {
        hipLaunchKernelGGL((logprobs_kernel<XT, false, THREADS>), grid, dim3(kThreads), 0, st, g);
    }
    return hip_status(hipGetLastError());
}

template <typename XT>
int launch(Args g, bool waves, hipStream_t st) {
    const int64_t most = ((int64_t)1 << 23) / g.slices;      // rows of a launch: a grid has fewer than 2^32 lanes
    const int64_t T = g.T;
    for (int64_t r = 0; r < T; r += most) {
        const int64_t rows = T - r < most ? T - r : most;
        g.first_row = r;
        g.T = r + rows;
        int rc = waves ? launch_rows<XT, 64>(g, rows, st) : launch_rows<XT, kThreads>(g, rows, st);
        if (rc != BS_OK) return rc;
        if (g.slices == 1) continue;
        hipLaunchKernelGGL(logprobs_join_kernel<XT>, dim3((unsigned)rows), dim3(kThreads), 0, st, g);
        rc = hip_status(hipGetLastError());
        if (rc != BS_OK) return rc;
    }
    return BS_OK;
}

template <typename XT>
int launch_backward(BackArgs g, int64_t T, hipStream_t st) {
    constexpr int E = Row<XT>::E, U = 16 / E;
    g.slices = (int)(((g.V + E - 1) / E + 1 + kThreads * U - 1) / (kThreads * U));
    const int64_t most = ((int64_t)1 << 23) / g.slices > 1 ? ((int64_t)1 << 23) / g.slices : 1;
    for (int64_t r = 0; r < T; r += most) {
        g.first_row = r;
        const int64_t rows = T - r < most ? T - r : most;
        hipLaunchKernelGGL(logprobs_backward_kernel<XT>, dim3((unsigned)(rows * g.slices)), dim3(kThreads), 0, st, g);
        const int rc = hip_status(hipGetLastError());
        if (rc != BS_OK) return rc;
    }
    return BS_OK;
}

}  // namespace

size_t logprobs_workspace_bytes(int dtype, int64_t T, int64_t V, int top_n) {
    const Plan p = plan_for(dtype, T, V);
    return p.slices == 1 ? 0 : stats_bytes(T, p) + (size_t)T * p.slices * top_n * 8;
}

int launch_logprobs(const void* logits, int dtype, int64_t T, int64_t V, int64_t ld, const int64_t* targets, int top_n, float* logprob,
                    float* entropy, float* lse, float* top_values, int32_t* top_ids, void* workspace, size_t workspace_bytes,
                    hipStream_t st) {
    const Plan p = plan_for(dtype, T, V);
    const size_t need = logprobs_workspace_bytes(dtype, T, V, top_n);
    if (need && (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 15))) return BS_ERR_WORKSPACE;
    Args g{};
    g.logits = logits; g.T = T; g.V = V; g.ld = ld; g.targets = targets; g.n = top_n;
    g.slices = p.slices; g.slice_vectors = p.slice_vectors;
    g.logprob = logprob; g.entropy = entropy; g.lse = lse; g.top_values = top_values; g.top_ids = top_ids;
    g.part_stats = static_cast<Stats*>(workspace);
    g.part_keys = need ? reinterpret_cast<uint64_t*>(static_cast<char*>(workspace) + stats_bytes(T, p)) : nullptr;
    switch (dtype) {
        case BS_F32: return launch<F32>(g, p.waves, st);
        case BS_F16: return launch<F16>(g, p.waves, st);
        default: return launch<BF16>(g, p.waves, st);
    }
}

int launch_logprobs_backward(const void* logits, int dtype, int64_t T, int64_t V, int64_t ld, const int64_t* targets, const float* lse,
                             const float* entropy, const float* g_logprob, const float* g_entropy, void* grad, int64_t ldg,
                             hipStream_t st) {
    BackArgs g{};
    g.logits = logits; g.grad = grad; g.V = V; g.ld = ld; g.ldg = ldg; g.targets = targets;
    g.lse = lse; g.entropy = entropy; g.g_logprob = g_logprob; g.g_entropy = g_entropy;
    switch (dtype) {
        case BS_F32: return launch_backward<F32>(g, T, st);
        case BS_F16: return launch_backward<F16>(g, T, st);
        default: return launch_backward<BF16>(g, T, st);
    }
}

}  // namespace bs

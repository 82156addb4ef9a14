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
// Measured: 4096 rows of 32003 bfloat16 logits with the 5 largest in 65 us (4.1 TB/s; 45 at the rate of reads), 58 without
// alternatives: the vector ALU is what is busy, with two instructions to convert, one for the maximum, three for u, one
// exponential (a quarter of the rate) and two sums an element.  One row of 131072 fp32 logits: 8.4 us in 16 slices, 4.7 to join
// them.  The gradient of 4096 x 32003: 106 us, 102 at the rate of a copy.
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
    int sharing;                // batches of a place
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
    __device__ __forceinline__ void load(int64_t v, float* out) const {
        const int64_t e = v * E - head;
        if (e >= 0 && e + E <= V) {
            const uint4 a = *reinterpret_cast<const uint4*>(p + e);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                if constexpr (sizeof(T) == 4) out[i] = __builtin_bit_cast(float, word_of(a, i));
                else out[i] = XT::load((uint16_t)(word_of(a, i >> 1) >> (16 * (i & 1))));
            }
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) out[i] = e + i >= 0 && e + i < V ? XT::load(p[e + i]) : -__builtin_inff();
        }
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
template <int LIST>
__device__ __forceinline__ void order_list(KeyList<LIST>& l, int count, int n) {
    for (int i = threadIdx.x; i < n; i += kThreads)
        if (i >= count) l.sorted[i] = 0;
    const int padded = (count + 7) & ~7;       // the walk below takes eight at a time
    if (threadIdx.x < 8 && count + (int)threadIdx.x < padded) l.keys[count + threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < count; i += kThreads) {
        const uint64_t key = l.keys[i];
        const int before = keys_before(l.keys, padded, key);
        if (before < n) l.sorted[before] = key;
    }
    __syncthreads();
}

// the k-th largest of the lanes' values
__device__ __forceinline__ float kth_largest(float v, int k) {
    float most = v;
    for (int j = 0; j < k; ++j) {
        most = max_of_wave(v);
        const uint64_t m = __ballot(v == most);
        if ((int)(threadIdx.x & 63) == __ffsll((unsigned long long)m) - 1) v = -__builtin_inff();
    }
    return most;
}

// how many of the list's keys are not below `least`; all threads
__device__ __forceinline__ int keys_from(TopList& l, const uint64_t* keys, int count, uint64_t least) {
    int n = 0;
    for (int i = threadIdx.x; i < (count + 63) / 64 * 64; i += kThreads) n += __popcll(__ballot(i < count && keys[i] >= least));
    if ((threadIdx.x & 63) == 0) l.wave_count[threadIdx.x >> 6] = n;
    __syncthreads();
    n = 0;
    for (int w = 0; w < kWaves; ++w) n += l.wave_count[w];
    __syncthreads();
    return n;
}

// The list flooded.  First what is larger than the bound, into the room of the eights' largest (`most` keys), out of which the
// n-th largest key is found bit by bit; if that is too many too, the n largest one after the other.
template <typename XT>
__device__ void flooded(TopList& l, const Row<XT>& row, int64_t v0, int64_t v1, float bound, int n, uint64_t* keys, int most) {
    constexpr int E = Row<XT>::E;
    __syncthreads();
    if (threadIdx.x == 0) l.count = 0;
    __syncthreads();
    for (int64_t v = v0 + threadIdx.x; v < v1; v += kThreads) {
        float x[E];
        row.load(v, x);
        for (int i = 0; i < E; ++i)
            if (x[i] > bound) {
                const int at = atomicAdd(&l.count, 1);
                if (at < most) keys[at] = order_key(x[i], (uint32_t)(v * E - row.head + i));
            }
    }
    __syncthreads();
    const int count = l.count;
    if (count <= most) {
        uint64_t least = 0;
        if (count > n)
            for (int bit = 63; bit >= 0; --bit)
                if (keys_from(l, keys, count, least | (uint64_t)1 << bit) >= n) least |= (uint64_t)1 << bit;
        __syncthreads();
        if (threadIdx.x == 0) l.count = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < count; i += kThreads)
            if (keys[i] >= least) l.keys[atomicAdd(&l.count, 1)] = keys[i];      // n at most: keys are different
        __syncthreads();
        order_list(l, min(count, n), n);
        return;
    }
    uint64_t last = ~(uint64_t)0;
    for (int j = 0; j < n; ++j) {
        uint64_t best = 0;
        for (int64_t v = v0 + threadIdx.x; v < v1; v += kThreads) {
            float x[E];
            row.load(v, x);
            for (int i = 0; i < E; ++i) {
                const int64_t e = v * E - row.head + i;
                const uint64_t key = order_key(x[i], (uint32_t)e);
                if (e >= 0 && e < row.V && key < last && key > best) best = key;
            }
        }
        best = wave_max(best);
        if ((threadIdx.x & 63) == 0) l.wave_best[threadIdx.x >> 6] = best;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) best = l.wave_best[w] > best ? l.wave_best[w] : best;
        last = best;
        if (threadIdx.x == 0) l.sorted[j] = best;
        __syncthreads();
    }
}

// Entries of sorted[] that are still 0: the first elements of the slice that are not larger than `bound` (all that are
// larger are there already)
template <typename XT>
__device__ void fill(TopList& l, const Row<XT>& row, int64_t v0, int64_t v1, float bound, int n) {
    constexpr int E = Row<XT>::E;
    int have = 0;
    while (have < n && l.sorted[have]) ++have;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // the equals of the bound, in order of their index; then, lower than any number, what is none
    for (int pass = 0; pass < 2 && have < n; ++pass) {
        for (int64_t b = v0; b < v1 && have < n; b += kThreads) {
            const int64_t v = b + threadIdx.x;
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
            __syncthreads();
            int at = have + before, all = 0;
            for (int w = 0; w < kWaves; ++w) {
                if (w < wave) at += l.wave_count[w];
                all += l.wave_count[w];
            }
            for (int i = 0; i < E; ++i)
                if (mine >> i & 1) {
                    if (at < n) l.sorted[at] = order_key(x[i], (uint32_t)(v * E - row.head + i));
                    ++at;
                }
            have += all;
            __syncthreads();
        }
    }
    __syncthreads();
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

// a row's results, by one lane
template <typename XT>
__device__ __forceinline__ Norm finish(const Args& g, int64_t row, Stats st) {
    constexpr double kLn2 = 0.69314718055994530942;
    const double log2_s = log2((double)st.s);
    const Norm z{st.m, log2_s};
    const bool words = st.s != 0.f;
    const double lse = extreme(st.m) ? (double)st.m + log2_s * kLn2 : ((double)(st.m * kLog2e) + log2_s) * kLn2;
    g.lse[row] = words ? (float)lse : -__builtin_inff();
    g.entropy[row] = words ? (float)((log2_s - (double)st.t / (double)st.s) * kLn2) : 0.f;
    const int64_t target = g.targets[row];
    float p = 0.f;
    if (target >= g.V) p = __builtin_nanf("");
    else if (target >= 0) p = logprob_of(XT::load(static_cast<const typename XT::type*>(g.logits)[row * g.ld + target]), z);
    g.logprob[row] = p;
    return z;
}

__device__ __forceinline__ void write_top(const Args& g, int64_t row, const uint64_t* sorted, Norm z) {
    for (int i = threadIdx.x; i < g.n; i += kThreads) {
        g.top_values[row * g.n + i] = logprob_of(value_of_key(sorted[i]), z);
        g.top_ids[row * g.n + i] = (int32_t)index_of_key(sorted[i]);
    }
}

template <typename XT, bool TOP>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(8))) void logprobs_kernel(Args g) {
    constexpr int E = Row<XT>::E, U = kBatch / E, V8 = 8 / E;      // pieces of a thread, and of eight elements
    extern __shared__ __align__(16) f32x4 largest[];               // [place][thread]: of the batches' four eights
    __shared__ TopList l;
    __shared__ Stats stats[kWaves];
    __shared__ Norm norm;
    const int64_t r = blockIdx.x / g.slices, slice = blockIdx.x % g.slices, row_no = g.first_row + r;
    const Row<XT> row(g.logits, row_no, g.ld, g.V);
    const int64_t v0 = slice * g.slice_vectors, v1 = min(row.vectors(), v0 + g.slice_vectors);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (TOP && threadIdx.x == 0) l.count = l.eight_count = 0;
    Stats st{-__builtin_inff(), 0.f, 0.f};
    int batches = 0;
    for (int64_t b = v0; b < v1; b += kThreads * U, ++batches) {
        float x[kBatch];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t v = b + u * kThreads + threadIdx.x;
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
        if constexpr (TOP) {
            f32x4& place = largest[batches / g.sharing * kThreads + threadIdx.x];
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
        for (int i = 0; i < kBatch; i += 2) {
            const float u0 = at_least(fmaf(x[i], kLog2e, -c), -200.f), u1 = at_least(fmaf(x[i + 1], kLog2e, -c), -200.f);
            const float p0 = exp2_hw(u0), p1 = exp2_hw(u1);
            s0 += p0; s1 += p1;
            t0 = fmaf(p0, u0, t0); t1 = fmaf(p1, u1, t1);
        }
        st.s += s0 + s1;
        st.t += t0 + t1;
    }
    float bound = 0.f;
    if constexpr (TOP) {
        const int with_words = __popcll(__ballot(st.m > -__builtin_inff()));
        if (lane == 0) l.wave_count[wave] = with_words;
        __syncthreads();
        // of the n, every wavefront answers for its share of the lanes that have words
        int mine = l.wave_count[wave], lanes = 0;
        for (int w = 0; w < kWaves; ++w) lanes += l.wave_count[w];
        const int k = lanes < g.n ? -1 : (g.n * mine + lanes - 1) / lanes;
        const float bound_here = k < 0 ? -__builtin_inff() : k ? kth_largest(st.m, k) : __builtin_inff();
        if (lane == 0) l.bound[wave] = bound_here;
    }
    st = join_wave(st);
    if (lane == 0) stats[wave] = st;
    __syncthreads();
    if constexpr (TOP) {
        bound = l.bound[0];
        for (int w = 1; w < kWaves; ++w) bound = fminf(bound, l.bound[w]);
        for (int b = 0; b * g.sharing < batches; ++b) {
            const f32x4 part = largest[b * kThreads + threadIdx.x];
#pragma unroll
            for (int i = 0; i < kParts; ++i)
                if (part[i] >= bound && part[i] > -__builtin_inff()) {
                    const int at = atomicAdd(&l.eight_count, 1);
                    if (at < kEights) l.eights[at] = (uint32_t)(b * kParts + i) * kThreads + threadIdx.x;
                }
        }
        __syncthreads();
        const int eights = l.eight_count;
        const int64_t pieces = (int64_t)min(eights, kEights) * V8 * g.sharing;
        for (int64_t j = threadIdx.x; j < pieces; j += kThreads) {
            const uint32_t eight = l.eights[j / (V8 * g.sharing)], place = eight / kThreads;
            const int64_t batch = place / kParts * (int64_t)g.sharing + j / V8 % g.sharing;
            const int64_t v = v0 + (batch * U + place % kParts * V8 + j % V8) * kThreads + eight % kThreads;
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
        if (threadIdx.x == kThreads - 64) {
            for (int w = 0; w < kWaves - 1; ++w) st = join(st, stats[w]);
            if (g.slices == 1) norm = finish<XT>(g, row_no, st);
            else g.part_stats[blockIdx.x] = st;
        }
        __syncthreads();
        const int count = l.count;
        if (eights > kEights || count > kList)
            flooded(l, row, v0, v1, bound, g.n, reinterpret_cast<uint64_t*>(largest), (batches + g.sharing - 1) / g.sharing * (kThreads * 2));
        else order_list(l, count, g.n);
        // a slice can have fewer words than n that are larger than its bound
        if (!l.sorted[g.n - 1]) fill(l, row, v0, v1, bound, g.n);
        if (g.slices == 1) write_top(g, row_no, l.sorted, norm);
        else
            for (int i = threadIdx.x; i < g.n; i += kThreads) g.part_keys[(int64_t)blockIdx.x * g.n + i] = l.sorted[i];
    } else if (threadIdx.x == 0) {
        for (int w = 1; w < kWaves; ++w) st = join(st, stats[w]);
        if (g.slices == 1) finish<XT>(g, row_no, st);
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
        if (threadIdx.x == 0) norm = finish<XT>(g, row, st);
    }
    __syncthreads();
    order_list(l, l.count, g.n);
    write_top(g, row, l.sorted, norm);
}

struct BackArgs {
    const void* logits;
    void* grad;
    int64_t V, ld, ldg, first_row;
    const int64_t* targets;
    const float *lse, *entropy, *g_logprob, *g_entropy;
    int slices;
};

// log p = (x - m) - log_s for all of a row, by all threads
struct Shift {
    float m, log_s;
};
template <typename XT>
__device__ __forceinline__ Shift shift_of(const typename XT::type* row, int64_t V) {
    __shared__ Stats stats[kWaves];
    Stats st{-__builtin_inff(), 0.f, 0.f};
    for (int64_t k = threadIdx.x; k < V; k += kThreads) {
        const float x = XT::load(row[k]);
        if (x > st.m) {
            st.s *= exp2_hw(at_least((st.m - x) * kLog2e, -200.f));
            st.m = x;
        }
        if (x != -__builtin_inff()) st.s += exp2_hw(at_least((x - st.m) * kLog2e, -200.f));
    }
    st = join_wave(st);
    if ((threadIdx.x & 63) == 0) stats[threadIdx.x >> 6] = st;
    __syncthreads();
    st = stats[0];
    for (int w = 1; w < kWaves; ++w) st = join(st, stats[w]);
    return {st.m, logf(st.s)};
}

// d = p * -(g_lp + g_H (log p + H)), and g_lp at the target.  A large lse (4096 is 2^12) has lost what a difference of logits
// needs: 1000 words that a mask of -1e9 leaves alike would have a probability of 1 each.  Such rows are summed up once more, and
// the row's first workgroup has all of it.
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
        const float v = exp2_hw(logp * kLog2e) * fmaf(-gh, logp, at0);
        return XT::store(hit ? v + gl : v);
    };
    if (!empty && fabsf(lse) > 4096.f) {
        if (slice) return;
        const Shift z = shift_of<XT>(row.p, g.V);      // every thread has read the row now, which may be overwritten
        for (int64_t k = threadIdx.x; k < g.V; k += kThreads) out[k] = gradient((XT::load(row.p[k]) - z.m) - z.log_s, k == target);
        return;
    }
    float x[U][E];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t v = v0 + u * kThreads + threadIdx.x;
        if (v < v1) row.load(v, x[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t v = v0 + u * kThreads + threadIdx.x, e = v * E - row.head;
        if (v >= v1) break;
        T d[E];
        const int64_t mine = target - e;
#pragma unroll
        for (int i = 0; i < E; ++i) d[i] = gradient(x[u][i] - lse, mine == i);
        if (together && e >= 0 && e + E <= g.V) {
            uint4 w;
            __builtin_memcpy(&w, d, 16);
            *reinterpret_cast<uint4*>(out + e) = w;
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (e + i >= 0 && e + i < g.V) out[e + i] = d[i];
        }
    }
}

struct Plan {
    int slices;
    int64_t slice_vectors;
};

Plan plan_for(int dtype, int64_t T, int64_t V) {
    const int e = 16 / dtype_bytes(dtype);
    const int64_t vectors = (V + e - 1) / e + 1;      // one more for a row that starts between boundaries
    // workgroups for every compute unit, but not slices of less than two pieces a thread
    int64_t slices = 1;
    while (slices < kSlices && T * slices < 512 && vectors / (slices * 2) >= 2 * kThreads) slices *= 2;
    const int64_t most = kPlaces * kThreads * (kBatch / e);      // longer slices share places
    while (slices < kSlices && slices * most < vectors) ++slices;
    Plan p;
    p.slice_vectors = (vectors + slices - 1) / slices;
    p.slices = (int)((vectors + p.slice_vectors - 1) / p.slice_vectors);
    return p;
}

size_t stats_bytes(int64_t T, const Plan& p) { return ((size_t)T * p.slices * sizeof(Stats) + 15) / 16 * 16; }

template <typename XT>
int launch(Args g, hipStream_t st) {
    const int64_t most = ((int64_t)1 << 23) / g.slices;      // rows of a launch: a grid has fewer than 2^32 lanes
    Stats* const stats = g.part_stats;
    for (int64_t r = 0; r < g.T; r += most) {
        const int64_t rows = g.T - r < most ? g.T - r : most;
        g.first_row = r;
        g.part_stats = stats;
        const dim3 grid((unsigned)(rows * g.slices));
        if (g.n) {
            constexpr int per = kThreads * (kBatch / Row<XT>::E);
            const int64_t batches = (g.slice_vectors + per - 1) / per;
            g.sharing = (int)((batches + kPlaces - 1) / kPlaces);
            const size_t lds = (size_t)((batches + g.sharing - 1) / g.sharing) * kThreads * sizeof(f32x4);
            hipLaunchKernelGGL((logprobs_kernel<XT, true>), grid, dim3(kThreads), lds, st, g);
        }
        else hipLaunchKernelGGL((logprobs_kernel<XT, false>), grid, dim3(kThreads), 0, st, g);
        int rc = hip_status(hipGetLastError());
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
        case BS_F32: return launch<F32>(g, st);
        case BS_F16: return launch<F16>(g, st);
        default: return launch<BF16>(g, st);
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

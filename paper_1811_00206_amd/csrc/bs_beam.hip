// One step of beam search, and the states that follow it (bs.h: bs_beam_step, bs_beam_reorder).
//
// The step.  Bound: HBM, the logits of the beams that go on once; measured: the vector ALU.  What orders the words of one beam are its
// logits; what orders those of different beams is a difference of two sums, which must not depend on how either was rounded, so sums are
// made in 64 bits: 2^u by a polynomial of degree 7 between -1/2 and 1/2 (off by 5e-11, and exact at 0: a word that is certain has log
// probability 0), its exponent, less that of the row's largest, added to the number's own.  64-bit operations run at the rate of 32-bit
// ones here (2.4 ns a wavefront's instruction on a SIMD), so the exponential of an element is 15 of them; with unpacking and the largest
// of every eight an element is 17.  Elements come to threads by their index, wherever a row starts in memory: beams with the same
// logits have the same sums to the last bit, and tie.  A row's n largest are found as bs_logprobs finds them.
// A second kernel joins the rows of a sequence: a candidate's total is scores + ((x - m) - log s); of the lists that are full each
// answers for its share of the n, the least of those totals is a bound, and what reaches it is ordered by counting what comes before.
// 256 x 16 rows of 32003 in bfloat16 take 91 to 96 us, of 9740 vector instructions each, and the join 6; 32 x 8 rows 14 and 4.3, latency.
//
// The states.  Bound: HBM.  8 states of 2048 and 513 words for 256 x 16 beams, 234 MB, take 40 us.
#include <type_traits>

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

typedef uint32_t Pair __attribute__((ext_vector_type(2)));

constexpr double kMagic = 0x1.8p52;      // added to a number, its whole part is in the low bits

// 2^f times 2^(the number in t's low bits), -1/2 <= f <= 1/2; 1 for 0 and 0
__device__ __forceinline__ double exp2_parts(double f, double t) {
    double p = 0x1.fde5fe3497e78p-17;
    p = fma(p, f, 0x1.445c8421d1ed2p-13);
    p = fma(p, f, 0x1.5d8a85ff048c0p-10);
    p = fma(p, f, 0x1.3b29f39d29c2ap-7);
    p = fma(p, f, 0x1.c6b08ac06b2ccp-5);
    p = fma(p, f, 0x1.ebfbe07787485p-3);
    p = fma(p, f, 0x1.62e42ff0e1927p-1);
    p = fma(p, f, 1.0);
    Pair v = __builtin_bit_cast(Pair, p);
    v[1] += __builtin_bit_cast(Pair, t)[0] << 20;
    return __builtin_bit_cast(double, v);
}
// exp(x) 2^-c, given magic = kMagic - c; c is whole, |x log2(e) - c| < 1000
__device__ __forceinline__ double exp_over(float x, double magic) {
    const double wide = (double)x, t = fma(wide, kLog2e, magic);
    return exp2_parts(fma(wide, kLog2e, -(t - magic)), t);
}
__device__ __forceinline__ double exp2_wide(double u) {      // -1000 < u < 1000
    const double t = u + kMagic;
    return exp2_parts(u - (t - kMagic), t);
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
// A thread's sum while it is made, in units of 2^c: c is the whole number next to m log2(e) when it was set, which the exponents absorb
// for nothing.  Far from 0 the unit is exp(m), and logits are taken as differences from m in fp32, exact or far beyond -600.
struct Running {
    double s = 0.0, magic = kMagic;      // kMagic - c
    float m = -__builtin_inff();
    bool far = false;
    __device__ __forceinline__ void raise(float to) {
        const bool now_far = !(fabsf(to) <= 0x1p20f);
        const double exponent = (double)to * kLog2e;
        const bool same = !now_far && !far && m != -__builtin_inff() && fabs(exponent - (kMagic - magic)) < 300.0;
        if (!same) {
            const double now = now_far ? kMagic : kMagic - rint(exponent);
            // both units as powers of 2
            const double before = (far ? (double)m * kLog2e : 0.0) + (kMagic - magic), after = (now_far ? exponent : 0.0) + (kMagic - now);
            if (m == -__builtin_inff()) s = s != s ? s : 0.0;      // what was cut off at -600 from nothing
            else if (to == __builtin_inff()) s = __builtin_nan("");
            else s *= exp2_wide(fmin(fmax(before - after, -900.0), 900.0));
            magic = now;
        }
        m = to;
        far = now_far;
    }
    // in units of exp(m), by the same exponential: a certain word's sum is 1
    __device__ __forceinline__ Sum sum() const {
        return Sum{m == -__builtin_inff() ? (s != s ? s : 0.0) : far ? s : s / exp_over(m, magic), m};
    }
};
template <int CTRL>
__device__ __forceinline__ double dpp_wide(double v) {
    Pair p = __builtin_bit_cast(Pair, v);
    p[0] = (uint32_t)dpp_move_i<CTRL>((int)p[0]);
    p[1] = (uint32_t)dpp_move_i<CTRL>((int)p[1]);
    return __builtin_bit_cast(double, p);
}
__device__ __forceinline__ double sum_of_16(double v) {
    v += dpp_wide<0xB1>(v);
    v += dpp_wide<0x4E>(v);
    v += dpp_wide<0x141>(v);
    return v + dpp_wide<0x140>(v);
}
__device__ __forceinline__ Sum join_wave(Sum a) {
    raise(a, max_of_wave(a.m));
    a.s = sum_of_16(a.s);
    a.s += moved(a.s, 16);
    a.s += moved(a.s, 32);
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
    static __device__ __forceinline__ uint4 none() {      // -inf
        const uint32_t w = sizeof(T) == 4 ? 0xff800000u : std::is_same_v<XT, F16> ? 0xfc00fc00u : 0xff80ff80u;
        return uint4{w, w, w, w};
    }
    __device__ __forceinline__ uint4 edge(int64_t v) const {      // a piece that is not whole
        T out[E];
        uint4 a = none();
        __builtin_memcpy(out, &a, 16);
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (v * E + i < V) out[i] = p[v * E + i];
        __builtin_memcpy(&a, out, 16);
        return a;
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
    uint32_t beam_magic, list_magic;      // division by slices * n, by n
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

// The k-th largest of the lanes' values, numbers of type XT, of which k are more than -inf.  Bit by bit, and the scalar unit
// counts: comparing every lane with all is 320 vector instructions (256 x 16 rows of 32003 109.5 us, this way 106; of 2000 23.7 and 20.8).
template <typename XT>
__device__ __forceinline__ float kth_of_lanes(float v, int k) {
    if (k == 1) return max_of_wave(v);
    constexpr int low = std::is_same_v<XT, F32> ? 0 : std::is_same_v<XT, F16> ? 13 : 16;      // bits that the type leaves empty
    const uint32_t bits = __builtin_bit_cast(uint32_t, v), key = bits ^ ((uint32_t)((int)bits >> 31) | 0x80000000u);
    uint32_t least = 0;
#pragma unroll
    for (int bit = 31; bit >= low; --bit) {
        const uint32_t more = least | 1u << bit;
        if (__popcll(__ballot(key >= more)) >= k) least = more;
    }
    return __builtin_bit_cast(float, least >> 31 ? least ^ 0x80000000u : ~(least | ((1u << low) - 1)));
}

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
    Running own;
    int batches = 0;
    // A batch's whole pieces are on their way while the one before is added up; those behind the last of them are that one again, and what
    // is no whole piece comes in first.
    const int first = (int)v0, behind = (int)v1, ragged = (int)(g.V / E), whole = min(behind, ragged);
    uint4 next[U] = {}, edge = R::none();
    const auto load = [&](int b) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (b + u * THREADS < whole) __builtin_memcpy(&next[u], row.p + (int64_t)min(b + u * THREADS + me, whole - 1) * E, 16);
    };
    load(first);
    if (ragged < behind && me == (ragged - first) % THREADS) edge = row.edge(ragged);
    for (int b = first; b < behind; b += THREADS * U, ++batches) {
        float x[kBatch];
        uint4 now[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            now[u] = next[u];
            asm volatile("" : "+v"(now[u].x), "+v"(now[u].y), "+v"(now[u].z), "+v"(now[u].w));
        }
        load(b + THREADS * U);
        if (b + THREADS * U > whole) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int v = b + u * THREADS + me;
                if (v >= whole) now[u] = R::none();
                if (v == ragged) now[u] = edge;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) R::values(now[u], x + u * E);
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
        if (most > own.m) own.raise(most);
        // At least -600 from the largest, where the exponential counts for nothing.
        const bool none = own.m == -__builtin_inff();
        if (own.far) {
#pragma unroll
            for (int i = 0; i < kBatch; ++i) x[i] -= own.m;
        }
        const float least = none || own.far ? -600.f : own.m - 600.f;
        double s0 = 0.0, s1 = 0.0;
#pragma unroll
        for (int j = 0; j < kParts; ++j) {
            if (b + j * V8 * THREADS >= behind) break;      // no thread has more
#pragma unroll
            for (int i = 8 * j; i < 8 * j + 8; i += 2) {
                s0 += exp_over(__builtin_elementwise_maximum(x[i], least), own.magic);
                s1 += exp_over(__builtin_elementwise_maximum(x[i + 1], least), own.magic);
            }
        }
        own.s += s0 + s1;
    }
    Sum st = own.sum();
    G::sync();
    const int with_words = __popcll(__ballot(st.m > -__builtin_inff()));
    if (lane == 0) l.wave_count[wave] = with_words;
    G::sync();
    // of the n, every wavefront answers for its share of the lanes that have words
    int here = l.wave_count[wave], lanes = 0;
    for (int w = 0; w < G::kWaves; ++w) lanes += l.wave_count[w];
    const int k = lanes < g.n ? -1 : (g.n * here + lanes - 1) / lanes;
    const float bound_here = k < 0 ? -__builtin_inff() : k ? kth_of_lanes<XT>(st.m, k) : __builtin_inff();
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
    const uint32_t each = V8 * (uint32_t)g.sharing, pieces = (uint32_t)min(eights, kEights) * each;      // pieces of an eight, of all
    for (uint32_t j = me; j < pieces; j += THREADS) {
        const uint32_t e = g.sharing == 1 ? j / V8 : j / each, rest = j - e * each;
        const uint32_t eight = l.eights[e], place = eight / THREADS;
        const int64_t batch = (int64_t)(place / kParts) * g.sharing + rest / V8;
        const int64_t v = v0 + (batch * U + place % kParts * V8 + rest % V8) * THREADS + eight % THREADS;
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

// the sum over 16 neighbouring lanes, in every one of them; m: the largest of theirs
__device__ __forceinline__ Sum join_16(Sum a) {
    float m = a.m;
    m = fmaxf(m, dpp_move<0xB1>(m));
    m = fmaxf(m, dpp_move<0x4E>(m));
    m = fmaxf(m, dpp_move<0x141>(m));
    m = fmaxf(m, dpp_move<0x140>(m));
    raise(a, m);
    a.s = sum_of_16(a.s);
    return a;
}

// A sequence's n best of what its lists (one for each beam and slice) offer, EACH * 256 candidates at most: candidate i is the one of
// place i % n in list i / n.
template <int EACH>
__global__ __launch_bounds__(kThreads) void beam_join_kernel(Args g) {
    constexpr int kMost = EACH * kThreads;
    __shared__ __align__(16) double totals[kMost + 8];
    __shared__ __align__(16) float logits[kMost + 8];
    __shared__ __align__(16) uint16_t from[kMost + 8];
    __shared__ double wave_bound[kWaves], wave_last[kWaves];
    __shared__ double log_s[kWidth], scores[kWidth];
    __shared__ float most[kWidth];
    __shared__ int kind[kWidth], kept, full;      // kind of a beam: 0 offers nothing, 1 goes on, 2 is finished
    const double none = -(double)__builtin_inff();
    const int64_t b = blockIdx.x, row0 = b * g.W;
    const int me = threadIdx.x, per_beam = g.slices * g.n, lists = g.W * g.slices, all = g.W * per_beam;
    const uint64_t* const keys = g.keys + b * all;
    // Keys are asked for before anything is waited for.  (Beams that offer nothing have written nothing: what is read of theirs is not
    // looked at.)
    uint64_t key[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) key[e] = keys[min(e * kThreads + me, all - 1)];
    if (me == 0) kept = full = 0;
#pragma unroll 1
    for (int w = me / 16; w < g.W; w += kThreads / 16) {      // 16 lanes a beam
        const int slice = me % 16;
        Sum st = g.sums[(row0 + w) * g.slices + min(slice, g.slices - 1)];
        const float score = g.scores[row0 + w];
        const bool done = g.finished && g.finished[row0 + w];
        int is = finite(score) ? done ? 2 : 1 : 0;
        if (is != 1 || slice >= g.slices) st = Sum{0.0, -__builtin_inff()};
        st = join_16(st);
        if (slice == 0) {
            if (is == 1 && !(st.s > 0.0)) is = 0;      // no words, or a logit that is NaN or +inf
            if (is == 1) log_s[w] = log(st.s);
            most[w] = st.m;
            scores[w] = (double)score;
            kind[w] = is;
        }
    }
    __syncthreads();
    double mine[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const int i = e * kThreads + me;
        mine[e] = none;      // the total of what is none
        if (i >= all) continue;
        const int beam = (int)div_magic((uint32_t)i, (uint32_t)per_beam, g.beam_magic);
        const float x = value_of_key(key[e]);
        if (kind[beam] == 2) mine[e] = i == beam * per_beam ? scores[beam] : none;
        else if (kind[beam] == 1 && key[e] && x != -__builtin_inff()) mine[e] = scores[beam] + (((double)x - (double)most[beam]) - log_s[beam]);
        totals[i] = mine[e];
        if (mine[e] > none && i - (int)div_magic((uint32_t)i, (uint32_t)g.n, g.list_magic) * g.n == g.n - 1) atomicAdd(&full, 1);
    }
    __syncthreads();
    // Every full list answers for its share of the n: as many are not below the least of those totals.  Nor are n below the last of any
    // full list.
    const int lists_full = full, share = lists_full ? (g.n + lists_full - 1) / lists_full : 0;
    double bound = -none, last = none;
#pragma unroll 1
    for (int i = me; i < lists && share; i += kThreads) {
        const double end = totals[i * g.n + g.n - 1];
        if (end > none) bound = fmin(bound, totals[i * g.n + share - 1]);
        last = fmax(last, end);
    }
#pragma unroll
    for (int by = 1; by < 64; by *= 2) {
        bound = fmin(bound, moved(bound, by));
        last = fmax(last, moved(last, by));
    }
    if ((me & 63) == 0) {
        wave_bound[me >> 6] = bound;
        wave_last[me >> 6] = last;
    }
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) {
        bound = fmin(bound, wave_bound[w]);
        last = fmax(last, wave_last[w]);
    }
    bound = share ? fmax(bound, last) : none;
    // what is left takes the place of all
#pragma unroll
    for (int e = 0; e < EACH; ++e)
        if (mine[e] > none && mine[e] >= bound) {
            const int at = atomicAdd(&kept, 1);
            totals[at] = mine[e];
            from[at] = (uint16_t)(e * kThreads + me);
            logits[at] = value_of_key(key[e]);
        }
    __syncthreads();
    const int count = kept;
    if (me < 8) totals[count + me] = none;      // the walk below takes eight at a time
    __syncthreads();
    // Four lanes a candidate.  Of equals the lower beam comes first, of one beam's what comes first among its logits: the order of the
    // candidates, unless slices have different logits that are equal as totals.
#pragma unroll 1
    for (int c0 = 0; c0 < count; c0 += kThreads / 4) {
        const int c = min(c0 + me / 4, count - 1);
        const int i = from[c], beam = (int)div_magic((uint32_t)i, (uint32_t)per_beam, g.beam_magic);
        const double t = totals[c];
        const float x = logits[c];
        int before = 0, odd = 0;
#pragma unroll 1
        for (int j = me % 4 * 8; j < count; j += 32) {
            double o[8];
            float l[8];
            uint32_t f[4];
#pragma unroll
            for (int u = 0; u < 8; ++u) o[u] = totals[j + u];
            __builtin_memcpy(f, from + j, 16);
            __builtin_memcpy(l, logits + j, 32);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const bool same = o[u] == t;
                before += o[u] > t || (same && (int)(f[u / 2] >> (16 * (u & 1)) & 0xffff) < i);
                odd |= same && l[u] != x;
            }
        }
        before = group_sum_i<4>(before);
        odd = group_sum_i<4>(odd);
        if (me % 4 || c0 + me / 4 >= count) continue;
        if (odd && g.slices > 1) {
            before = 0;
#pragma unroll 1
            for (int j = 0; j < count; ++j) {
                const int o = from[j];
                bool first = o < i;
                if (totals[j] == t && (int)div_magic((uint32_t)o, (uint32_t)per_beam, g.beam_magic) == beam) first = keys[o] > keys[i];
                before += totals[j] > t || (totals[j] == t && first);
            }
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
#pragma unroll 1
    for (int j = count + me; j < g.n; j += kThreads) {
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
    const int64_t vectors = (V + E - 1) / E;
    // A wavefront for a row takes the n-th largest of its 64 lanes' largest for the bound: near n = 64 that is the least of all of them,
    // and so many words reach it that the list floods, unless it has room for the whole row.  256 x 16 rows of 2000 in bfloat16 take 64 us
    // for n = 58, 183 for 60 and 329 for 64, a workgroup for a row 65, 67 and 69; 32 x 64 of 8003 for n = 64 850, and 207; 128 x 64 of
    // 32003 2824, and 379; 256 x 16 of 700 in binary16 for n = 56 62, and 67, for 58 140, and 70; 1024 x 4 of 256 for n = 64 47, and 54.
    if ((n < 58 || V <= kList) && rows >= (V <= 2048 ? 1024 : 2048)) return {true, 1, vectors};
    // Slices of a row: as many as an estimate of the time, in microseconds, is least for.  A compute unit's workgroups take .04 for each
    // element of a thread and 1 more, one alone is bound by latency, and the join takes longer from one candidate a thread on.  (Seventeen
    // sizes that were timed with 1 to 16 slices meet it within 2: 5 x 9 rows of 101681 22.3 us with 16, 16.1 with 5, 28.8 with 1; 123 x 4 of
    // 72125 38.2 with 2, 34.7 with 1; 38 x 8 of 53421 27.9 with 1, 24.1 with 3, 32.7 with 8.)
    int slices = 1;
    double least = 0;
    for (int s = 1; s <= kSlices && (s == 1 || (W * n * s <= kCandidates && vectors >= s * kThreads)); ++s) {
        const double each = (double)V / s / kThreads, alone = .05 * each + 1.5, all = (double)((rows * s + 255) / 256) * (.04 * each + 1);
        const int candidates = W * n * s;
        const double join = candidates <= kThreads ? 0 : 1 + candidates / 600. + (candidates <= 4 * kThreads ? 0 : 3);
        const double cost = (all > alone ? all : alone) + .03 * s + join;
        if (s > 1 && cost >= least) continue;
        least = cost;
        slices = s;
    }
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
        const int candidates = g.W * g.slices * g.n;
        if (candidates <= kThreads) hipLaunchKernelGGL(beam_join_kernel<1>, dim3((unsigned)g.B), dim3(kThreads), 0, st, g);
        else if (candidates <= 4 * kThreads) hipLaunchKernelGGL(beam_join_kernel<4>, dim3((unsigned)g.B), dim3(kThreads), 0, st, g);
        else hipLaunchKernelGGL((beam_join_kernel<kCandidates / kThreads>), dim3((unsigned)g.B), dim3(kThreads), 0, st, g);
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
    uint32_t pieces, rest;      // of a row: 16 bytes each, and the bytes behind them
    uint32_t first;             // workgroup, of those of a sequence
};
struct States {
    State s[kStates];
    int count;
    uint32_t groups;            // workgroups of a sequence
};
typedef uint32_t Anywhere __attribute__((ext_vector_type(4), aligned(1)));

// A lane has 16 bytes (or one, behind the last 16) of all of a sequence's rows and reads all of them before it writes any: a row may be
// overwritten by another's, and lanes have nothing to do with one another.  Rows behind the last are read as the last and go nowhere.
template <typename T, int ROWS>
__device__ __forceinline__ void move_rows(const State& s, int64_t row0, int W, uint32_t at, const int* parent) {
    T v[ROWS];
#pragma unroll
    for (int j = 0; j < ROWS; ++j) v[j] = *reinterpret_cast<const T*>(s.in + (row0 + parent[j]) * s.pitch + at);
#pragma unroll
    for (int j = 0; j < ROWS; ++j)
        if (j < W && (parent[j] != j || s.in != s.out)) *reinterpret_cast<T*>(s.out + (row0 + j) * s.out_pitch + at) = v[j];
}

// ROWS >= W.  Bound: HBM, the parents' rows once and all rows once.
template <int ROWS>
__global__ __launch_bounds__(256) void beam_reorder_kernel(States all, int W, const int32_t* parents) {
    const uint32_t b = blockIdx.x / all.groups, group = blockIdx.x % all.groups;
    int parent[ROWS];
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        const int own = min(j, W - 1), p = parents[(int64_t)b * W + own];
        parent[j] = p >= 0 && p < W ? p : own;
    }
    int i = 0;
    while (i + 1 < all.count && group >= all.s[i + 1].first) ++i;
    const State& s = all.s[i];
    const int64_t row0 = (int64_t)b * W;
    const uint32_t piece = (group - s.first) * 256 + threadIdx.x;
    if (piece < s.pieces) move_rows<Anywhere, ROWS>(s, row0, W, piece * 16, parent);
    else if (piece - s.pieces < s.rest) move_rows<uint8_t, ROWS>(s, row0, W, s.pieces * 16 + (piece - s.pieces), parent);
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
    // A sequence's workgroup of the join reads that sequence's scores and flags, and stores its outputs behind a barrier: those may take
    // the others' place where they are as many.
    const Rows outs[] = {{out_scores, 1, B * n, 0, 4}, {out_tokens, 1, B * n, 0, 4}, {out_parents, 1, B * n, 0, 4}, {out_finished, 1, B * n, 0, 1}};
    const Rows x(logits, B * W, V, ld, dtype_bytes(dtype)), before(scores, 1, B * W, 0, 4), over(finished, 1, B * W, 0, 1);
    for (int i = 0; i < 4; ++i) {
        if (rows_meet(outs[i], x)) return BS_ERR_UNSUPPORTED;
        if (!(i == 0 && out_scores == scores && n == W) && rows_meet(outs[i], before)) return BS_ERR_UNSUPPORTED;
        if (finished && !(i == 3 && out_finished == finished && n == W) && rows_meet(outs[i], over)) return BS_ERR_UNSUPPORTED;
        for (int j = 0; j < i; ++j)
            if (rows_meet(outs[i], outs[j])) return BS_ERR_UNSUPPORTED;
    }
    const Plan p = plan_for(dtype, B * W, W, V, n);
    Args g{};
    g.logits = logits; g.B = B; g.V = V; g.ld = ld; g.end = end; g.W = W; g.n = n;
    g.slices = p.slices; g.slice_vectors = p.slice_vectors;
    g.beam_magic = magic_u32((uint32_t)(p.slices * n)); g.list_magic = magic_u32((uint32_t)n);
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
        s.pieces = (uint32_t)(row_bytes[i] / 16);
        s.rest = (uint32_t)(row_bytes[i] % 16);
        s.first = (uint32_t)groups;
        groups += (s.pieces + s.rest + 255) / 256;
    }
    all.groups = (uint32_t)groups;
    // sequences of a launch: a grid has fewer than 2^32 lanes
    const int64_t most = ((int64_t)1 << 23) / (int64_t)groups > 1 ? ((int64_t)1 << 23) / (int64_t)groups : 1;
    for (int64_t b = 0; b < B; b += most) {
        const unsigned grid = (unsigned)((B - b < most ? B - b : most) * (int64_t)groups);
        if (W <= 4) hipLaunchKernelGGL(beam_reorder_kernel<4>, dim3(grid), dim3(256), 0, st, all, W, parents + b * W);
        else if (W <= 8) hipLaunchKernelGGL(beam_reorder_kernel<8>, dim3(grid), dim3(256), 0, st, all, W, parents + b * W);
        else if (W <= 16) hipLaunchKernelGGL(beam_reorder_kernel<16>, dim3(grid), dim3(256), 0, st, all, W, parents + b * W);
        else if (W <= 32) hipLaunchKernelGGL(beam_reorder_kernel<32>, dim3(grid), dim3(256), 0, st, all, W, parents + b * W);
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

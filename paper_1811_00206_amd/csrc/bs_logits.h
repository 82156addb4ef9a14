// Rows of logits: how their elements come to threads, and how the n largest of them are found and put in order
// (bs_logprobs.hip, bs_beam.hip).
#pragma once

#include "bs_q4.h"

namespace bs {

#ifdef __HIPCC__

constexpr int kRowThreads = 256;               // of a workgroup
constexpr int kList = 256;                     // keys in LDS
constexpr int kEights = 256;                   // listed eights
constexpr int kTopMax = BS_LOGPROBS_TOP_MAX;

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
        if constexpr (THREADS == kRowThreads) __syncthreads();
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
    float bound[kRowThreads / 64];
    int eight_count, wave_count[kRowThreads / 64];
    uint64_t wave_best[kRowThreads / 64];
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
template <int THREADS, typename R>
__device__ void flooded(TopList& l, const R& row, int64_t v0, int64_t v1, float bound, int n, uint64_t* keys, int most) {
    constexpr int E = R::E;
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
template <int THREADS, typename R>
__device__ void fill(TopList& l, const R& row, int64_t v0, int64_t v1, float bound, int n) {
    constexpr int E = R::E;
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

#endif  // __HIPCC__

}  // namespace bs

// Tiles of y = x W^T for MX 4-bit x and W (bs_mx4_gemm.hip).
//
// A workgroup makes TN rows of y by TM columns with four wavefronts, WN by WM of them, in 32x32x64 matrix instructions.  Both sides pass
// through LDS in stages of 256 columns, which are whole cache lines of a row, NB stages in turns: direct-to-LDS loads bring the others
// while one is multiplied.  A row's eight 16-byte blocks lie in the order block ^ (row / 2 & 7): sixteen lanes' reads of one block, rows
// of 128 bytes, fall on all 64 LDS banks.  Scale bytes come for four stages at a time, 32 bytes of a row: a request to the cache takes as
// long for a row's eight bytes as for a whole line, and those of every stage were half of all requests.  A wavefront's operands of the
// next step are read while this one's are multiplied, over the end of a stage too: its last step first waits for the next stage, meets
// the others, and sends for the one after it.
//
// 4096 rows by 16384 x 8192 take 255 us at 256 x 256, 4.3 PFLOP/s (300 where calls follow one another without a pause), bound by the power that
// the matrix unit takes: with nothing but its instructions the loop takes 222 to 235 on the same data, 251 without loads, 172 without the
// instructions.  256 rows by 32003 x 1500 take 15 to 17 us, beginning and end of a tile of six stages as much as the stages.
#pragma once

#include "bs_mx4.h"

namespace bs {

struct Mx4Tiles {
    const uint8_t *codes, *scales, *x_codes, *x_scales;
    int64_t M, N;
    int chunks;                 // of 128 columns
    int m_tiles, n_tiles, split;
    int stages;                 // of 256 columns, for each of the `split` shares of K
    const float* bias;
    void* y;
    int64_t ldy;
    float* sums;                // [split][N][M], where K is split
};

#ifdef __HIPCC__

constexpr int kMx4Group = 4;      // stages whose scales come together
template <int TN, int TM>
constexpr int kMx4StageBytes = (TN + TM) * 128;
template <int TN, int TM>
constexpr int kMx4ScaleBytes = (TN + TM) * 8 * kMx4Group;
template <int TN, int TM, int NB>
constexpr int kMx4LdsBytes = NB * kMx4StageBytes<TN, TM> + 2 * kMx4ScaleBytes<TN, TM>;

// 16 (4) bytes for each lane of `lanes` (of the first 32 and of the last), from `base` + a lane's offset to LDS at `to`, lane after lane.
// In assembly: the compiler takes every read of LDS for one of what such a load brings, and would wait for all that are on their way.
// Nothing in registers is written but M0, which nothing else here uses and which has to be there a wait state before; all lanes are active
// before and after.  A load of no lanes is counted and comes back in order like the others: products of one stage, whose first wait lets
// twice as many loads go on as that stage has, would be wrong otherwise.
template <int BYTES>
__device__ __forceinline__ void send_to_lds(const uint8_t* base, uint32_t offset, uint32_t to, uint32_t lanes) {
    static_assert(BYTES == 16 || BYTES == 4);
    if constexpr (BYTES == 16)
        asm volatile("s_mov_b32 exec_lo, %3\n\ts_mov_b32 exec_hi, %3\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\t"
                     "global_load_lds_dwordx4 %0, %1\n\ts_mov_b64 exec, -1" ::"v"(offset),
                     "s"(base), "s"(to), "s"(lanes)
                     : "memory");
    else
        asm volatile("s_mov_b32 exec_lo, %3\n\ts_mov_b32 exec_hi, %3\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\t"
                     "global_load_lds_dword %0, %1\n\ts_mov_b64 exec, -1" ::"v"(offset),
                     "s"(base), "s"(to), "s"(lanes)
                     : "memory");
}

// Workgroups of one XCD (every eighth) have neighbouring tiles, eight rows of tiles of W at a time, which share what its cache holds.
__device__ __forceinline__ void mx4_tile_of(const Mx4Tiles& g, uint32_t id, int& m, int& n, int& part) {
    const uint32_t tiles = (uint32_t)g.m_tiles * g.n_tiles, all = tiles * g.split;
    const uint32_t xcd = id & 7, each = all >> 3, more = all & 7;
    id = (id >> 3) + xcd * each + min(xcd, more);
    part = id / tiles;
    id -= part * tiles;
    constexpr uint32_t kRows = 8;
    const uint32_t group = id / (kRows * g.n_tiles), first = group * kRows, rows = min(kRows, g.m_tiles - first);
    id -= first * g.n_tiles;
    n = id / rows;
    m = first + id % rows;
}

template <typename XT, int TN, int TM, int WN, int WM, int NB, bool SPLIT>
__global__ __launch_bounds__(256) void mx4_tiles_kernel(Mx4Tiles g) {
    static_assert(WN * WM == 4);
    constexpr int IN = TN / WN / 32, IM = TM / WM / 32, kSlots = IN * IM;
    constexpr int kRows = TN + TM, kCodeLoads = kRows / 8 / 4;      // of a wavefront and stage
    constexpr int kScaleLoads = (kRows / 32 + 3) / 4;               // of a wavefront and group
    static_assert(TN % 32 == 0 && TM % 32 == 0 && kScaleLoads <= kMx4Group);
    extern __shared__ __align__(16) uint8_t lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    int mt, nt, part;
    mx4_tile_of(g, blockIdx.x, mt, nt, part);
    mt = __builtin_amdgcn_readfirstlane(mt);
    nt = __builtin_amdgcn_readfirstlane(nt);
    part = __builtin_amdgcn_readfirstlane(part);
    const int64_t m0 = (int64_t)mt * TM, n0 = (int64_t)nt * TN;
    const int first = part * g.stages, last = min((g.chunks + 1) / 2, first + g.stages);
    const uint32_t pitch = 64u * g.chunks, scale_pitch = 4u * g.chunks;

    // Rows of a stage: those of x, then those of W; rows behind the last repeat it.  Of a load's 64 lanes eight bring a row's blocks.
    const uint8_t *const xc = g.x_codes + n0 * pitch, *const wc = g.codes + m0 * pitch;
    const uint8_t *const xsc = g.x_scales + n0 * scale_pitch, *const wsc = g.scales + m0 * scale_pitch;
    const uint32_t x_last = (uint32_t)min(g.N - 1 - n0, (int64_t)TN - 1), w_last = (uint32_t)min(g.M - 1 - m0, (int64_t)TM - 1);
    const int block = (lane & 7) ^ (4 * (wave & 1) + (lane >> 4));
    uint32_t from[kCodeLoads];               // a lane's block of stage 0
    const auto row_of = [&](int r) { return r < TN ? min((uint32_t)r, x_last) : min((uint32_t)(r - TN), w_last); };
#pragma unroll
    for (int i = 0; i < kCodeLoads; ++i) from[i] = row_of((i * 4 + wave) * 8 + (lane >> 3)) * pitch + 16 * block;
    // Scales: two lanes bring a row's 32 bytes, the second half in front in every other eight rows, for the sake of LDS banks.  A group that
    // is not whole comes by words, eight lanes a row, those behind the last again the last.  (Where rows are no multiple of 128 some
    // wavefronts bring what another brings too.)
    const auto scale_row = [&](int i) { return min((i * 4 + wave) * 32, kRows - 32); };
    uint32_t scale_from[kScaleLoads];
    uint32_t word_from[kScaleLoads][4];
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i) {
        scale_from[i] = row_of(scale_row(i) + (lane >> 1)) * scale_pitch + 16 * ((lane & 1) ^ (lane >> 4 & 1));
#pragma unroll
        for (int j = 0; j < 4; ++j) word_from[i][j] = row_of(scale_row(i) + 8 * j + (lane >> 3)) * scale_pitch;
    }
    const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    constexpr int kScalesAt = NB * kMx4StageBytes<TN, TM>;
    // Lanes that bring blocks 4 .. 7 stay out of a last stage of one chunk, all of a stage behind the last one.
    const uint32_t first_blocks = wave & 1 ? 0xf0f0f0f0u : 0x0f0f0f0fu;
    const auto send = [&](int stage, int i0, int i1) {      // loads i0 .. i1 - 1 of a stage
        const uint32_t to = lds_at + stage % NB * kMx4StageBytes<TN, TM>;
        const uint32_t lanes = __builtin_amdgcn_readfirstlane(stage >= last ? 0u : 2 * stage + 2 > g.chunks ? first_blocks : ~0u);
#pragma unroll
        for (int i = 0; i < kCodeLoads; ++i)
            if (i >= i0 && i < i1) send_to_lds<16>((i * 32 < TN ? xc : wc) + (int64_t)stage * 128, from[i], to + (i * 4 + wave) * 1024, lanes);
    };
    const auto send_scales = [&](int group, int i) {      // load i of a group, counted from the first stage's
        if (i >= kScaleLoads) return;
        const int chunk = 2 * (first + kMx4Group * group), r = scale_row(i);
        const uint32_t to = lds_at + kScalesAt + (group & 1) * kMx4ScaleBytes<TN, TM> + r * 32;
        const bool any = first + kMx4Group * group < last, whole = chunk + 2 * kMx4Group <= g.chunks;
        const uint32_t lanes = __builtin_amdgcn_readfirstlane(any && whole ? ~0u : 0u),
                       by_words = __builtin_amdgcn_readfirstlane(any && !whole ? ~0u : 0u);
        const uint8_t* const base = r < TN ? xsc : wsc;
        send_to_lds<16>(base + (int64_t)chunk * 4, scale_from[i], to, lanes);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            send_to_lds<4>(base, word_from[i][j] + 4 * (uint32_t)min(chunk + ((lane & 7) ^ 4 * (j & 1)), g.chunks - 1), to + j * 256, by_words);
    };

    const int wn = wave / WM * (IN * 32), wm = wave % WM * (IM * 32), half = lane >> 5;
    const int x_row = wn + (lane & 31), w_row = TN + wm + (lane & 31);
    uint4 x[2][IN], w[2][IM];
    uint32_t xs[IN][2], ws[IM][2];            // scale bytes of a stage, a lane's own in the bytes 0 and 2
    uint2 x_next[IN], w_next[IM];             // those of the next, as they lie in memory
    f32x16 acc[IN][IM];
#pragma unroll
    for (int i = 0; i < IN; ++i)
#pragma unroll
        for (int j = 0; j < IM; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    // (Sums stay where they are, which a compiler that knows the zeros does not see to where K has no whole stage.)
#pragma unroll
    for (int i = 0; i < IN; ++i)
#pragma unroll
        for (int j = 0; j < IM; ++j) asm volatile("" : "+a"(acc[i][j]));
    const auto read_scales = [&](int slot, int stage) {
        const int n = stage - first;
        const uint8_t* const at = lds + kScalesAt + (n / kMx4Group & 1) * kMx4ScaleBytes<TN, TM> + ((n % kMx4Group * 8) ^ ((lane & 8) * 2));
#pragma unroll
        for (int e = 0; e < IN + IM; ++e) {
            if (min(e / 2, kSlots - 1) != slot) continue;      // early in a step: they are the first that the next one needs
            if (e < IN) x_next[e] = *reinterpret_cast<const uint2*>(at + (x_row + 32 * e) * 32);
            else w_next[e - IN] = *reinterpret_cast<const uint2*>(at + (w_row + 32 * (e - IN)) * 32);
        }
    };
    const auto take_scales = [&]() {
#pragma unroll
        for (int i = 0; i < IN; ++i) {
            xs[i][0] = x_next[i].x >> (8 * half);
            xs[i][1] = x_next[i].y >> (8 * half);
        }
#pragma unroll
        for (int j = 0; j < IM; ++j) {
            ws[j][0] = w_next[j].x >> (8 * half);
            ws[j][1] = w_next[j].y >> (8 * half);
        }
    };
    // What this wavefront has read is there, and what it has sent for: all, or all but the loads of the last NB - 2 stages.  (Scales among
    // those make it wait for a few more.)
    const auto arrive = [&](auto LEFT) {
        pin_order();
        wait_vm_and_lds<decltype(LEFT)::value>();
        __builtin_amdgcn_s_barrier();
        pin_order();
    };
    // Step s of a stage; between(n) goes in front of its n-th instruction and nothing moves across: what it issues runs while the matrix
    // unit is busy with the one before.
    const auto step = [&](auto S, auto&& between) {
        constexpr int s = decltype(S)::value;
#pragma unroll
        for (int n = 0; n < kSlots; ++n) {
            const int i = n / IM, j = n % IM;
            between(n);
            __builtin_amdgcn_sched_barrier(0);
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx4_operand(w[s & 1][j]), mx4_operand(x[s & 1][i]), acc[i][j], 4, 4,
                                                                        2 * (s & 1), (int)ws[j][s >> 1], 2 * (s & 1), (int)xs[i][s >> 1]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const std::integral_constant<int, 0> S0;
    const std::integral_constant<int, 1> S1;
    const std::integral_constant<int, 2> S2;
    const std::integral_constant<int, 3> S3;
    // operands of step s of a stage, one read in each of the first slots
    const auto read = [&](int n, int stage, int s) {
        const uint8_t* const at = lds + stage % NB * kMx4StageBytes<TN, TM> + 16 * ((2 * s + half) ^ (lane >> 1 & 7));
#pragma unroll
        for (int e = 0; e < IN + IM; ++e) {
            if (e * kSlots / (IN + IM) != n) continue;      // in the order in which they are needed
            if (e == 0) x[s & 1][0] = *reinterpret_cast<const uint4*>(at + x_row * 128);
            else if (e <= IM) w[s & 1][e - 1] = *reinterpret_cast<const uint4*>(at + (w_row + 32 * (e - 1)) * 128);
            else x[s & 1][e - IM] = *reinterpret_cast<const uint4*>(at + (x_row + 32 * (e - IM)) * 128);
        }
    };
    const auto all_of = [&](auto&& part) {
#pragma unroll
        for (int n = 0; n < kSlots; ++n) part(n);
    };
    constexpr int kEarly = kCodeLoads / 2, kLeft = (NB - 2) * kCodeLoads;
    static_assert(kLeft < 64);
    const std::integral_constant<int, kLeft> ALL_BUT_LATER;
    const int whole = min(last, g.chunks / 2);      // stages of two chunks
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i) send_scales(0, i);
#pragma unroll
    for (int i = 0; i < NB - 1; ++i) send(first + i, 0, kCodeLoads);
    arrive(ALL_BUT_LATER);
    send(first + NB - 1, 0, kEarly);
    all_of([&](int n) { read(n, first, 0); });
    all_of([&](int n) { read_scales(n, first); });
    for (int k = first; k < whole; ++k) {
        take_scales();
        step(S0, [&](int n) {
            read(n, k, 1);
            send(k + NB - 1, kEarly + n * (kCodeLoads - kEarly) / kSlots, kEarly + (n + 1) * (kCodeLoads - kEarly) / kSlots);
        });
        // the next group's scales, all at the group's first stage: their place is free since the stage before
        if ((k - first) % kMx4Group == 0) {
#pragma unroll
            for (int i = 0; i < kScaleLoads; ++i) send_scales((k - first) / kMx4Group + 1, i);
        }
        step(S1, [&](int n) { read(n, k, 2); });
        step(S2, [&](int n) { read(n, k, 3); });
        arrive(ALL_BUT_LATER);      // the next stage is there, and this one's place may be taken
        step(S3, [&](int n) {
            read(n, k + 1, 0);
            read_scales(n, k + 1);
            send(k + NB, n * kEarly / kSlots, (n + 1) * kEarly / kSlots);
        });
    }
    if (whole < last) {      // a stage of one chunk, which is the last one
        take_scales();
        step(S0, [&](int n) { read(n, whole, 1); });
        step(S1, [&](int) {});
    }

    // Results: a lane has four neighbouring columns of a row at a time.  32 rows of a wavefront pass through its part of LDS and leave as
    // whole rows.
    using T = std::conditional_t<SPLIT, float, typename XT::type>;
    constexpr int kCols = IM * 32, kPitch = kCols + 16 / (int)sizeof(T);      // elements
    static_assert(4 * 32 * kPitch * (int)sizeof(T) <= kMx4LdsBytes<TN, TM, NB>);
    __syncthreads();
    T* const mine = reinterpret_cast<T*>(lds) + wave * 32 * kPitch;
    float* const bias = reinterpret_cast<float*>(lds + 4 * 32 * kPitch * sizeof(T));
    static_assert(4 * 32 * kPitch * (int)sizeof(T) + TM * 4 <= kMx4LdsBytes<TN, TM, NB>);
    if constexpr (!SPLIT) {
        for (int i = threadIdx.x; i < TM; i += 256) bias[i] = g.bias ? g.bias[min(m0 + i, g.M - 1)] : 0.f;
        __syncthreads();
    }
    T* const y = SPLIT ? reinterpret_cast<T*>(g.sums) + (int64_t)part * g.N * g.M : static_cast<T*>(g.y);
    const int64_t ld = SPLIT ? g.M : g.ldy, mw = m0 + wm;
    const bool inside = m0 + TM <= g.M && n0 + TN <= g.N;
#pragma unroll
    for (int i = 0; i < IN; ++i) {
#pragma unroll
        for (int j = 0; j < IM; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int col = 32 * j + 8 * q + 4 * half;
                f32x4 a{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                if constexpr (SPLIT) {
                    *reinterpret_cast<f32x4*>(mine + (lane & 31) * kPitch + col) = a;
                } else {
                    a += *reinterpret_cast<const f32x4*>(bias + wm + col);
                    alignas(16) T v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = XT::store(a[e]);
                    if constexpr (sizeof(T) == 4) *reinterpret_cast<uint4*>(mine + (lane & 31) * kPitch + col) = *reinterpret_cast<const uint4*>(v);
                    else *reinterpret_cast<uint2*>(mine + (lane & 31) * kPitch + col) = *reinterpret_cast<const uint2*>(v);
                }
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        constexpr int kPer = 16 / sizeof(T), kLanes = kCols / kPer;      // lanes of a row
        typedef uint32_t Anywhere __attribute__((ext_vector_type(4), aligned(2)));
        const int r = lane / kLanes, col = lane % kLanes * kPer;
        T* const to = y + (n0 + wn + 32 * i + r) * ld + mw + col;
        if (inside) {
#pragma unroll
            for (int r0 = 0; r0 < 32; r0 += 64 / kLanes) {
                const uint4 v = *reinterpret_cast<const uint4*>(mine + (r0 + r) * kPitch + col);
                *reinterpret_cast<Anywhere*>(to + r0 * ld) = Anywhere{v.x, v.y, v.z, v.w};
            }
        } else {
            const bool piece = mw + col + kPer <= g.M;
#pragma unroll
            for (int r0 = 0; r0 < 32; r0 += 64 / kLanes) {
                if (n0 + wn + 32 * i + r0 + r >= g.N) continue;
                const T* const v = mine + (r0 + r) * kPitch + col;
                if (piece) {
                    const uint4 a = *reinterpret_cast<const uint4*>(v);
                    *reinterpret_cast<Anywhere*>(to + r0 * ld) = Anywhere{a.x, a.y, a.z, a.w};
                } else {
#pragma unroll 1
                    for (int e = 0; mw + col + e < g.M; ++e) to[r0 * ld + e] = v[e];
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

#endif  // __HIPCC__

}  // namespace bs

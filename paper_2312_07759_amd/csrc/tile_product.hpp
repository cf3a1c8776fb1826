// out[m, n] = sum_c A[m, c] B[n, c]: the product of two matrices whose rows lie along the sum, on the matrix cores.
//
// A workgroup of WM x WN wavefronts computes a BM x BN tile.  128 bytes of every row of A and B (64 elements of 16 bits, 32
// of float) make a step; ST steps are in flight, each copied from memory straight into LDS.  Row r's 16-byte pieces lie in
// the order c ^ (r mod 8), so that the eight lanes that LDS serves together read eight different bank groups.
// Operands are padded: a row's elements up to the next whole step are there (and zero in one of the two), rows begin at
// multiples of 16 bytes.  Rows behind the last one are read from the last one and not stored.
// 2048 x 4096 x 4096 in bfloat16: 62 us, 1100 TFLOP/s (the library's 61.9); 4096 x 4096 x 2048 with float32 results: 62 to 65 (the library's 52.8, with
// results of 16 bits); 512 x 4608 x 1024 in float32: 57 (the library's 64); 2048 x 4096 x 4096 in 8-bit integers: 38 (the library's 45.7).  Bound by the matrix cores and, between two steps, by the
// barrier: nothing covers it where a workgroup fills a compute unit (16 bits: 256 x 128, 256 x 256 and 128 x 128 with four stages; float: 128 x 128);
// of the other shapes two fit.
#pragma once
#include <type_traits>

#include "elem.hpp"

namespace idkm {

struct TileArgs {
    const void* A;
    const void* B;
    int64_t lda, ldb;  // elements between rows
    int64_t M, N;
    int steps;         // steps of 128 bytes along the sum
    void* out;         // T [M, ldo], or float when `wide`
    int64_t ldo;
    int wide;          // 1: float32 sums (int32 ones of 8-bit integers); the z-th of `parts` parts of the sum goes to out + z M ldo
    int tiles_m, tiles_n, parts;
    // kernels with scales: B's element c of row n stands for scales[(c / group) scale_pitch + n] times itself
    const float* scales;  // its rows go on to a multiple of 128 rows of B
    int64_t scale_pitch;
    int groups;
    int group;  // in steps (SC = 1) or in half steps (SC = 2)
    // 8-bit integers, not wide: out[m, n] = by_m[m] by_n[n] sum, in the type that `dtype` names
    // float16 without scales, not wide: out[m, n] = by_m[m] sum where by_m is not null
    const float* by_m;
    const float* by_n;
    int dtype;
};

// Four consecutive results of a row, the last ones of it fewer.
template <typename V, typename O>
__device__ __forceinline__ void store_four(O* o, const V* v, bool quad, int64_t have) {
    if (have >= 4) {
        struct alignas(4 * sizeof(O)) Quad { O v[4]; } w;
#pragma unroll
        for (int r = 0; r < 4; ++r) w.v[r] = v[r];
        if (quad) {
            *reinterpret_cast<Quad*>(o) = w;
        } else if constexpr (sizeof(O) == 2) {  // rows that begin anywhere: still one store, which global memory allows
            u32x2_any raw;
            __builtin_memcpy(&raw, &w, sizeof(raw));
            *reinterpret_cast<u32x2_any*>(o) = raw;
        } else {
            u32x4 raw;
            __builtin_memcpy(&raw, &w, sizeof(raw));
            *reinterpret_cast<u32x4_word*>(o) = raw;
        }
    } else {
        for (int r = 0; r < 4 && r < have; ++r) o[r] = v[r];
    }
}

// .. float32 ones, rounded to the type that dtype names; at: elements from `out` on.
__device__ __forceinline__ void store_four_as(void* out, int64_t at, int dtype, const float* v, bool quad, int64_t have) {
    if (dtype == 0) {
        store_four(static_cast<float*>(out) + at, v, quad, have);
    } else if (dtype == 1) {
        const f16 w[4] = {Elem<f16>::down(v[0]), Elem<f16>::down(v[1]), Elem<f16>::down(v[2]), Elem<f16>::down(v[3])};
        store_four(static_cast<f16*>(out) + at, w, quad, have);
    } else {
        const bf16 w[4] = {Elem<bf16>::down(v[0]), Elem<bf16>::down(v[1]), Elem<bf16>::down(v[2]), Elem<bf16>::down(v[3])};
        store_four(static_cast<bf16*>(out) + at, w, quad, have);
    }
}

// One product, or two that do not depend on each other in one launch: the workgroups of the first come first.
struct TileJobs {
    TileArgs job[2];
    unsigned first;  // workgroups of job[0]
};

constexpr int TP_STEP = 128;  // bytes

// SC: 0 no scales; 1 one scale of a row of B for every step (64 elements of 16 bits), 2 one for every half step, which is what one matrix
// instruction sums.  The instructions of a step, or half step, begin at zero and their float32 sum times the scale is added to the tile's, so
// that a scaled weight is never rounded to T.  Scales come into LDS with the step that they belong to.  2048 x 4096 x 4096 in bfloat16: 74 to 87 us
// with SC = 1, 90 with SC = 2, where SC = 0 takes 62 to 70: an addition for every element of the tile and step, beside two matrix instructions for 64.
template <typename T, int BM, int BN, int WM, int WN, int ST, int SC>
__global__ __launch_bounds__(64 * WM * WN, SC > 0 ? 2 : 1) void k_tile_product(const TileJobs jobs) {
    constexpr int NW = WM * WN;
    constexpr int PIECES = (BM + BN) / 8;      // 8 rows of 128 bytes: what a wavefront copies at once
    constexpr int PPW = PIECES / NW;
    static_assert(PIECES % NW == 0 && BM % (16 * WM) == 0 && BN % (16 * WN) == 0, "tile and wavefronts");
    constexpr int TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int STAGE = (BM + BN) * TP_STEP + SC * BN * 4;
    constexpr int COPIES = PPW + SC;  // of a wavefront for a step
    extern __shared__ __align__(1024) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Workgroups go to the eight dies in turn: a die gets a run of neighbouring tiles, which share rows of A and B in its
    // cache.  Inside a run tiles go down strips of eight rows of tiles.
    const int of = blockIdx.x < jobs.first ? 0 : 1;
    const TileArgs& a = jobs.job[of];
    const int total = a.tiles_m * a.tiles_n;
    int t = blockIdx.x - (of ? jobs.first : 0u);
    const int parts = a.parts, z = __builtin_amdgcn_readfirstlane(t / total);
    t -= z * total;
    {
        const int die = t & 7, at = t >> 3, whole = total >> 3, rest = total & 7;
        t = die * whole + (die < rest ? die : rest) + at;
    }
    const int strip = 8 * a.tiles_n, s0 = __builtin_amdgcn_readfirstlane(t / strip), in = t - s0 * strip;
    const int high = min(8, a.tiles_m - s0 * 8);
    const int tn = __builtin_amdgcn_readfirstlane(in / high), tm = s0 * 8 + in - tn * high;
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    // this workgroup's part of the sum
    const int each = (a.steps + parts - 1) / parts;
    const int first = min(a.steps, z * each), last = min(a.steps, first + each);

    const unsigned char* src[PPW];
#pragma unroll
    for (int p = 0; p < PPW; ++p) {
        const int r = (wave * PPW + p) * 8 + (lane >> 3);
        const int c = (lane & 7) ^ (lane >> 3);
        const bool of_a = r < BM;  // uniform over the piece: BM is a multiple of 8
        const int64_t row = of_a ? min(m0 + r, a.M - 1) : min(n0 + (r - BM), a.N - 1);
        src[p] = static_cast<const unsigned char*>(of_a ? a.A : a.B) + row * ((of_a ? a.lda : a.ldb) * (int64_t)sizeof(T)) + c * 16;
    }
    // the group of the next step that is fetched, and its steps (half steps) that are left
    int group_at[SC + 1], group_left[SC + 1];
    constexpr int EACH = BN / NW;  // rows of B whose scales a wavefront copies, a lane to each
    const float* scales = nullptr;
    if constexpr (SC > 0) {
        scales = a.scales + n0 + wave * EACH + lane;
#pragma unroll
        for (int h = 0; h < SC; ++h) {
            group_at[h] = (first * SC + h) / a.group;
            group_left[h] = a.group - (first * SC + h - group_at[h] * a.group);
        }
    }
    auto fetch = [&](int step, int slot) {
        // behind the last step the last one is fetched again, into a slot that nobody reads: the count of copies in flight stays the same
        const int64_t off = (int64_t)min(step, last - 1) * TP_STEP;
        unsigned char* to = lds + slot * STAGE;
        if constexpr (SC > 0) {
#pragma unroll
            for (int h = 0; h < SC; ++h) {
                if (lane < EACH)
                    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(scales + min(group_at[h], a.groups - 1) * a.scale_pitch),
                                                     (__attribute__((address_space(3))) void*)(to + (BM + BN) * TP_STEP + (h * BN + wave * EACH) * 4), 4, 0, 0);
                group_left[h] -= SC;
#pragma unroll
                for (int again = 0; again < SC; ++again)
                    if (group_left[h] <= 0) {
                        group_left[h] += a.group;
                        ++group_at[h];
                    }
            }
        }
#pragma unroll
        for (int p = 0; p < PPW; ++p)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src[p] + off),
                                             (__attribute__((address_space(3))) void*)(to + (wave * PPW + p) * 1024), 16, 0, 0);
    };
    typename Sum<T>::four acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = typename Sum<T>::four{0, 0, 0, 0};

    const int wm = wave / WN, wn = wave % WN;
    const int li = lane & 15, q = lane >> 4;
    const int row_a = wm * (BM / WM) + li, row_b = BM + wn * (BN / WN) + li;
    constexpr bool TURNS = SC == 0 && TM * TN >= 8;  // fewer matrix instructions do not cover what is put between them
    if (TURNS && first < last) {
        // Half a step's fragments are read while the matrix cores work on the other half's, and the next steps' copies are issued a few at a time between
        // matrix instructions: issued one after another they hold up the wavefront for as long as the loads of all wavefronts take to be accepted.
        constexpr int MMAS = TM * TN, READS = TM + TN, LATER = PPW / 2, NOW = PPW - LATER;
        u32x4 fa[2][TM], fb[2][TN];
        auto read = [&](int h, int slot, int i) {
            const unsigned char* base = lds + slot * STAGE;
            const int c = (((h << 2) | q) ^ (li & 7)) << 4;
            if (i < TN) fb[h][i] = *reinterpret_cast<const u32x4*>(base + (row_b + i * 16) * TP_STEP + c);
            else fa[h][i - TN] = *reinterpret_cast<const u32x4*>(base + (row_a + (i - TN) * 16) * TP_STEP + c);
        };
        auto copy = [&](int step, int slot, int p) {
            const int64_t off = (int64_t)min(step, last - 1) * TP_STEP;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src[p] + off),
                                             (__attribute__((address_space(3))) void*)(lds + slot * STAGE + (wave * PPW + p) * 1024), 16, 0, 0);
        };
        // matrix instructions of half h; between them the other half's fragments are read, from read_slot, and copies [from, to) of copy_step are issued
        auto multiply = [&](int h, int read_slot, int copy_step, int copy_slot, auto from_, auto to_) {
            constexpr int from = decltype(from_)::value, to = decltype(to_)::value;
            int r = 0, p = from;
#pragma unroll
            for (int m = 0; m < MMAS; ++m) {
                mma16<T>(acc[m / TN][m % TN], fb[h][m % TN], fa[h][m / TN]);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int again = 0; again < READS; ++again)
                    if (r < READS && r * 3 * MMAS <= m * 4 * READS) read(1 - h, read_slot, r++);
#pragma unroll
                for (int again = from; again < to; ++again)
                    if (p < to && (2 * (p - from) + 1) * MMAS <= 2 * (m + 1) * (to - from)) copy(copy_step, copy_slot, p++);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int again = 0; again < READS; ++again)
                if (r < READS) read(1 - h, read_slot, r++);
            __builtin_amdgcn_sched_barrier(0);
        };
        // vmcnt: so many copies of this wavefront may still be on their way; lgkmcnt 0: its own reads have returned
        constexpr auto wait = [](int copies) { return 0x0070 | (copies & 15) | ((copies >> 4) << 14); };
        constexpr std::integral_constant<int, 0> none;
        constexpr std::integral_constant<int, NOW> now;
        constexpr std::integral_constant<int, PPW> all;
#pragma unroll
        for (int s = 0; s < ST; ++s)
#pragma unroll
            for (int p = 0; p < (s < ST - 1 ? PPW : NOW); ++p) copy(first + s, s, p);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(wait((ST - 2) * PPW + NOW));
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < READS; ++i) read(0, 0, i);
        int slot = 0;
        for (int step = first; step < last; ++step) {
            const int before = slot == 0 ? ST - 1 : slot - 1, next = slot + 1 == ST ? 0 : slot + 1;
            multiply(0, slot, step + ST - 1, before, now, all);
            // behind the barrier everybody's copies of the next step are there, and everybody has read this step's slot, which is fetched into next
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(wait((ST - 2) * PPW));
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            multiply(1, next, step + ST, slot, none, now);  // behind the last step: fragments that nobody uses
            slot = next;
        }
        __builtin_amdgcn_s_waitcnt(0x0f70);  // nothing may still be written into this LDS when it is given to others
    }
    if (!TURNS && first < last) {
#pragma unroll
        for (int s = 0; s < ST - 1; ++s) fetch(first + s, s);
        int slot = 0;
        for (int step = first; step < last; ++step) {
            // all but the newest ST - 2 steps' copies of this wavefront are there; after the barrier everybody's are, and
            // everybody has read the slot that is fetched into next
            // (vmcnt: ST - 2 steps' copies; lgkmcnt 0: this wavefront's own reads of that slot have returned)
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(0x0070 | ((COPIES * (ST - 2)) & 15) | (((COPIES * (ST - 2)) >> 4) << 14));
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            const int next = slot == 0 ? ST - 1 : slot - 1;
            const unsigned char* base = lds + slot * STAGE;
            // All of the step's fragments are read first, then the copies are issued: the other way round the reads wait
            // behind the copies' issue (256 x 128 x 4096: 66 us instead of 62 for 2048 x 4096).
            u32x4 fa[2][TM], fb[2][TN];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int c = (((h << 2) | q) ^ (li & 7)) << 4;
#pragma unroll
                for (int j = 0; j < TN; ++j) fb[h][j] = *reinterpret_cast<const u32x4*>(base + (row_b + j * 16) * TP_STEP + c);
#pragma unroll
                for (int i = 0; i < TM; ++i) fa[h][i] = *reinterpret_cast<const u32x4*>(base + (row_a + i * 16) * TP_STEP + c);
            }
            floatx4 scale[SC + 1][TN];  // of this lane's rows n0 + .. + 4 q + r of B (see the stores below)
            if constexpr (SC > 0) {
#pragma unroll
                for (int h = 0; h < SC; ++h)
#pragma unroll
                    for (int j = 0; j < TN; ++j)
                        scale[h][j] = *reinterpret_cast<const floatx4*>(base + (BM + BN) * TP_STEP + (h * BN + wn * (BN / WN) + j * 16 + q * 4) * 4);
            }
            fetch(step + ST - 1, next);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (SC == 0) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < TM; ++i)
#pragma unroll
                        for (int j = 0; j < TN; ++j) mma16<T>(acc[i][j], fb[h][j], fa[h][i]);
            } else {
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        floatx4 part{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            mma16<T>(part, fb[h][j], fa[h][i]);
                            if (SC == 1 && h == 0) continue;
#pragma unroll
                            for (int r = 0; r < 4; ++r) acc[i][j][r] = fmaf(scale[SC - 1 < h ? 0 : h][j][r], part[r], acc[i][j][r]);
                            part = floatx4{0.f, 0.f, 0.f, 0.f};
                        }
                    }
                // A sum's additions come behind the matrix instructions of the next two sums: the wavefront would wait for the last one otherwise
                constexpr int AHEAD = SC == 1 ? 2 : 3, SUMS = TM * TN * SC;
#pragma unroll
                for (int p = 0; p < SUMS; ++p) {
                    __builtin_amdgcn_sched_group_barrier(0x8, 2 / SC, 0);
                    if (p >= AHEAD) __builtin_amdgcn_sched_group_barrier(0x2, 4, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x2, 4 * AHEAD, 0);
            }
            slot = slot + 1 == ST ? 0 : slot + 1;
        }
        __builtin_amdgcn_s_waitcnt(0x0f70);  // nothing may still be written into this LDS when it is given to others
    }
    // lane: row m = .. + li, columns n = .. + 4 q + r
    const bool quad = (a.ldo & 3) == 0 && (reinterpret_cast<uintptr_t>(a.out) & 15) == 0;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t m = m0 + wm * (BM / WM) + i * 16 + li;
        if (m >= a.M) continue;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t n = n0 + wn * (BN / WN) + j * 16 + q * 4;
            if (n >= a.N) continue;
            if constexpr (sizeof(T) == 1) {
                if (a.wide) {
                    const int v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
                    store_four(static_cast<int*>(a.out) + ((int64_t)z * a.M + m) * a.ldo + n, v, quad, a.N - n);
                } else {
                    const TokenScale by(a.by_m[m]);
                    float v[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[r] = by.result(acc[i][j][r], a.by_n[min(n + r, a.N - 1)]);
                    store_four_as(a.out, m * a.ldo + n, a.dtype, v, quad, a.N - n);
                }
            } else {
                const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
                if (a.wide) {
                    store_four(static_cast<float*>(a.out) + ((int64_t)z * a.M + m) * a.ldo + n, v, quad, a.N - n);
                } else {
                    const float by = __is_same(T, f16) && SC == 0 && a.by_m ? a.by_m[m] : 1.f;
                    const T w[4] = {Elem<T>::down(v[0] * by), Elem<T>::down(v[1] * by), Elem<T>::down(v[2] * by), Elem<T>::down(v[3] * by)};
                    store_four(static_cast<T*>(a.out) + m * a.ldo + n, w, quad, a.N - n);
                }
            }
        }
    }
}

}  // namespace idkm

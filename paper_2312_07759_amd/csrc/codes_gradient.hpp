// Gradients of a product with a coded layer in its group scales and its codebook, from P[n, c] = sum_t dY[t, n] X[t, c]:
//   dS[n, g] = sum over the group's columns of P[n, c] C[code, x]        (x = c mod d)
//   dC[j, x] = sum over all (n, c) with that codeword and component of S[n, g] P[n, c]
// P is read once (float32).  A wavefront takes some groups of a row at a time, `lanes` columns a step;
// lanes is a multiple of d, so a lane always has the same component x.  It keeps bins of its own for the codewords in LDS
// ([codeword][lane], a bank to a lane): no two lanes ever add to the same word, and the order of every sum is fixed.
// A workgroup's bins go to `bins` [k d][workgroup]; k_join_gradients adds them up in float64.
// Bound by reading P: STEPS of them are asked for before the first is used.
#pragma once
#include "codes_dense.hpp"

namespace idkm {

struct BinArgs {
    const uint32_t* words;
    int64_t nwords;
    int64_t rows, cols;
    const void* C;
    int k, d, bits;
    const float* S;     // [rows, groups] or null
    int group, groups;  // groups of some hundred columns where there are no scales
    const float* P;     // [count][ldp], rows [first, first + count) of the layer
    int64_t ldp, first, count;
    float* dS;        // [rows, groups] or null
    float* segments;  // [rows][ceil(cols / 32)], or null: see k_codes_bins_runs
    float* bins;  // [k d][pitch] or null, this launch's workgroups from `at` on
    int64_t pitch, at;
    int code0, codes;  // codewords binned by this launch
    int lanes;         // of a wavefront that take part: a multiple of d
    int run;           // groups of a row that a wavefront takes at a time
    int c_in_lds;
    unsigned group_magic;  // ceil(2^31 / (group / 32)) where a row has several groups, which are multiples of 32; 0 for one
    __device__ __forceinline__ int group_of(int c) const {  // a division would be half of a column's instructions
        const unsigned x = (unsigned)c >> 5;
        unsigned g = __umulhi(2u * x, group_magic);
        if (__umul24(g, (unsigned)group >> 5) > x) --g;  // the rounded-up inverse is off by one at most, and then too large; both below 2^17
        return (int)g;
    }
    // LISTED: P's row i belongs to the layer's row listed[i], for *listed_count rows; `segments` has a row for each of them
    const int32_t* listed;
    const int32_t* listed_count;
    __device__ __forceinline__ int64_t row_of(int64_t rr, bool of_list) const { return of_list ? (int64_t)listed[rr] : first + rr; }
    __device__ __forceinline__ int64_t rows_here(bool of_list) const { return of_list ? (int64_t)*listed_count : count; }
};

// The sum over a lane's aligned neighbours, `lanes` of them, a power of two.  Up to 16 without LDS: once the lanes of a half agree, a mirrored one is as good
// as the other half's.
__device__ __forceinline__ float sum_of_lanes(float v, int lanes) {
    auto moved = [&](auto control) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(control)::value, 0xf, 0xf, true));
    };
    if (lanes >= 2) v += moved(std::integral_constant<int, 0xb1>());   // lanes 1 0 3 2 of four
    if (lanes >= 4) v += moved(std::integral_constant<int, 0x4e>());   // 2 3 0 1
    if (lanes >= 8) v += moved(std::integral_constant<int, 0x141>());  // eight, mirrored
    if (lanes >= 16) v += moved(std::integral_constant<int, 0x140>()); // sixteen, mirrored
    if (lanes >= 32) v += __shfl_xor(v, 16);
    if (lanes >= 64) v += __shfl_xor(v, 32);
    return v;
}

template <typename T, bool LISTED>
__global__ __launch_bounds__(256) void k_codes_bins(const BinArgs a) {
    constexpr int STEPS = 8;
    extern __shared__ __align__(16) float bin_lds[];  // [wave][codes][64], then the codebook
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nw = blockDim.x >> 6;
    float* mine = bin_lds + wave * a.codes * 64 + lane;
    const T* C = static_cast<const T*>(a.C);
    if (a.bins)
        for (int j = 0; j < a.codes; ++j) mine[j * 64] = 0.f;
    if (a.dS && a.c_in_lds) {
        T* copy = reinterpret_cast<T*>(bin_lds + (a.bins ? nw * a.codes * 64 : 0));
        for (int i = threadIdx.x; i < a.k * a.d; i += blockDim.x) copy[i] = C[i];
        C = copy;
    }
    __syncthreads();
    const int per_row = (int)(a.cols / a.d);
    const int runs = (a.groups + a.run - 1) / a.run;  // of a row
    const int steps = (a.group + a.lanes - 1) / a.lanes;  // of a group
    const int64_t tasks = a.rows_here(LISTED) * runs;
    const int own_code = lane / a.d, x = lane - own_code * a.d;
    const int group_codes = a.group / a.d, step_codes = a.lanes / a.d;
    const uint32_t mask = (1u << a.bits) - 1u;
    const int two = a.nwords > 1 ? 1 : 0;
    for (int64_t task = (int64_t)blockIdx.x * nw + wave; task < tasks; task += (int64_t)gridDim.x * nw) {
        const int64_t rr = task / runs, r = a.row_of(rr, LISTED);
        const int g0 = (int)(task - rr * runs) * a.run, g1 = min(a.groups, g0 + a.run);
        const float* P = a.P + rr * a.ldp;
        const float* S = a.S ? a.S + r * a.groups : nullptr;
        int g = g0, j = 0;  // the step about to be asked for: group g, its j-th
        int gu = g0, ju = 0;  // .. and used
        float sum = 0.f;
        while (g < g1) {
            float p[STEPS], s[STEPS];
            uint32_t lo[STEPS], hi[STEPS];
            int sh[STEPS];
            bool there[STEPS];
#pragma unroll
            for (int u = 0; u < STEPS; ++u) {
                const bool step = g < g1;
                const int in = j * a.lanes + lane, c = step ? g * a.group + in : 0;
                there[u] = step && lane < a.lanes && in < a.group && c < a.cols;
                p[u] = P[there[u] ? c : 0];
                s[u] = S ? S[step ? g : g0] : 1.f;
                const int64_t bit = (r * per_row + (there[u] ? g * group_codes + j * step_codes + own_code : 0)) * a.bits;
                const int64_t w = min(bit >> 5, a.nwords - 1 - two);
                sh[u] = (int)(bit - (w << 5));
                lo[u] = a.words[w];
                hi[u] = a.words[w + two];
                if (step && ++j == steps) {
                    j = 0;
                    ++g;
                }
            }
#pragma unroll
            for (int u = 0; u < STEPS; ++u) {
                if (gu >= g1) break;
                const uint32_t code = (uint32_t)(((uint64_t)hi[u] << 32 | lo[u]) >> sh[u]) & mask;
                if (a.dS && there[u]) sum = fmaf(p[u], code < (uint32_t)a.k ? Elem<T>::up(C[(int)code * a.d + x]) : __builtin_nanf(""), sum);
                const int b = (int)code - a.code0;
                if (a.bins && there[u] && b >= 0 && b < a.codes) {
                    mine[b * 64] += s[u] * p[u];
                }
                if (++ju == steps) {
                    if (a.dS) {
#pragma unroll
                        for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
                        if (lane == 0) a.dS[r * a.groups + gu] = sum;
                        sum = 0.f;
                    }
                    ju = 0;
                    ++gu;
                }
            }
        }
    }
    if (!a.bins) return;
    __syncthreads();
    // component i of codeword j: the lanes i, i + d, ..
    for (int e = threadIdx.x; e < a.codes * a.d; e += blockDim.x) {
        const int j = e / a.d, i = e - j * a.d;
        if (a.code0 + j >= a.k) continue;
        double sum = 0.0;
        for (int w = 0; w < nw; ++w)
            for (int l = i; l < a.lanes; l += a.d) sum += (double)bin_lds[(w * a.codes + j) * 64 + l];
        a.bins[((a.code0 + j) * a.d + i) * a.pitch + a.at + blockIdx.x] = (float)sum;
    }
}

// The same for codes of up to 8 bits, D in {1, 2, 4, 8} and small codebooks: a lane takes 8 consecutive columns at a time and
// keeps bins for all k D components.  Ten instructions a column instead of some 75, which bound the kernel above (4096 x 4096, k = 16:
// 127 us; this one 23, of which P at the rate of a copy is 13).  dS: lanes of a group are added up where they are a power of two of at most 64, otherwise sums of 32 columns go to
// `segments`, which k_join_gradients adds up.
template <typename T, int D, bool LISTED>
__global__ __launch_bounds__(256) void k_codes_bins_runs(const BinArgs a) {
    constexpr int NC = 8 / D;
    extern __shared__ __align__(16) float bin_lds[];  // [wave][k D][64], then the codebook
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nw = blockDim.x >> 6;
    const int kd = a.k * D;
    float* mine = bin_lds + wave * kd * 64 + lane;
    float* book = bin_lds + (a.bins ? nw * kd * 64 : 0);
    if (a.bins)
        for (int j = 0; j < kd; ++j) mine[j * 64] = 0.f;
    for (int i = threadIdx.x; i < kd; i += blockDim.x) book[i] = Elem<T>::up(static_cast<const T*>(a.C)[i]);
    __syncthreads();
    const int strips = (int)((a.cols + 511) / 512), per_row = (int)(a.cols / D);
    const int64_t step = (int64_t)gridDim.x * nw;
    const uint32_t mask = (1u << a.bits) - 1u;
    const int group_lanes = a.group / 8;
    int64_t rr = ((int64_t)blockIdx.x * nw + wave) / strips;
    int strip = (int)((int64_t)blockIdx.x * nw + wave - rr * strips);
    const int64_t rows_step = step / strips;
    const int strips_step = (int)(step - rows_step * strips);
    struct Item {
        float p[8], s;
        uint32_t w[3];
        int sh;
    };
    const int64_t count = a.rows_here(LISTED);
    auto ask = [&](Item& t, int64_t row, int of) {
        const int64_t r = a.row_of(row, LISTED);
        const int at = min(of * 512 + lane * 8, (int)(a.cols - 1) & ~7);  // lanes behind the last column read it and do not count
        const float* P = a.P + row * a.ldp + at;  // ldp is a multiple of 8
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const floatx4 v = reinterpret_cast<const floatx4*>(P)[h];
#pragma unroll
            for (int e = 0; e < 4; ++e) t.p[h * 4 + e] = v[e];
        }
        // up to 64 bits of codes, in three words; near the stream's end the words are taken from further ahead
        const int64_t bit = (r * per_row + at / D) * a.bits, from = min(bit >> 5, a.nwords - 3);
        t.sh = (int)(bit - (from << 5));
#pragma unroll
        for (int i = 0; i < 3; ++i) t.w[i] = a.words[from + i];
        t.s = a.S ? a.S[r * a.groups + a.group_of(at)] : 1.f;
    };
    Item now, next;
    if (rr < count) ask(now, rr, strip);
    while (rr < count) {
        int64_t rn = rr + rows_step;
        int sn = strip + strips_step;
        if (sn >= strips) {
            sn -= strips;
            ++rn;
        }
        if (rn < count) ask(next, rn, sn);
        const int64_t r = a.row_of(rr, LISTED);
        const int c = strip * 512 + lane * 8;
        const bool there = c < a.cols;
        const int have = there ? min(8, (int)a.cols - c) : 0;
        const float* p = now.p;
        const float s = now.s;
        const int sh = now.sh;
        const uint32_t b0 = sh < 32 ? now.w[0] : sh < 64 ? now.w[1] : now.w[2], b1 = sh < 32 ? now.w[1] : sh < 64 ? now.w[2] : 0u,
                       b2 = sh < 32 ? now.w[2] : 0u;
        uint32_t low = __builtin_amdgcn_alignbit(b1, b0, sh & 31), high = __builtin_amdgcn_alignbit(b2, b1, sh & 31);
        float sum = 0.f;
        // sure: all eight columns are there and every code is one; word: the codes lie in 32 bits
        auto add = [&](auto sure_, auto word_) {
            constexpr bool sure = decltype(sure_)::value, word = decltype(word_)::value;
#pragma unroll
            for (int e = 0; e < NC; ++e) {
                const uint32_t code = word ? __builtin_amdgcn_ubfe(low, e * a.bits, a.bits) : low & mask;
                if (!word) {
                    low = __builtin_amdgcn_alignbit(high, low, a.bits);
                    high >>= a.bits;
                }
                const bool none = !sure && code >= (uint32_t)a.k;
                const int j = none ? 0 : (int)code * D;
#pragma unroll
                for (int i = 0; i < D; ++i) {
                    const bool counts = sure || e * D + i < have;
                    if (a.dS) {
                        const float w = none ? __builtin_nanf("") : book[j + i];
                        sum = counts ? fmaf(p[e * D + i], w, sum) : sum;
                    }
                    if (a.bins) mine[(j + i) * 64] += counts && !none ? s * p[e * D + i] : 0.f;
                }
            }
        };
        const bool sure = strip * 512 + 512 <= a.cols && a.k > (int)mask;
        if (sure && NC * a.bits <= 32) add(std::true_type(), std::true_type());
        else if (sure) add(std::true_type(), std::false_type());
        else add(std::false_type(), std::false_type());
        if (a.segments) {
            sum = sum_of_lanes(sum, 4);
            if (there && (lane & 3) == 0) a.segments[(LISTED ? rr : r) * ((a.cols + 31) / 32) + (c >> 5)] = sum;
        } else if (a.dS) {
            sum = sum_of_lanes(sum, group_lanes);
            if (there && (lane & (group_lanes - 1)) == 0) a.dS[r * a.groups + a.group_of(c)] = sum;
        }
        now = next;
        rr = rn;
        strip = sn;
    }
    if (!a.bins) return;
    __syncthreads();
    // A component's 64 bins of every wavefront go to `split` lanes, as many as there are for each: with a wavefront to one component, seven
    // exchanges for each, 200 components took some 30 us.  Lanes begin at different banks.
    int split = 64;
    while (split > 1 && split * kd > (int)blockDim.x) split >>= 1;
    const int part = threadIdx.x & (split - 1), n = 64 / split;
    for (int e0 = 0; e0 < kd; e0 += blockDim.x / split) {
        const int e = e0 + threadIdx.x / split;
        double sum = 0.0;
        for (int w = 0; w < nw && e < kd; ++w) {
            const float* of = bin_lds + (w * kd + e) * 64;
            for (int i = 0; i < n; i += 8) {
                float v[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) v[u] = of[((i + u) * split + part + e * split) & 63];
#pragma unroll
                for (int u = 0; u < 8; ++u) sum += i + u < n ? (double)v[u] : 0.0;
            }
        }
        for (int o = split / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
        if (e < kd && part == 0) a.bins[e * a.pitch + a.at + blockIdx.x] = (float)sum;
    }
}

// The same codes with larger codebooks: a lane has one component, as in the first kernel, and a wavefront takes 512 columns of a row
// in eight steps of 64; the next 512 are asked for before these are used.  dS goes through `segments` always.
// SHARE lanes have the same bins and add to them one after another: with bins for every lane, 256 codewords leave room for two wavefronts
// on a compute unit, which wait for every one of their loads (512 x 4608, k = 256, d = 4: 30 us; 18 with eight wavefronts, whose turns are then what takes longest).
template <typename T, int D, int SHARE, bool LISTED>
__global__ __launch_bounds__(256) void k_codes_bins_wide(const BinArgs a) {
    constexpr int STEPS = 8, WIDTH = 64 / SHARE;
    extern __shared__ __align__(16) float bin_lds[];  // [wave][k][WIDTH]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nw = blockDim.x >> 6;
    float* mine = bin_lds + wave * a.k * WIDTH + lane % WIDTH;
    const int turn = lane / WIDTH;
    if (a.bins)
        for (int j = lane; j < a.k * WIDTH; j += 64) bin_lds[wave * a.k * WIDTH + j] = 0.f;
    const T* C = static_cast<const T*>(a.C) + lane % D;
    const int strips = (int)((a.cols + 511) / 512), per_row = (int)(a.cols / D), segments = (int)((a.cols + 31) / 32);
    const uint32_t mask = (1u << a.bits) - 1u;
    const int64_t step = (int64_t)gridDim.x * nw, rows_step = step / strips;
    const int strips_step = (int)(step - rows_step * strips);
    int64_t rr = ((int64_t)blockIdx.x * nw + wave) / strips;
    int strip = (int)((int64_t)blockIdx.x * nw + wave - rr * strips);
    struct Batch {
        float p[STEPS], s[STEPS];
        uint32_t lo[STEPS], hi[STEPS];
        int sh[STEPS];
    };
    const int64_t count = a.rows_here(LISTED);
    auto ask = [&](Batch& t, int64_t row, int at) {
        const int64_t r = a.row_of(row, LISTED), bit0 = (r * per_row + at * (512 / D)) * a.bits;
        const uint32_t* words = a.words + (bit0 >> 5);
        const int limit = (int)min(a.nwords - 2 - (bit0 >> 5), (int64_t)1 << 30);  // at least -1: a word is there
        const float* P = a.P + row * a.ldp;
        const float* S = a.S ? a.S + r * a.groups : nullptr;
#pragma unroll
        for (int u = 0; u < STEPS; ++u) {
            const int c = min(at * 512 + u * 64 + lane, (int)a.cols - 1);  // columns behind the last: read as it, not counted
            t.p[u] = P[c];
            t.s[u] = S ? S[a.group_of(c)] : 1.f;
            const int bit = (int)(bit0 & 31) + min(u * (64 / D) + lane / D, per_row - 1 - at * (512 / D)) * a.bits;
            const int from = min(bit >> 5, limit);
            t.sh[u] = bit - from * 32;
            t.lo[u] = words[from];
            t.hi[u] = words[from + 1];
        }
    };
    Batch now, next;
    if (rr < count) ask(now, rr, strip);
    while (rr < count) {
        int64_t rn = rr + rows_step;
        int sn = strip + strips_step;
        if (sn >= strips) {
            sn -= strips;
            ++rn;
        }
        if (rn < count) ask(next, rn, sn);
        uint32_t code[STEPS];
        float w[STEPS];
#pragma unroll
        for (int u = 0; u < STEPS; ++u) {
            code[u] = (uint32_t)(((uint64_t)now.hi[u] << 32 | now.lo[u]) >> now.sh[u]) & mask;
            if (a.segments) w[u] = Elem<T>::up(C[code[u] < (uint32_t)a.k ? code[u] * D : 0]);
        }
        if (a.bins) {
#pragma unroll
            for (int u = 0; u < STEPS; ++u) {
                const bool none = code[u] >= (uint32_t)a.k, counts = strip * 512 + u * 64 + lane < a.cols;
                const float v = counts && !none ? now.s[u] * now.p[u] : 0.f;
#pragma unroll
                for (int t = 0; t < SHARE; ++t) {
                    if (turn == t) mine[(none ? 0 : code[u]) * WIDTH] += v;
                    asm volatile("" ::: "memory");  // one turn after another
                }
            }
        }
        if (a.segments) {
            // Sums over 32 lanes of eight steps: lanes exchange the half of their values that the other one goes on with, so that a lane
            // ends with one step's sum after nine exchanges instead of forty.
#pragma unroll
            for (int u = 0; u < STEPS; ++u) {
                const bool counts = strip * 512 + u * 64 + lane < a.cols;
                w[u] = counts ? now.p[u] * (code[u] < (uint32_t)a.k ? w[u] : __builtin_nanf("")) : 0.f;
            }
#pragma unroll
            for (int o = 16, half = 4; half > 0; o >>= 1, half >>= 1) {
                const bool upper = lane & o;
#pragma unroll
                for (int i = 0; i < half; ++i) {
                    const float send = upper ? w[i] : w[i + half], keep = upper ? w[i + half] : w[i];
                    w[i] = keep + __shfl_xor(send, o);
                }
            }
            w[0] += __shfl_xor(w[0], 2);
            w[0] += __shfl_xor(w[0], 1);
            const int u = (lane >> 4 & 1) * 4 + (lane >> 3 & 1) * 2 + (lane >> 2 & 1), c = strip * 512 + u * 64 + (lane & 32);
            if ((lane & 3) == 0 && c < a.cols) a.segments[(LISTED ? rr : a.first + rr) * segments + (c >> 5)] = w[0];
        }
        now = next;
        rr = rn;
        strip = sn;
    }
    if (!a.bins) return;
    __syncthreads();
    for (int e = threadIdx.x; e < a.k * D; e += blockDim.x) {
        const int j = e / D, i = e % D;
        double sum = 0.0;
        for (int w = 0; w < nw; ++w)
            for (int l = i; l < WIDTH; l += D) sum += (double)bin_lds[(w * a.k + j) * WIDTH + (l + j * D) % WIDTH];
        a.bins[e * a.pitch + a.at + blockIdx.x] = (float)sum;
    }
}

}  // namespace idkm

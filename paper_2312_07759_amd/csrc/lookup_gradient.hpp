// Gradients of a lookup in a stored table, in the codebook and the group scales, in one pass over dY: a row's sum P[c] = alpha sum dY[t, c] stays in the
// registers of the wavefront that forms it, which reads the row's codes and scales and adds
//   S P  to its bins of the codebook's components (in LDS, those of a lane or of some lanes that take turns: the order of every sum is fixed)
//   P C[code]  over the lanes of a group: dS of the row, or of its part where the row's tokens lie in several blocks.
// For codes of up to 8 bits and D in {1, 2, 4, 8}, but for the largest codebooks with many tokens; the others write the sums P out and go through the kernels of the
// gradient of a product, as do rows of fewer than eight columns.
#pragma once
#include "codes_gradient.hpp"
#include "token_sums.hpp"

namespace idkm {

struct LookupGradArgs {
    TokenIds ids;
    TokenOrder order;  // up to FEW_TOKENS tokens: row_at[t] is written, the row of the first token of each row (`rows`: of others)
    int few;
    float alpha;
    const void* dY;  // T [n, ldy]
    int64_t ldy;
    int cols;
    const uint32_t* words;
    int64_t nwords, row_bits;
    const void* C;  // T [k, D]
    int k, bits;
    const float* S;  // [rows, groups] or null
    int group, groups;
    float* dS;     // [rows, groups] or null
    float* parts;  // [n][per_part]: of the row or part that ends at a place (few: of a row's first token); segments of 32 columns, or groups
    int per_part;
    int segmented;  // every row's go to `parts`: a group is not a power of two of lanes
    float* bins;    // [k D][pitch]
    int64_t pitch;
    int each;          // places to a block, at most LOOKUP_PLACES
    int sums_log;      // sums of groups (segments) that a row has in a strip of 512 columns: 1 << sums_log, at most 16
    int width_log;     // lanes with bins of their own: 1 << width_log
    unsigned summing;  // few: workgroups that sum; the ones behind them clear the other rows of dS
};

constexpr int LOOKUP_PLACES = 32;
constexpr int LOOKUP_KEPT = LOOKUP_PLACES * 17;  // words of LDS for a wavefront: sums of groups, and whose they are

// 8192 tokens of 4096 columns, 4 bits, groups of 128, bfloat16: 21.5 us, where dY alone is 13 at the rate of a copy.  Bound by issue and by the turns of the bins: some
// 5,100 sums of rows and parts of rows, 42,000 strips of 512 columns at about 100 vector and as many scalar instructions, and eight LDS updates one after
// another in each.  Beginning and end take 6 us (bins cleared and added up), as many wavefronts as the registers allow the rest.
// A strip's sums of groups are kept in LDS and stored at the block's end, so that no load waits behind a store.
// SHARED: 64 >> width_log lanes have the same bins and add to them one after another: the bins of larger codebooks leave room for more wavefronts then, see
// lookup_grad_plan.  A code's D bins of a lane lie together and are read and written at once.
template <typename T, int D, bool FEW, bool SHARED>
__global__ __launch_bounds__(256) void k_lookup_gradient(const LookupGradArgs a) {
    constexpr int NC = 8 / D, WORD = 1, SURE = 2, SCALED = 4, SUMS = 8;
    struct alignas(4 * D) Code { float part[D]; };
    extern __shared__ __align__(16) float bin_lds[];  // [wave][k][width][D], then the codebook
    const int width_log = SHARED ? a.width_log : 6, width = 1 << width_log;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nw = blockDim.x >> 6;
    if (FEW && blockIdx.x >= a.summing) {
        if (a.dS) clear_other_rows(a.ids, a.dS, a.groups, (int64_t)(blockIdx.x - a.summing) * nw + wave, (int64_t)(gridDim.x - a.summing) * nw);
        return;
    }
    const int kd = a.k * D;
    Code* mine = reinterpret_cast<Code*>(bin_lds + (wave * kd << width_log)) + (lane & (width - 1));
    float* book = bin_lds + (nw * kd << width_log);
    const int turn = lane >> width_log;
    float* kept = book + kd + wave * LOOKUP_KEPT;
    int* kept_for = reinterpret_cast<int*>(kept + LOOKUP_PLACES * 16);  // a row of dS, or ~ a place of `parts`
    for (int i = lane; i < kd << (width_log - 2); i += 64) reinterpret_cast<floatx4*>(bin_lds + (wave * kd << width_log))[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int i = threadIdx.x; i < kd; i += blockDim.x) book[i] = Elem<T>::up(static_cast<const T*>(a.C)[i]);
    __syncthreads();
    const int strips = (a.cols + 511) / 512, n = (int)a.ids.n;
    const int blocks = FEW ? n : (n + a.each - 1) / a.each;
    const uint32_t mask = (1u << a.bits) - 1u;
    // without scales some word is read in their place, so that every row makes the same loads
    const float* S = a.S ? a.S : reinterpret_cast<const float*>(a.words);
    const int groups = a.S ? a.groups : 0;
    const int sum_lanes = a.segmented ? 4 : min(64, a.group / 8), lanes_log = 31 - __builtin_clz(sum_lanes);
    // a row's codes and scale of the lane's columns
    struct Item {
        uint32_t w[3];
        int sh;
        float s;
    };
    for (int task = blockIdx.x * nw + wave; task < blocks * strips; task += (int)a.summing * nw) {
        const int b = task / strips, strip = task - b * strips;
        const Columns columns(strip, a.cols);
        const int skip = columns.skip, at_bit = columns.c / D * a.bits, g = a.S ? min(columns.c + skip, a.cols - 1) / a.group : 0;
        const int g_first = strip * 512 / a.group;
        int held = 0;
        // sure: all eight columns are there and every code is one; word: the codes lie in 32 bits
        const bool sure = strip * 512 + 512 <= a.cols && a.k > (int)mask;
        const int form = (sure ? NC * a.bits <= 32 ? WORD : SURE : 0) | (a.S ? SCALED : 0) | (a.dS ? SUMS : 0);
        // word: of the stream, where the row's words begin; row_sh: its codes' bit there; near: three words from a lane's first one on may not be there, and
        // are taken from further ahead
        auto ask = [&](Item& t, const uint32_t* word, int row_sh, bool near, const float* scale) {
            const int bit = row_sh + at_bit;
            int from = bit >> 5;
            if (near) from = min(from, (int)(a.words + (a.nwords - 3) - word));
            t.sh = bit - from * 32;
            const u32x3_word w = *reinterpret_cast<const u32x3_word*>(word + from);
#pragma unroll
            for (int i = 0; i < 3; ++i) t.w[i] = w[i];
            t.s = scale[g];
        };
        auto finish = [&](const Item& t, int who, const float* p) {
            // looked at anew for every row: the conditions and shifts that follow from them would take more scalar registers than there are
            int how = form, bits = a.bits, lanes = sum_lanes;
            asm volatile("" : "+s"(how), "+s"(bits), "+s"(lanes));
            uint32_t b0 = t.w[0], b1 = t.w[1], b2 = t.w[2];
            if (__any(t.sh >= 32)) {  // only near the stream's end
                const bool two = t.sh >= 64, one = t.sh >= 32;
                b0 = two ? b2 : one ? b1 : b0;
                b1 = two ? 0u : one ? b2 : b1;
                b2 = one ? 0u : b2;
            }
            uint32_t low = __builtin_amdgcn_alignbit(b1, b0, t.sh & 31), high = __builtin_amdgcn_alignbit(b2, b1, t.sh & 31);
            const float by = how & SCALED ? a.alpha * t.s : a.alpha;
            float sum = 0.f;
            auto add = [&](auto sure_, auto word_) {
                constexpr bool sure = decltype(sure_)::value, word = decltype(word_)::value;
                int place[NC];
#pragma unroll
                for (int e = 0; e < NC; ++e) {
                    const uint32_t code = word ? __builtin_amdgcn_ubfe(low, e * bits, bits) : low & mask;
                    if (!word) {
                        low = __builtin_amdgcn_alignbit(high, low, bits);
                        high >>= bits;
                    }
                    const bool none = !sure && code >= (uint32_t)a.k, counts = sure || e * D >= skip;  // skip is a multiple of D
                    const int j = none ? 0 : (int)code;
                    const Code w = reinterpret_cast<const Code*>(book)[j];
#pragma unroll
                    for (int i = 0; i < D; ++i) sum = counts ? fmaf(p[e * D + i], none ? __builtin_nanf("") : w.part[i], sum) : sum;
                    place[e] = counts && !none ? j << width_log : -1;
                }
                if constexpr (!SHARED) {
#pragma unroll
                    for (int e = 0; e < NC; ++e) {
                        const bool there = sure || place[e] >= 0;
                        Code bin = mine[there ? place[e] : 0];
#pragma unroll
                        for (int i = 0; i < D; ++i) bin.part[i] = there ? fmaf(by, p[e * D + i], bin.part[i]) : bin.part[i];
                        mine[there ? place[e] : 0] = bin;
                    }
                }
                if constexpr (SHARED) {
                    for (int t = 0; t < 64 >> width_log; ++t) {
                        if (turn == t) {
#pragma unroll
                            for (int e = 0; e < NC; ++e) {
                                if (!sure && place[e] < 0) continue;
                                Code bin = mine[place[e]];
#pragma unroll
                                for (int i = 0; i < D; ++i) bin.part[i] = fmaf(by, p[e * D + i], bin.part[i]);
                                mine[place[e]] = bin;
                            }
                        }
                        // one turn after another
                        __builtin_amdgcn_wave_barrier();
                        asm volatile("" ::: "memory");
                    }
                }
            };
            if (how & WORD) add(std::true_type(), std::true_type());
            else if (how & SURE) add(std::true_type(), std::false_type());
            else add(std::false_type(), std::false_type());
            if (!(how & SUMS)) return;
            sum *= a.alpha;
            sum = sum_of_lanes(sum, lanes);
            if ((lane & (sum_lanes - 1)) == 0 && lane >> lanes_log < 1 << a.sums_log) kept[held << a.sums_log | lane >> lanes_log] = sum;
            if (lane == 0) kept_for[held] = who;
            ++held;
        };
        auto store_kept = [&] {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            const int g0 = (a.segmented ? strip * 16 : g_first), all = a.segmented ? a.per_part : a.groups;
            for (int i = lane; i < held << a.sums_log; i += 64) {
                const int f = i >> a.sums_log, of = g0 + (i & ((1 << a.sums_log) - 1)), who = kept_for[f];
                if (of < all) (who >= 0 ? a.dS + (int64_t)who * a.groups : a.parts + (int64_t)~who * a.per_part)[of] = kept[i];
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        };
        if constexpr (FEW) {
            const Mates::Rows rows(a.ids);
            const int row = a.ids.row(b);  // the same for all lanes
            const Mates mates(rows, row);
            const bool first = row < a.ids.rows && mates.first() == b;
            if (strip == 0 && lane == 0) a.order.row_at[b] = first ? row : a.ids.rows;
            if (!first) continue;
            Item t;
            const int64_t row_bit = row * a.row_bits;
            ask(t, a.words + (row_bit >> 5), (int)(row_bit & 31), (row_bit + a.row_bits + 31) / 32 + 3 > a.nwords, S + (int64_t)row * groups);
            float sum[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = 0.f;
            sum_of_mates<T, false>(sum, mates, static_cast<const T*>(a.dY), a.ldy, columns.c, a.cols);
            finish(t, a.segmented ? ~b : row, sum);
            if (a.dS) store_kept();
        } else {
            const Places places(a.order, n, a.ids.rows, b, a.each);
            const int row = min(places.row, a.ids.rows - 1);
            const int64_t row_bit = row * a.row_bits;
            const uint64_t word = reinterpret_cast<uint64_t>(a.words + (row_bit >> 5)), scale = reinterpret_cast<uint64_t>(S + (int64_t)row * groups);
            // the row's bit, and whether its last word but two ends behind the stream
            const int start = (int)(row_bit & 31) | ((row_bit + a.row_bits + 31) / 32 + 3 > a.nwords ? 32 : 0);
            sum_places_of<T, false, Item>(
                places, static_cast<const T*>(a.dY), a.ldy, columns.c, a.cols,
                [&](Item& t, int p) {
                    const int at = __builtin_amdgcn_readlane(start, p);
                    ask(t, of_lane<uint32_t>(word, p), at & 31, at & 32, of_lane<float>(scale, p));
                },
                [&](const Item& t, int p, bool complete, bool, const float* sum) {
                    finish(t, complete && !a.segmented ? __builtin_amdgcn_readlane(places.row, p) : ~(int)(places.first + p), sum);
                });
            if (a.dS) store_kept();
        }
    }
    __syncthreads();
    // A component's bins to as many lanes as there are; components of different codes begin with different lanes' bins
    int split_log = width_log;
    while (split_log > 0 && kd << split_log > (int)blockDim.x) --split_log;
    const int part = threadIdx.x & ((1 << split_log) - 1), count = width >> split_log;
    for (int e0 = 0; e0 < kd; e0 += blockDim.x >> split_log) {
        const int e = e0 + (threadIdx.x >> split_log), j = e / D;
        double sum = 0.0;
        for (int i = 0; i < count && e < kd; i += 4) {
            float v[4][4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int at = (((j << width_log) + ((((i + u) << split_log) + part + j) & (width - 1))) * D) + (e - j * D);
#pragma unroll
                for (int w = 0; w < 4; ++w) v[u][w] = w < nw ? bin_lds[(w * kd << width_log) + at] : 0.f;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i + u < count) sum += ((double)v[u][0] + (double)v[u][1]) + ((double)v[u][2] + (double)v[u][3]);
        }
        for (int o = 1 << split_log >> 1; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
        if (e < kd && part == 0) a.bins[e * a.pitch + blockIdx.x] = (float)sum;
    }
}

}  // namespace idkm

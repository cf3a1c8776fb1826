// Gradients of a lookup in a stored table, in the codebook and the group scales, in one pass over dY: a row's sum P[c] = alpha sum dY[t, c] stays in the
// registers of the wavefront that forms it, which reads the row's codes and scales and adds
//   S P  to its bins of the codebook's components (in LDS, 64 for each, one to a lane: no two lanes add to the same word, and the order of every sum is fixed)
//   P C[code]  over the lanes of a group: dS of the row, or of its part where the row's tokens lie in several blocks.
// For codes of up to 8 bits, D in {1, 2, 4, 8} and codebooks of up to 256 components; the others write the sums P out and go through the kernels of the
// gradient of a product.
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
    int each;          // places to a block
    unsigned summing;  // few: workgroups that sum; the ones behind them clear the other rows of dS
};

template <typename T, int D, bool FEW>
__global__ __launch_bounds__(256) void k_lookup_gradient(const LookupGradArgs a) {
    constexpr int NC = 8 / D;
    extern __shared__ __align__(16) float bin_lds[];  // [wave][k D][64], then the codebook
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nw = blockDim.x >> 6;
    if (FEW && blockIdx.x >= a.summing) {
        if (a.dS) clear_other_rows(a.ids, a.dS, a.groups, (int64_t)(blockIdx.x - a.summing) * nw + wave, (int64_t)(gridDim.x - a.summing) * nw);
        return;
    }
    const int kd = a.k * D;
    float* mine = bin_lds + wave * kd * 64 + lane;
    float* book = bin_lds + nw * kd * 64;
    for (int j = 0; j < kd; ++j) mine[j * 64] = 0.f;
    for (int i = threadIdx.x; i < kd; i += blockDim.x) book[i] = Elem<T>::up(static_cast<const T*>(a.C)[i]);
    __syncthreads();
    const int strips = (a.cols + 511) / 512, n = (int)a.ids.n;
    const int blocks = FEW ? n : (n + a.each - 1) / a.each;
    const uint32_t mask = (1u << a.bits) - 1u;
    const int group_lanes = a.group / 8;
    // a row's codes and scale of the lane's columns
    struct Item {
        uint32_t w[3];
        int sh;
        float s;
    };
    for (int task = blockIdx.x * nw + wave; task < blocks * strips; task += (int)a.summing * nw) {
        const int b = task / strips, strip = task - b * strips;
        const EightColumns<T> columns(a.dY, a.ldy, strip, a.cols);
        const int c = columns.c, at = min(c, (a.cols - 1) & ~7), g = at / a.group;
        const bool there = c < a.cols, sure = strip * 512 + 512 <= a.cols && a.k > (int)mask;
        auto ask = [&](Item& t, int row) {
            const int64_t bit = row * a.row_bits + (unsigned)(at / D * a.bits), from = min(bit >> 5, a.nwords - 3);
            t.sh = (int)(bit - (from << 5));
#pragma unroll
            for (int i = 0; i < 3; ++i) t.w[i] = a.words[from + i];
            t.s = a.S ? a.S[(int64_t)row * a.groups + g] : 1.f;
        };
        auto finish = [&](const Item& t, int row, int64_t place, bool complete, const float* p) {
            uint32_t b0 = t.w[0], b1 = t.w[1], b2 = t.w[2];
            if (__any(t.sh >= 32)) {  // only near the stream's end
                const bool two = t.sh >= 64, one = t.sh >= 32;
                b0 = two ? b2 : one ? b1 : b0;
                b1 = two ? 0u : one ? b2 : b1;
                b2 = one ? 0u : b2;
            }
            uint32_t low = __builtin_amdgcn_alignbit(b1, b0, t.sh & 31), high = __builtin_amdgcn_alignbit(b2, b1, t.sh & 31);
            const float by = a.alpha * t.s;
            float sum = 0.f;
            auto add = [&](auto sure_) {  // sure: all eight columns are there and every code is one
                constexpr bool sure = decltype(sure_)::value;
                const int have = there ? min(8, a.cols - c) : 0;
#pragma unroll
                for (int e = 0; e < NC; ++e) {
                    const uint32_t code = low & mask;
                    low = __builtin_amdgcn_alignbit(high, low, a.bits);
                    high >>= a.bits;
                    const bool none = !sure && code >= (uint32_t)a.k;
                    const int j = none ? 0 : (int)code * D;
#pragma unroll
                    for (int i = 0; i < D; ++i) {
                        const bool counts = sure || e * D + i < have;
                        const float w = none ? __builtin_nanf("") : book[j + i];
                        sum = counts ? fmaf(p[e * D + i], w, sum) : sum;
                        float& bin = mine[(j + i) * 64];
                        bin = counts && !none ? fmaf(by, p[e * D + i], bin) : bin;
                    }
                }
            };
            if (sure) add(std::true_type());
            else add(std::false_type());
            if (!a.dS) return;
            sum *= a.alpha;
            if (a.segmented) {
                sum += __shfl_xor(sum, 1);
                sum += __shfl_xor(sum, 2);
                if (there && (lane & 3) == 0) a.parts[place * a.per_part + (c >> 5)] = sum;
            } else {
                for (int o = 1; o < group_lanes; o <<= 1) sum += __shfl_xor(sum, o);
                if (there && (lane & (group_lanes - 1)) == 0) (complete ? a.dS + (int64_t)row * a.groups : a.parts + place * a.per_part)[g] = sum;
            }
        };
        if constexpr (FEW) {
            const Mates::Rows rows(a.ids);
            const int row = a.ids.row(b);  // the same for all lanes
            const Mates mates(rows, row);
            const bool first = row < a.ids.rows && mates.first() == b;
            if (strip == 0 && lane == 0) a.order.row_at[b] = first ? row : a.ids.rows;
            if (!first) continue;
            Item t;
            ask(t, row);
            float sum[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = 0.f;
            sum_of_mates<T>(sum, mates, columns);
            finish(t, row, b, true, sum);
        } else {
            const Places places(a.order, n, a.ids.rows, b, a.each);
            sum_places_of<T, Item>(places, columns, ask,
                                   [&](const Item& t, int row, int64_t place, bool complete, bool, const float* p) { finish(t, row, place, complete, p); });
        }
    }
    __syncthreads();
    // A component's bins to as many lanes as there are, see k_codes_bins_runs
    int split = 64;
    while (split > 1 && split * kd > (int)blockDim.x) split >>= 1;
    const int part = threadIdx.x & (split - 1), count = 64 / split;
    for (int e0 = 0; e0 < kd; e0 += blockDim.x / split) {
        const int e = e0 + threadIdx.x / split;
        double sum = 0.0;
        for (int w = 0; w < nw && e < kd; ++w) {
            const float* of = bin_lds + (w * kd + e) * 64;
            for (int i = 0; i < count; i += 8) {
                float v[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) v[u] = of[((i + u) * split + part + e * split) & 63];
#pragma unroll
                for (int u = 0; u < 8; ++u) sum += i + u < count ? (double)v[u] : 0.0;
            }
        }
        for (int o = split / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
        if (e < kd && part == 0) a.bins[e * a.pitch + blockIdx.x] = (float)sum;
    }
}

}  // namespace idkm

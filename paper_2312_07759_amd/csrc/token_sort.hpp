// Tokens brought into the order of their rows of a table, so that a row's gradients are summed one after another, in the order of the
// tokens: row_at[p] and token_at[p] of the p-th place.  Tokens of no row (negative ids, ids >= rows) come last, with row_at = rows.
#pragma once
#include "elem.hpp"

namespace idkm {

struct TokenIds {
    const void* ids;  // int32 or int64 [n]
    int wide;         // 1: int64
    int64_t n;
    int rows;
    __device__ __forceinline__ int64_t raw(int64_t t) const {
        return wide ? static_cast<const int64_t*>(ids)[t] : (int64_t) static_cast<const int32_t*>(ids)[t];
    }
    __device__ __forceinline__ int row(int64_t t) const {
        const int64_t v = raw(t);
        return v < 0 || v >= rows ? rows : (int)v;
    }
};

struct TokenOrder {
    int32_t* row_at;    // [n]
    int32_t* token_at;  // [n]
};

// Up to RANK_TOKENS tokens: a token's place is the number of tokens that come before it, counted.  All rows lie in LDS; a workgroup places 64
// tokens, one to a lane, and its wavefronts share what they are compared with.  One launch, two vector instructions for 64 comparisons.
constexpr int RANK_TOKENS = 16384, RANK_WAVES = 16;

__device__ __forceinline__ void rank_tokens(const TokenIds& in, const TokenOrder& out, int block, int* lds) {
    const int n = (int)in.n, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int* sums = lds;                       // [RANK_WAVES][64]
    int* rows = lds + RANK_WAVES * 64;     // [n], rounded up to four
    const int padded = (n + 3) & ~3;
    for (int t = threadIdx.x; t < padded; t += RANK_WAVES * 64) rows[t] = t < n ? in.row(t) : INT32_MAX;  // behind all
    __syncthreads();
    const int t0 = block * 64, t = t0 + lane;
    const int mine = rows[min(t, n - 1)];
    const int quads = padded / 4, each = (quads + RANK_WAVES - 1) / RANK_WAVES;
    const int first = min(quads, wave * each) * 4, last = min(quads, wave * each + each) * 4;
    int count = 0;
    auto compare = [&](int from, int to, int below) {
        for (int u = from; u < to; u += 4) {
            const int4 v = *reinterpret_cast<const int4*>(rows + u);
            count += (v.x < below) + (v.y < below) + (v.z < below) + (v.w < below);
        }
    };
    // earlier tokens of the same row come before, later ones behind; this workgroup's own are compared one by one
    const int own0 = min(last, max(first, t0)), own1 = min(last, max(first, t0 + 64));
    compare(first, own0, mine + 1);
    for (int u = own0; u < own1; ++u) count += rows[u] < mine + (u < t ? 1 : 0);
    compare(own1, last, mine);
    sums[wave * 64 + lane] = count;
    __syncthreads();
    if (wave == 0 && t < n) {
        int place = 0;
#pragma unroll
        for (int w = 0; w < RANK_WAVES; ++w) place += sums[w * 64 + lane];
        out.row_at[place] = mine;
        out.token_at[place] = t;
    }
}

// More tokens: eight bits of the row at a time, the lowest first, each time in the order of the last.  A workgroup takes RADIX_BLOCK tokens; `counts`
// [256][workgroups] holds how many of them have each value of the eight bits, then where they begin.
constexpr int RADIX_BLOCK = 4096, RADIX_WAVE = RADIX_BLOCK / 4;

struct RadixPass {
    TokenIds ids;
    TokenOrder from, to;  // from: of the last pass; the first takes the tokens as they come
    int first, shift;
    int32_t* counts;
    int blocks;
    __device__ __forceinline__ int row(int64_t p) const { return first ? ids.row(p) : from.row_at[p]; }
};

}  // namespace idkm

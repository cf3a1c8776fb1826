// Tokens brought together by their rows of a table, so that a row's gradients are summed one after another, in the order of the tokens: row_at[p]
// and token_at[p] of the p-th place.  The rows come in some order that depends on them alone; tokens of no row (negative ids, ids >= rows) come last, with
// row_at = rows.
#pragma once
#include "elem.hpp"

namespace idkm {

struct TokenIds {
    const void* ids;  // int32 or int64 [n]
    int wide;         // 1: int64
    int64_t n;
    int rows;
    // without a branch: the words of an id, the higher one of an int32 its sign
    __device__ __forceinline__ int64_t raw(int64_t t) const {
        const int32_t* word = static_cast<const int32_t*>(ids) + (t << wide);
        const int32_t low = word[0], high = word[wide];
        return wide ? (int64_t)high << 32 | (uint32_t)low : (int64_t)low;
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

// Up to GROUP_TOKENS tokens, one launch: a workgroup to the rows with the same lowest eight bits (neighbouring rows, the frequent ones of a text, are in
// different ones), and one to the tokens of no row.  Each looks at all tokens, counts those of lower workgroups, which come before, and lists its own; a
// short list is ordered by counting, a long one by seven bits of the row at a time.  8192 tokens of a text: 10 us (13 where every token was compared with all others), 301: 4.5.
constexpr int GROUP_TOKENS = 16384, GROUP_WAVES = 16, GROUP_DIGITS = 128, GROUP_COUNTED = 256;
static_assert(GROUP_TOKENS <= 1 << 14, "a token and the higher bits of its row share a word");
inline size_t group_lds(int64_t n) { return 4 * (size_t)(2 * ((n + 3) & ~(int64_t)3) + 4 + GROUP_WAVES * GROUP_DIGITS + 2 * GROUP_WAVES); }

__device__ __forceinline__ void group_tokens(const TokenIds& in, const TokenOrder& out, int* lds) {
    constexpr int HELD = GROUP_TOKENS / (GROUP_WAVES * 64);
    const int n = (int)in.n, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), b = blockIdx.x;
    const int padded = (n + 3) & ~3;
    int* list = lds;                                     // [padded + 4]: the higher bits of the row, then 14 bits of the token
    int* other = lds + padded + 4;                       // [padded]
    int* hist = other + padded;                          // [GROUP_WAVES][GROUP_DIGITS]
    int* totals = hist + GROUP_WAVES * GROUP_DIGITS;     // [2][GROUP_WAVES]
    // a wavefront's tokens follow one another
    const int each = ((n + 63) / 64 + GROUP_WAVES - 1) / GROUP_WAVES, first = wave * each * 64;
    uint32_t row[HELD], high[HELD];
    if (in.wide) {
#pragma unroll
        for (int i = 0; i < HELD; ++i)
            if (i < each) {
                const u32x2 v = reinterpret_cast<const u32x2*>(in.ids)[min(first + i * 64 + lane, n - 1)];
                row[i] = v[0];
                high[i] = v[1];
            }
    } else {
#pragma unroll
        for (int i = 0; i < HELD; ++i)
            if (i < each) {
                row[i] = reinterpret_cast<const uint32_t*>(in.ids)[min(first + i * 64 + lane, n - 1)];
                high[i] = 0;
            }
    }
    int own = 0, below = 0;
#pragma unroll
    for (int i = 0; i < HELD; ++i)
        if (i < each) {
            const bool held = row[i] < (uint32_t)in.rows && high[i] == 0;
            const int bucket = first + i * 64 + lane >= n ? 512 : held ? (int)(row[i] & 255) : 256;
            own += __popcll(__ballot(bucket == b));
            below += __popcll(__ballot(bucket < b));
            row[i] = bucket == b ? row[i] >> 8 : ~0u;  // ~0: not here; of a token of no row it means nothing
            if (bucket == b && !held) row[i] = 0;
        }
    if (lane == 0) {
        totals[wave] = own;
        totals[GROUP_WAVES + wave] = below;
    }
    __syncthreads();
    int at = 0, m = 0, base = 0;
#pragma unroll
    for (int w = 0; w < GROUP_WAVES; ++w) {
        at += w < wave ? totals[w] : 0;
        m += totals[w];
        base += totals[GROUP_WAVES + w];
    }
    if (m == 0) return;
#pragma unroll
    for (int i = 0; i < HELD; ++i)
        if (i < each) {
            const uint64_t mask = __ballot(row[i] != ~0u);
            if (row[i] != ~0u) list[at + __popcll(mask & (((uint64_t)1 << lane) - 1))] = (int)(row[i] << 14) | (first + i * 64 + lane);
            at += __popcll(mask);
        }
    if (tid < 4) list[m + tid] = INT32_MAX;
    if (tid < GROUP_COUNTED) hist[tid] = 0;
    __syncthreads();
    if (b == 256) {
        for (int i = tid; i < m; i += GROUP_WAVES * 64) {
            out.row_at[base + i] = in.rows;
            out.token_at[base + i] = list[i] & (GROUP_TOKENS - 1);
        }
        return;
    }
    if (m <= GROUP_COUNTED) {
        // four threads to an entry, each counts the smaller ones in a quarter of the list; entries are all different
        const int i = tid & (GROUP_COUNTED - 1), mine = i < m ? list[i] : 0, quads = (m + 3) / 4, part = (quads + 3) / 4;
        const int from = (tid / GROUP_COUNTED) * part, to = min(quads, from + part);
        int count = 0;
        if ((wave & 3) * 64 < m)
            for (int u = from; u < to; ++u) {
                const int4 v = reinterpret_cast<const int4*>(list)[u];
                count += (v.x < mine) + (v.y < mine) + (v.z < mine) + (v.w < mine);
            }
        if (i < m && count > 0) atomicAdd(&hist[i], count);
        __syncthreads();
        if (tid < m) {
            out.row_at[base + hist[tid]] = mine >> 14 << 8 | b;
            out.token_at[base + hist[tid]] = mine & (GROUP_TOKENS - 1);
        }
        return;
    }
    const int chunks = ((m + 63) / 64 + GROUP_WAVES - 1) / GROUP_WAVES, mine0 = wave * chunks * 64;
    for (int shift = 14; shift == 14 || (in.rows >> 8) >> (shift - 14) > 0; shift += 7) {
        __syncthreads();
        for (int i = tid; i < GROUP_WAVES * GROUP_DIGITS; i += GROUP_WAVES * 64) hist[i] = 0;
        __syncthreads();
        for (int i = 0; i < chunks; ++i) {
            const int p = mine0 + i * 64 + lane;
            if (p < m) atomicAdd(&hist[wave * GROUP_DIGITS + (list[p] >> shift & (GROUP_DIGITS - 1))], 1);
        }
        __syncthreads();
        if (wave == 0) {  // two digits to a lane: where each wavefront's begin
            int sum[2] = {0, 0};
            for (int w = 0; w < GROUP_WAVES; ++w)
#pragma unroll
                for (int e = 0; e < 2; ++e) sum[e] += hist[w * GROUP_DIGITS + lane * 2 + e];
            int upto = sum[0] + sum[1];
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int left = __shfl_up(upto, o);
                if (lane >= o) upto += left;
            }
            int begin[2] = {upto - sum[0] - sum[1], upto - sum[1]};
            for (int w = 0; w < GROUP_WAVES; ++w)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int have = hist[w * GROUP_DIGITS + lane * 2 + e];
                    hist[w * GROUP_DIGITS + lane * 2 + e] = begin[e];
                    begin[e] += have;
                }
        }
        __syncthreads();
        for (int i = 0; i < chunks; ++i) {
            const int p = mine0 + i * 64 + lane;
            const bool there = p < m;
            const int entry = there ? list[p] : 0, digit = entry >> shift & (GROUP_DIGITS - 1);
            uint64_t same = __ballot(there);
#pragma unroll
            for (int bit = 0; bit < 7; ++bit) {
                const uint64_t set = __ballot(digit >> bit & 1);
                same &= digit >> bit & 1 ? set : ~set;
            }
            int* next = &hist[wave * GROUP_DIGITS + digit];
            if (there) other[*next + __popcll(same & (((uint64_t)1 << lane) - 1))] = entry;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // every lane has read where its digit's places begin
            if (there && same >> lane == 1) *next += __popcll(same);  // the last lane of its kind
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        int* swap = list;
        list = other;
        other = swap;
    }
    __syncthreads();
    for (int i = tid; i < m; i += GROUP_WAVES * 64) {
        out.row_at[base + i] = list[i] >> 14 << 8 | b;
        out.token_at[base + i] = list[i] & (GROUP_TOKENS - 1);
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

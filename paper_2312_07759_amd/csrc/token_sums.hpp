// Sums of rows of dY over the tokens of one row of a table: who has to be summed, and the rows asked for ahead.
//
// A wavefront takes 512 columns, eight to a lane.  Up to FEW_TOKENS tokens: a wavefront to a token, which compares all tokens' rows with its own (a
// vector load and a comparison for 64), leaves if an earlier token has the same row, and otherwise sums those that do; nothing is sorted.  More:
// a wavefront to `each` places of the sorted tokens; a row whose places lie in several blocks is summed in parts.
#pragma once
#include "token_sort.hpp"

namespace idkm {

// Tokens of a text, taken so and sorted: 301 of float32, 734 columns, k = 100, d = 2 13.6 us and 17.9; bfloat16, 4096 columns, k = 16 16 and 17.7; a table of
// 32000 x 1024 22.6 and 29.3.  512 of them: 15.2 and 18.5, 18.1 and 17.7, 24.2 and 29.9; 1024, when that was measured, 29 and 21, 33 and 21, 27 and 31.  One row's
// tokens follow one another here, 0.07 us each: 512 of the same row take 49 us, and 17 to 33 sorted.
constexpr int FEW_TOKENS = 512;

// A lane's eight columns of rows of dY, from column c on.  The last lane of a row whose length is no multiple of eight takes the last eight columns, of which
// the first `skip` are its neighbour's: all rows are read in the same way, 16 bytes at a time.  Lanes behind the row's end skip all eight.  NARROW: rows of
// fewer than eight columns, element by element.
struct Columns {
    int c, skip;
    __device__ __forceinline__ Columns(int strip, int cols) {
        const int from = strip * 512 + (int)(threadIdx.x & 63) * 8;
        c = max(0, min(from, cols - 8));
        skip = from >= cols ? 8 : from - c;
    }
};

// .. of a few rows on their way.
template <typename T, int U, bool NARROW>
struct RowsAhead {
    static constexpr int FR = 8 / Elem<T>::PER16;
    u32x4 raw[U][FR];
    // row: the same for all lanes
    __device__ __forceinline__ void ask(int u, const T* row, unsigned c, int cols) {
        if constexpr (NARROW) {
            struct alignas(16) Eight { T v[8]; } y;
#pragma unroll
            for (int e = 0; e < 8; ++e) y.v[e] = e < cols ? row[e] : (T)0.f;
            __builtin_memcpy(raw[u], &y, sizeof(y));
        } else {
#pragma unroll
            for (int f = 0; f < FR; ++f) raw[u][f] = *reinterpret_cast<const u32x4_any*>(reinterpret_cast<const char*>(row) + (c * (unsigned)sizeof(T) + f * 16));
        }
    }
    __device__ __forceinline__ void add(int u, float* sum) const {
        struct alignas(16) Eight { T v[8]; } y;
        __builtin_memcpy(&y, raw[u], sizeof(y));
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += Elem<T>::up(y.v[e]);
    }
    __device__ __forceinline__ void begin(int u, float* sum) const {
        struct alignas(16) Eight { T v[8]; } y;
        __builtin_memcpy(&y, raw[u], sizeof(y));
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = Elem<T>::up(y.v[e]);
    }
};

// Tokens with the same row, out of up to FEW_TOKENS: one bit for each, 64 to a word.
struct Mates {
    uint64_t word[FEW_TOKENS / 64];
    // the rows of the lane's tokens, one of every 64
    struct Rows {
        int of[FEW_TOKENS / 64];
        __device__ __forceinline__ explicit Rows(const TokenIds& ids) {
            const int lane = threadIdx.x & 63;
#pragma unroll
            for (int j = 0; j < FEW_TOKENS / 64; ++j) of[j] = j * 64 + lane < (int)ids.n ? ids.row(j * 64 + lane) : -1;
        }
    };
    __device__ __forceinline__ Mates(const Rows& rows, int row) {
#pragma unroll
        for (int j = 0; j < FEW_TOKENS / 64; ++j) word[j] = __ballot(rows.of[j] == row);
    }
    __device__ __forceinline__ bool any() const {
        uint64_t all = 0;
#pragma unroll
        for (int j = 0; j < FEW_TOKENS / 64; ++j) all |= word[j];
        return all != 0;
    }
    __device__ __forceinline__ int count() const {
        int n = 0;
#pragma unroll
        for (int j = 0; j < FEW_TOKENS / 64; ++j) n += __popcll(word[j]);
        return n;
    }
    // the i-th token, another one for each lane; i < count()
    __device__ __forceinline__ int at(int i) const {
        uint64_t of = word[0];
        int base = 0;
#pragma unroll
        for (int j = 0; j + 1 < FEW_TOKENS / 64; ++j) {
            const int before = __popcll(word[j]);
            const bool on = base == j * 64 && i >= before;
            i -= on ? before : 0;
            of = on ? word[j + 1] : of;
            base += on ? 64 : 0;
        }
        const int low = __popc((uint32_t)of);
        const bool high = i >= low;
        uint32_t bits = high ? (uint32_t)(of >> 32) : (uint32_t)of;
        i -= high ? low : 0;
        base += high ? 32 : 0;
#pragma unroll
        for (int half = 16; half > 0; half >>= 1) {
            const int before = __popc(bits & ((1u << half) - 1u));
            const bool on = i >= before;
            i -= on ? before : 0;
            bits = on ? bits >> half : bits;
            base += on ? half : 0;
        }
        return base;
    }
    __device__ __forceinline__ int first() const {
#pragma unroll
        for (int j = 0; j < FEW_TOKENS / 64; ++j)
            if (word[j]) return j * 64 + __builtin_ctzll(word[j]);
        return 0;
    }
};

// The sum over all mates, eight of them asked for at a time, where there are more the next eight before these are added.  Each lane finds one of 64 mates'
// tokens first: found one after another by scalar instructions they took longer than their rows.
template <typename T, bool NARROW>
__device__ __forceinline__ void sum_of_mates(float* sum, const Mates& mates, const T* dY, int64_t ldy, unsigned c, int cols) {
    const int all = mates.count(), lane = threadIdx.x & 63;
    using Rows = RowsAhead<T, 8, NARROW>;
    for (int first = 0; first < all; first += 64) {
        const int there = min(64, all - first), tokens = mates.at(first + min(lane, there - 1));
        auto ask = [&](Rows& rows, int i) {
#pragma unroll
            for (int u = 0; u < 8; ++u) {  // the last one again where there are fewer
                const int token = __builtin_amdgcn_readlane(tokens, min(i + u, there - 1));
                rows.ask(u, dY + (int64_t)token * ldy, c, cols);
            }
        };
        auto add = [&](const Rows& rows, int i) {
            if (i + 8 <= there) {
#pragma unroll
                for (int u = 0; u < 8; ++u) rows.add(u, sum);
            } else {
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    if (i + u < there) rows.add(u, sum);
            }
        };
        Rows now, next;
        ask(now, 0);
        if (there > 8) {
            for (int i = 0; i < there; i += 16) {
                ask(next, i + 8);
                add(now, i);
                ask(now, i + 16);
                add(next, i + 8);
            }
        } else {
            add(now, 0);
        }
    }
}

// A block of places: the row and the token of place `first` + lane, and bits of the places with which a row, or the block, ends.
struct Places {
    int64_t first;
    int count, row, token;   // row, token: the lane's
    uint64_t row_ends;       // the row's last place of all
    bool began;              // the first place's row began before this block
    __device__ __forceinline__ Places(const TokenOrder& order, int64_t n, int rows, int64_t b, int each) {
        const int lane = threadIdx.x & 63;
        first = b * each;
        count = (int)min((int64_t)each, n - first);
        const int64_t p = first + min(lane, count - 1);
        row = order.row_at[p];
        token = order.token_at[p];
        const int before = first > 0 ? order.row_at[first - 1] : -1;
        const int behind = p + 1 < n ? order.row_at[p + 1] : rows;
        row_ends = __ballot(lane < count && row < rows && behind != row);
        began = before == __builtin_amdgcn_readlane(row, 0);
        // tokens of no row come last
        count = __popcll(__ballot(lane < count && row < rows));
    }
};

// An address in the card's memory, of one lane.  Said to be there: a load from any address counts as one of LDS too, and every wait for LDS, of the bins or
// the codebook, then waits for the rows asked for ahead (8192 tokens, k = 16: 24 us against 21.5).
template <typename P>
__device__ __forceinline__ const P* of_lane(uint64_t v, int lane) {
    const uint64_t at = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
    return (const P*)reinterpret_cast<const __attribute__((address_space(1))) P*>(at);
}

// Sums the places of a block, one row after another, and calls finish(item, p, complete, began, sum) with a row's last place there, the p-th; begin(item, p)
// where that row is asked for, to ask for what finish takes.  complete: the row has all of its places there; began: it has places before them.
// Most rows have one token or two, so a step is up to two places of one row, and the next step is asked for before this one is added.  Every step makes the
// same loads, its last place's again where it has fewer: how many are on their way has to be known for a wait that leaves the next step's alone.
// Addresses are formed for all places at once, a lane to each: formed for one place after another they took as many scalar instructions as the sums take
// vector ones.
template <typename T, bool NARROW, class Item, class Begin, class Finish>
__device__ __forceinline__ void sum_places_of(const Places& at, const T* dY, int64_t ldy, unsigned c, int cols, Begin begin, Finish finish) {
    struct Step {
        RowsAhead<T, 2, NARROW> rows;
        Item item;
        int count, last;  // last: the row's last place here if that is in the step, or -1
    };
    if (at.count == 0) return;
    const int lane = threadIdx.x & 63;
    const uint64_t from_lane = reinterpret_cast<uint64_t>(dY + (int64_t)at.token * ldy), left = lane < at.count ? at.row_ends >> lane : 0;
    const int last_of_lane = left ? lane + (int)__builtin_ctzll(left) : at.count - 1;
    const bool open = !(at.row_ends >> (at.count - 1) & 1);  // the last row goes on
    int p = 0;
    auto ask = [&](Step& s) {
        const int from = min(p, at.count - 1), last = __builtin_amdgcn_readlane(last_of_lane, from), to = min(from + 1, last);
        begin(s.item, from);
        s.rows.ask(0, of_lane<T>(from_lane, from), c, cols);
        s.rows.ask(1, of_lane<T>(from_lane, to), c, cols);
        s.count = p < at.count ? to - from + 1 : 0;
        s.last = to == last ? last : -1;
        p += s.count;
    };
    float sum[8];
    bool began = at.began, fresh = true;
    auto use = [&](const Step& s) {
        if (fresh) s.rows.begin(0, sum);
        else s.rows.add(0, sum);
        if (s.count > 1) s.rows.add(1, sum);
        fresh = s.last >= 0;
        if (fresh) {
            finish(s.item, s.last, !began && !(open && s.last == at.count - 1), began, sum);
            began = false;
        }
    };
    Step one, two;  // taken in turns: a copy would cost as much as the sum
    ask(one);
    for (;;) {
        ask(two);
        use(one);
        if (two.count == 0) break;
        ask(one);
        use(two);
        if (one.count == 0) break;
    }
}

// How many blocks before block b the row of its first place reaches into; all lanes take part.
__device__ __forceinline__ int64_t blocks_before(const TokenOrder& order, int64_t b, int each, int row) {
    const int lane = threadIdx.x & 63;
    int64_t before = 0;
    for (;;) {
        const int64_t q = b - before - lane;  // its first place's neighbour on the left
        const uint64_t there = __ballot(q > 0 && order.row_at[max(q, (int64_t)1) * each - 1] == row);
        const int run = ~there ? __builtin_ctzll(~there) : 64;
        before += run;
        if (run < 64) return before;
    }
}

// Clears the rows [.., width] of a table that no token has, a wavefront to a row; up to FEW_TOKENS tokens.
__device__ __forceinline__ void clear_other_rows(const TokenIds& ids, float* out, int64_t width, int64_t wave, int64_t waves) {
    const Mates::Rows rows(ids);
    const int lane = threadIdx.x & 63;
    for (int64_t r = wave; r < ids.rows; r += waves) {
        if (Mates(rows, (int)r).any()) continue;
        float* to = out + r * width;
        if (((reinterpret_cast<uintptr_t>(to) | (uintptr_t)(width * 4)) & 15) == 0) {
            for (int64_t c = lane * 4; c < width; c += 256) *reinterpret_cast<floatx4*>(to + c) = floatx4{0.f, 0.f, 0.f, 0.f};
        } else {
            for (int64_t c = lane; c < width; c += 64) to[c] = 0.f;
        }
    }
}

}  // namespace idkm

// Sums of rows of dY over the tokens of one row of a table: who has to be summed, and the rows asked for ahead.
//
// A wavefront takes 512 columns, eight to a lane.  Up to FEW_TOKENS tokens: a wavefront to a token, which compares all tokens' rows with its own (a
// vector load and a comparison for 64), leaves if an earlier token has the same row, and otherwise sums those that do; nothing is sorted.  More:
// a wavefront to `each` places of the sorted tokens; a row whose places lie in several blocks is summed in parts.
#pragma once
#include "token_sort.hpp"

namespace idkm {

constexpr int FEW_TOKENS = 256;

// A lane's eight columns of rows of dY.
template <typename T>
struct EightColumns {
    const T* dY;
    int64_t ldy;
    int c, cols;
    bool clean;  // every lane of the wavefront has all eight columns or none (those read the row's first ones)
    __device__ __forceinline__ EightColumns(const void* dY_, int64_t ldy_, int strip, int cols_) : ldy(ldy_), c(strip * 512 + (threadIdx.x & 63) * 8), cols(cols_) {
        clean = (cols & 7) == 0 || strip * 512 + 512 <= cols;
        dY = static_cast<const T*>(dY_) + (c < cols ? c : 0);
    }
};

// .. of four rows on their way.
template <typename T>
struct RowsAhead {
    static constexpr int U = 4, FR = 8 / Elem<T>::PER16;
    u32x4 raw[U][FR];
    __device__ __forceinline__ void ask(int u, const EightColumns<T>& at, int token) {
        const T* row = at.dY + (int64_t)token * at.ldy;
        if (at.clean) {
#pragma unroll
            for (int f = 0; f < FR; ++f) raw[u][f] = reinterpret_cast<const u32x4_any*>(row)[f];
        } else {
            struct alignas(16) Eight { T v[8]; } y;
#pragma unroll
            for (int e = 0; e < 8; ++e) y.v[e] = at.c + e < at.cols ? row[e] : (T)0.f;
            __builtin_memcpy(raw[u], &y, sizeof(y));
        }
    }
    __device__ __forceinline__ void add(int u, float* sum) const {
        struct alignas(16) Eight { T v[8]; } y;
        __builtin_memcpy(&y, raw[u], sizeof(y));
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += Elem<T>::up(y.v[e]);
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
    // the lowest token, taken out; only where any()
    __device__ __forceinline__ int next() {
#pragma unroll
        for (int j = 0; j < FEW_TOKENS / 64; ++j)
            if (word[j]) {
                const int at = __builtin_ctzll(word[j]);
                word[j] &= word[j] - 1;
                return j * 64 + at;
            }
        return 0;
    }
    __device__ __forceinline__ int first() const {
#pragma unroll
        for (int j = 0; j < FEW_TOKENS / 64; ++j)
            if (word[j]) return j * 64 + __builtin_ctzll(word[j]);
        return 0;
    }
};

// The sum over all mates, four of them asked for ahead.
template <typename T>
__device__ __forceinline__ void sum_of_mates(float* sum, Mates mates, const EightColumns<T>& at) {
    struct Step {
        RowsAhead<T> rows;
        int count;
    };
    auto ask = [&](Step& s) {
        s.count = 0;
#pragma unroll
        for (int u = 0; u < RowsAhead<T>::U; ++u)
            if (mates.any()) {
                s.rows.ask(u, at, mates.next());
                s.count = u + 1;
            }
    };
    Step now, next;
    ask(now);
    while (now.count > 0) {
        ask(next);
#pragma unroll
        for (int u = 0; u < RowsAhead<T>::U; ++u)
            if (u < now.count) now.rows.add(u, sum);
        now = next;
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

// Sums the places of a block, one row after another, and calls finish(item, row, place, complete, began, sum) with its last place there; begin(item, row) where
// that place is asked for, to ask for what finish takes.  complete: the row has all of its places there; began: it has places before them.
// Most rows have one token or two, so a step is up to four places of one row, and the next step is asked for before this one is added.
template <typename T, class Item, class Begin, class Finish>
__device__ __forceinline__ void sum_places_of(const Places& at, const EightColumns<T>& columns, Begin begin, Finish finish) {
    struct Step {
        RowsAhead<T> rows;
        Item item;
        int row, count, last;  // last: the row's last place here if that is in the step, or -1
    };
    int p = 0;
    auto ask = [&](Step& s) {
        s.count = 0;
        if (p >= at.count) return;
        s.row = __builtin_amdgcn_readlane(at.row, p);
        const uint64_t left = at.row_ends >> p;
        const int last = left ? min(p + (int)__builtin_ctzll(left), at.count - 1) : at.count - 1;
        s.count = min(RowsAhead<T>::U, last - p + 1);
        s.last = p + s.count > last ? last : -1;
        if (s.last >= 0) begin(s.item, s.row);
#pragma unroll
        for (int u = 0; u < RowsAhead<T>::U; ++u)
            if (u < s.count) s.rows.ask(u, columns, __builtin_amdgcn_readlane(at.token, p + u));
        p += s.count;
    };
    float sum[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = 0.f;
    bool began = at.began;
    Step now, next;
    ask(now);
    while (now.count > 0) {
        ask(next);
#pragma unroll
        for (int u = 0; u < RowsAhead<T>::U; ++u)
            if (u < now.count) now.rows.add(u, sum);
        if (now.last >= 0) {
            finish(now.item, now.row, at.first + now.last, (at.row_ends >> now.last & 1) && !began, began, sum);
            began = false;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = 0.f;
        }
        now = next;
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

// Lookups of tokens' rows in tables, float32 or stored as codes, and the sums of their gradients.
#include <algorithm>

#include "embedding.h"
#include "layers.h"

namespace idkm {

// ---- the order of the tokens

__global__ __launch_bounds__(RANK_WAVES * 64) void k_rank_tokens(const TokenIds in, const TokenOrder out) {
    extern __shared__ __align__(16) int rank_lds[];
    rank_tokens(in, out, blockIdx.x, rank_lds);
}

__global__ __launch_bounds__(256) void k_radix_count(const RadixPass a) {
    __shared__ int hist[256];
    hist[threadIdx.x] = 0;
    __syncthreads();
    const int64_t p0 = (int64_t)blockIdx.x * RADIX_BLOCK;
    for (int i = threadIdx.x; i < RADIX_BLOCK; i += 256)
        if (p0 + i < a.ids.n) atomicAdd(&hist[a.row(p0 + i) >> a.shift & 255], 1);  // whole numbers: their order does not show
    __syncthreads();
    a.counts[threadIdx.x * a.blocks + blockIdx.x] = hist[threadIdx.x];
}

// counts[i] = the sum of counts[j], j < i; one workgroup.
__global__ __launch_bounds__(1024) void k_running_sum(int32_t* counts, int n) {
    __shared__ int waves[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int before = 0;
    for (int at = 0; at < n; at += 4096) {
        const int i = at + threadIdx.x * 4;
        int v[4], sum = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = i + e < n ? counts[i + e] : 0;
            sum += v[e];
        }
        int upto = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int left = __shfl_up(upto, o);
            if (lane >= o) upto += left;
        }
        if (lane == 63) waves[wave] = upto;
        __syncthreads();
        int run = before + upto - sum;
        for (int w = 0; w < 16; ++w) {
            if (w < wave) run += waves[w];
            before += waves[w];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i + e < n) {
                counts[i + e] = run;
                run += v[e];
            }
        __syncthreads();
    }
}

// A wavefront takes RADIX_WAVE places in order, 64 at a time: lanes with the same eight bits go to consecutive places.
__global__ __launch_bounds__(256) void k_radix_place(const RadixPass a) {
    __shared__ int next[4][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int w = 0; w < 4; ++w) next[w][threadIdx.x] = 0;
    __syncthreads();
    const int64_t p0 = (int64_t)blockIdx.x * RADIX_BLOCK + wave * RADIX_WAVE;
    for (int i = lane; i < RADIX_WAVE; i += 64)
        if (p0 + i < a.ids.n) atomicAdd(&next[wave][a.row(p0 + i) >> a.shift & 255], 1);
    __syncthreads();
    int begin = a.counts[threadIdx.x * a.blocks + blockIdx.x];
    for (int w = 0; w < 4; ++w) {
        const int own = next[w][threadIdx.x];
        next[w][threadIdx.x] = begin;
        begin += own;
    }
    __syncthreads();
    for (int i = 0; i < RADIX_WAVE; i += 64) {
        const int64_t p = p0 + i + lane;
        const bool there = p < a.ids.n;
        const int row = there ? a.row(p) : 0, token = there ? (a.first ? (int)p : a.from.token_at[p]) : 0;
        const int digit = row >> a.shift & 255;
        uint64_t same = __ballot(there);
#pragma unroll
        for (int b = 0; b < 8; ++b) {
            const uint64_t set = __ballot(digit >> b & 1);
            same &= digit >> b & 1 ? set : ~set;
        }
        if (there) {
            const int before = __popcll(same & (((uint64_t)1 << lane) - 1));
            const int place = next[wave][digit] + before;
            a.to.row_at[place] = row;
            a.to.token_at[place] = token;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // every lane has read where its bits' places begin
        if (there && same >> lane == 1) next[wave][digit] += __popcll(same);  // the last lane of its kind
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

int64_t sort_words(int64_t n) {
    if (n <= RANK_TOKENS) return 2 * n;
    return 4 * n + 256 * ((n + RADIX_BLOCK - 1) / RADIX_BLOCK);
}

TokenOrder launch_sort(const TokenIds& ids, int32_t* ws, hipStream_t s) {
    const int64_t n = ids.n;
    TokenOrder order{ws, ws + n};
    if (n <= RANK_TOKENS) {
        const size_t lds = 4 * (RANK_WAVES * 64 + (size_t)up_to(n, 4));
        allow_lds(reinterpret_cast<const void*>(&k_rank_tokens), lds);
        hipLaunchKernelGGL(k_rank_tokens, dim3((unsigned)((n + 63) / 64)), dim3(RANK_WAVES * 64), lds, s, ids, order);
        return order;
    }
    TokenOrder other{ws + 2 * n, ws + 3 * n};
    RadixPass a{};
    a.ids = ids;
    a.first = 1;
    a.counts = ws + 4 * n;
    a.blocks = (int)((n + RADIX_BLOCK - 1) / RADIX_BLOCK);
    for (a.shift = 0; a.shift == 0 || ids.rows >> a.shift > 0; a.shift += 8) {
        a.from = other;
        a.to = order;
        hipLaunchKernelGGL(k_radix_count, dim3((unsigned)a.blocks), dim3(256), 0, s, a);
        hipLaunchKernelGGL(k_running_sum, dim3(1), dim3(1024), 0, s, a.counts, 256 * a.blocks);
        hipLaunchKernelGGL(k_radix_place, dim3((unsigned)a.blocks), dim3(256), 0, s, a);
        std::swap(order, other);
        a.first = 0;
    }
    return other;
}

// One workgroup.
__global__ __launch_bounds__(1024) void k_rows_of_tokens(const TokenOrder order, int64_t n, int rows, const RowsOfTokens out) {
    __shared__ int waves[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int before = 0;
    for (int64_t at = 0; at < n; at += 1024) {
        const int64_t p = at + threadIdx.x;
        const int row = p < n ? order.row_at[p] : rows;
        const bool begins = row < rows && (p == 0 || order.row_at[p - 1] != row);
        const uint64_t all = __ballot(begins);
        if (lane == 0) waves[wave] = __popcll(all);
        __syncthreads();
        int index = before + __popcll(all & (((uint64_t)2 << lane) - 1)) - 1;
        for (int w = 0; w < 16; ++w) {
            if (w < wave) index += waves[w];
            before += waves[w];
        }
        if (p < n) out.index_at[p] = index;
        if (begins) out.row_of[index] = row;
        __syncthreads();
    }
    if (threadIdx.x == 0) *out.count = before;
}

void launch_rows(const TokenOrder& order, int64_t n, int rows, const RowsOfTokens& out, hipStream_t s) {
    hipLaunchKernelGGL(k_rows_of_tokens, dim3(1), dim3(1024), 0, s, order, n, rows, out);
}

// ---- sums by row

// A wavefront takes `each` places of 64 x 8 columns: rows of dY in the order of their tokens, asked for eight ahead.  The sum of a
// row that has all of its places there goes to `out`; the first and last rows' may go on before and behind: their parts go to `partial` (2 b: a row that
// began before block b, 2 b + 1: one that begins in it and goes on), which the second kernel adds up in order.
template <typename T>
__global__ __launch_bounds__(256) void k_sums(const SumArgs a) {
    constexpr int U = 8, FR = 8 / Elem<T>::PER16;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int strips = (int)((a.cols + 511) / 512);
    const int64_t task = (int64_t)blockIdx.x * 4 + wave, b = task / strips;
    const int strip = (int)(task - b * strips), c = strip * 512 + lane * 8;
    const int64_t first = b * a.each, last = min(a.n, first + a.each);
    if (first >= a.n || c >= a.cols) return;  // lanes behind the last column take no part: no exchanges between lanes follow
    const bool whole = c + 8 <= a.cols;
    const T* dY = static_cast<const T*>(a.dY) + c;
    float sum[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = 0.f;
    auto store = [&](float* to) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] *= a.alpha;
        if (whole && ((reinterpret_cast<uintptr_t>(to + c)) & 15) == 0) {
            reinterpret_cast<floatx4*>(to + c)[0] = floatx4{sum[0], sum[1], sum[2], sum[3]};
            reinterpret_cast<floatx4*>(to + c)[1] = floatx4{sum[4], sum[5], sum[6], sum[7]};
        } else {
            for (int e = 0; e < 8 && c + e < a.cols; ++e) to[c + e] = sum[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = 0.f;
    };
    bool began = first > 0 && a.order.row_at[first - 1] == a.order.row_at[first];  // before this block
    for (int64_t p0 = first; p0 < last; p0 += U) {
        u32x4 raw[U][FR];
        int row[U + 1];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t p = min(p0 + u, last - 1);
            row[u] = a.order.row_at[p];
            const T* from = dY + (int64_t)a.order.token_at[p] * a.ldy;
            if (whole) {
#pragma unroll
                for (int f = 0; f < FR; ++f) raw[u][f] = reinterpret_cast<const u32x4_any*>(from)[f];
            } else {
                struct alignas(16) Eight { T v[8]; } y;
#pragma unroll
                for (int e = 0; e < 8; ++e) y.v[e] = c + e < a.cols ? from[e] : (T)0.f;
                __builtin_memcpy(raw[u], &y, sizeof(y));
            }
        }
        row[U] = p0 + U < a.n ? a.order.row_at[p0 + U] : a.rows;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t p = p0 + u;
            if (p >= last || row[u] >= a.rows) break;
            struct alignas(16) Eight { T v[8]; } y;
            __builtin_memcpy(&y, raw[u], sizeof(y));
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += Elem<T>::up(y.v[e]);
            const int behind = p + 1 >= a.n ? a.rows : p + 1 < last || u == U - 1 ? row[u + 1] : a.order.row_at[p + 1];
            const bool ends = behind != row[u];
            if (ends && !began) {
                store(a.out + (a.index_at ? (int64_t)a.index_at[p] : (int64_t)row[u]) * a.ldo);
            } else if (ends || p + 1 == last) {
                store(a.partial + (2 * b + (began ? 0 : 1)) * a.ldp);
                began = false;
            }
        }
    }
}

// Rows whose places lie in several blocks: the block in which such a row begins adds up its parts.
__global__ __launch_bounds__(256) void k_join_sums(const SumArgs a) {
    const int64_t b = blockIdx.x, behind = (b + 1) * a.each;  // a block follows
    const int row = a.order.row_at[behind - 1];
    if (row >= a.rows || a.order.row_at[behind] != row) return;
    if (b > 0 && a.order.row_at[b * a.each] == row && a.order.row_at[b * a.each - 1] == row) return;  // it began before
    int64_t inside = behind, outside = a.n;  // its last place, halving
    while (outside - inside > 1) {
        const int64_t p = (inside + outside) >> 1;
        if (a.order.row_at[p] == row) inside = p;
        else outside = p;
    }
    const int64_t end = inside / a.each;
    const int64_t c = (int64_t)blockIdx.y * 256 + threadIdx.x;
    if (c >= a.cols) return;
    float sum = a.partial[(2 * b + 1) * a.ldp + c];
    const float* part = a.partial + c;
    int64_t i = b + 1;
    for (; i + 8 <= end + 1; i += 8) {
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = part[2 * (i + u) * a.ldp];
#pragma unroll
        for (int u = 0; u < 8; ++u) sum += v[u];
    }
    for (; i <= end; ++i) sum += part[2 * i * a.ldp];
    a.out[(a.index_at ? (int64_t)a.index_at[behind - 1] : (int64_t)row) * a.ldo + c] = sum;
}

// Places to a wavefront: some 4096 wavefronts, at most 64 places each.
int sum_places(int64_t n, int64_t cols) {
    const int64_t strips = (cols + 511) / 512, each = n * strips / 4096;
    return each < 8 ? 8 : each > 64 ? 64 : (int)each;
}

int64_t sum_partials(int64_t n, int64_t cols) {
    const int each = sum_places(n, cols);
    const int64_t blocks = (n + each - 1) / each;
    return blocks > 1 ? 2 * blocks * up_to(cols, 4) : 0;
}

void launch_sums(int dtype, const SumArgs& args, hipStream_t s) {
    SumArgs a = args;
    a.each = sum_places(a.n, a.cols);
    a.ldp = up_to(a.cols, 4);
    const int64_t blocks = (a.n + a.each - 1) / a.each, tasks = blocks * ((a.cols + 511) / 512);
    BY_TYPE(dtype, T, hipLaunchKernelGGL(k_sums<T>, dim3((unsigned)((tasks + 3) / 4)), dim3(256), 0, s, a));
    if (blocks > 1) hipLaunchKernelGGL(k_join_sums, dim3((unsigned)(blocks - 1), (unsigned)((a.cols + 255) / 256)), dim3(256), 0, s, a);
}

// ---- lookups

template <typename T>
struct EightOut {
    struct alignas(16) Eight { T v[8]; } y;
    __device__ __forceinline__ void store(T* to, int64_t have) const {
        if (have >= 8) {
            u32x4 raw[8 / Elem<T>::PER16];
            __builtin_memcpy(raw, &y, sizeof(y));
#pragma unroll
            for (int f = 0; f < 8 / Elem<T>::PER16; ++f) reinterpret_cast<u32x4_any*>(to)[f] = raw[f];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < have) to[e] = y.v[e];
        }
    }
};

// A thread takes 8 columns of a token's row.
template <typename T>
__global__ __launch_bounds__(256) void k_lookup_table(const LookupArgs a) {
    const int64_t per_row = (a.cols + 7) / 8, total = a.ids.n * per_row;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < total; at += (int64_t)gridDim.x * 256) {
        const int64_t t = at / per_row, c = (at - t * per_row) * 8, id = a.ids.raw(t);
        EightOut<T> out;
        const bool there = id >= 0 && id < a.ids.rows;
        const float* w = a.W + (there ? id : 0) * a.cols + c;
        float v[8];
        if (c + 8 <= a.cols) {
            u32x4 raw[2];
#pragma unroll
            for (int f = 0; f < 2; ++f) raw[f] = reinterpret_cast<const u32x4_word*>(w)[f];
            __builtin_memcpy(v, raw, sizeof(v));
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = c + e < a.cols ? w[e] : 0.f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) out.y.v[e] = there ? Elem<T>::down(a.alpha * v[e]) : id < 0 ? (T)0.f : Elem<T>::nan();
        out.store(static_cast<T*>(a.Y) + t * a.ldy + c, a.cols - c);
    }
}

// The same of a stored table, one code at a time.
template <typename T>
__global__ __launch_bounds__(256) void k_lookup_codes(const LookupArgs a) {
    extern __shared__ __align__(16) unsigned char lds[];
    const T* C = static_cast<const T*>(a.C);
    if (a.c_in_lds) {
        T* copy = reinterpret_cast<T*>(lds);
        for (int i = threadIdx.x; i < a.k * a.d; i += 256) copy[i] = C[i];
        __syncthreads();
        C = copy;
    }
    const int64_t per_row = (a.cols + 7) / 8, total = a.ids.n * per_row, codes = a.cols / a.d;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < total; at += (int64_t)gridDim.x * 256) {
        const int64_t t = at / per_row, c = (at - t * per_row) * 8, id = a.ids.raw(t);
        EightOut<T> out;
        if (id < 0 || id >= a.ids.rows) {
#pragma unroll
            for (int e = 0; e < 8; ++e) out.y.v[e] = id < 0 ? (T)0.f : Elem<T>::nan();
        } else {
            int64_t j = c / a.d;
            int x = (int)(c - j * a.d);
            uint32_t code = code_at(a.words, a.nwords, id * codes + j, a.bits);
            const float by = a.S ? a.alpha * a.S[id * a.groups + c / a.group] : a.alpha;  // groups are multiples of 32: eight columns lie in one
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (c + e >= a.cols) {
                    out.y.v[e] = (T)0.f;
                    continue;
                }
                out.y.v[e] = code >= (uint32_t)a.k ? Elem<T>::nan() : Elem<T>::down(Elem<T>::up(C[(int64_t)code * a.d + x]) * by);
                if (++x == a.d) {
                    x = 0;
                    ++j;
                    if (e < 7 && c + e + 1 < a.cols) code = code_at(a.words, a.nwords, id * codes + j, a.bits);
                }
            }
        }
        out.store(static_cast<T*>(a.Y) + t * a.ldy + c, a.cols - c);
    }
}

static unsigned grid_of(int64_t threads, int64_t most) {
    const int64_t g = (threads + 255) / 256;
    return (unsigned)(g < 1 ? 1 : g > most ? most : g);
}

void launch_lookup_table(int dtype, const LookupArgs& a, hipStream_t s) {
    BY_TYPE(dtype, T, hipLaunchKernelGGL(k_lookup_table<T>, dim3(grid_of(a.ids.n * ((a.cols + 7) / 8), 8192)), dim3(256), 0, s, a));
}

void launch_lookup_codes(int dtype, const LookupArgs& args, hipStream_t s) {
    LookupArgs a = args;
    const size_t book = (size_t)a.k * a.d * (dtype == 0 ? 4 : 2);
    a.c_in_lds = book <= 32 * 1024;
    BY_TYPE(dtype, T, hipLaunchKernelGGL(k_lookup_codes<T>, dim3(grid_of(a.ids.n * ((a.cols + 7) / 8), 2048)), dim3(256), a.c_in_lds ? book : 0, s, a));
}

}  // namespace idkm

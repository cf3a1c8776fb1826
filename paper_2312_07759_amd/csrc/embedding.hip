// Lookups of tokens' rows in tables, float32 or stored as codes, and the sums of their gradients.
#include <algorithm>

#include "embedding.h"
#include "layers.h"

namespace idkm {

// ---- the order of the tokens

// The workgroups behind the first GROUPS clear `count` floats, beside them.
constexpr unsigned GROUPS = 257;
__global__ __launch_bounds__(GROUP_WAVES * 64) void k_group_tokens(const TokenIds in, const TokenOrder out, float* clear, int64_t count) {
    extern __shared__ __align__(16) int group_lds_words[];
    if (blockIdx.x < GROUPS) {
        group_tokens(in, out, group_lds_words);
        return;
    }
    const int64_t t = (int64_t)(blockIdx.x - GROUPS) * blockDim.x + threadIdx.x, step = (int64_t)(gridDim.x - GROUPS) * blockDim.x;
    if ((reinterpret_cast<uintptr_t>(clear) & 15) == 0) {
        for (int64_t i = t; i < count / 4; i += step) reinterpret_cast<floatx4*>(clear)[i] = floatx4{0.f, 0.f, 0.f, 0.f};
        if (t < (count & 3)) clear[count - 1 - t] = 0.f;
    } else {
        for (int64_t i = t; i < count; i += step) clear[i] = 0.f;
    }
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
    if (n <= GROUP_TOKENS) return 2 * n;
    return 4 * n + 256 * ((n + RADIX_BLOCK - 1) / RADIX_BLOCK);
}

TokenOrder launch_sort(const TokenIds& ids, int32_t* ws, float* clear, int64_t count, hipStream_t s) {
    const int64_t n = ids.n;
    TokenOrder order{ws, ws + n};
    if (n <= GROUP_TOKENS) {
        allow_lds(reinterpret_cast<const void*>(&k_group_tokens), group_lds(n));
        const unsigned clearing = (unsigned)std::min<int64_t>(512, (count + 4095) / 4096);
        hipLaunchKernelGGL(k_group_tokens, dim3(GROUPS + clearing), dim3(GROUP_WAVES * 64), group_lds(n), s, ids, order, clear, count);
        return order;
    }
    if (count > 0) launch_fill_zero(clear, count, s);
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

// Eight columns of a row's sum.
__device__ __forceinline__ void store_sum(float* to, const Columns& at, int cols, float alpha, const float* sum) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = alpha * sum[e];
    if (at.skip == 0 && cols >= 8 && (reinterpret_cast<uintptr_t>(to + at.c) & 15) == 0) {
        reinterpret_cast<floatx4*>(to + at.c)[0] = floatx4{v[0], v[1], v[2], v[3]};
        reinterpret_cast<floatx4*>(to + at.c)[1] = floatx4{v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e >= at.skip && at.c + e < cols) to[at.c + e] = v[e];
    }
}

// The sum of a row that has all of its places in a block goes to `out`; parts of others go to `partial` (2 b: of a row that began before block b,
// 2 b + 1: of one that begins in it and goes on), which the next kernel adds up in order.  4096 tokens of 1024 columns, bfloat16: 6 us, and 5 to join the parts; latency of
// the order, the rows and, in the other launch, the parts.
template <typename T, bool NARROW>
__global__ __launch_bounds__(256) void k_sums(const SumArgs a) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int cols = (int)a.cols, strips = (cols + 511) / 512;
    const int64_t task = (int64_t)blockIdx.x * 4 + wave, b = task / strips;
    const Columns columns((int)(task - b * strips), cols);
    if (b * a.each >= a.n) return;
    const Places places(a.order, a.n, a.rows, b, a.each);
    struct None {};
    auto begin = [&](None&, int) {};
    auto end = [&](const None&, int p, bool complete, bool began, const float* sum) {
        const int row = a.index_at ? a.index_at[places.first + p] : __builtin_amdgcn_readlane(places.row, p);
        float* to = complete ? a.out + row * a.ldo : a.partial + (2 * b + (began ? 0 : 1)) * a.ldp;
        if (columns.skip < 8) store_sum(to, columns, cols, a.alpha, sum);
    };
    sum_places_of<T, NARROW, None>(places, static_cast<const T*>(a.dY), a.ldy, columns.c, cols, begin, end);
}

// Up to FEW_TOKENS tokens: the first workgroups sum, the ones behind them clear the rows of which there is no token.  33 tokens, 1000 rows of 512: 3.8 us.
template <typename T, bool NARROW>
__global__ __launch_bounds__(256) void k_sums_of_few(const TokenIds ids, float alpha, const T* dY, int64_t ldy, int cols, float* dW, unsigned summing) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (blockIdx.x >= summing) {
        clear_other_rows(ids, dW, cols, (int64_t)(blockIdx.x - summing) * 4 + wave, (int64_t)(gridDim.x - summing) * 4);
        return;
    }
    const int strips = (cols + 511) / 512, task = blockIdx.x * 4 + wave, t = task / strips;
    if (t >= (int)ids.n) return;
    const Columns columns(task - t * strips, cols);
    const Mates::Rows rows(ids);
    const int row = ids.row(t);
    const Mates mates(rows, row);
    if (row >= ids.rows || mates.first() != t) return;
    float sum[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = 0.f;
    sum_of_mates<T, NARROW>(sum, mates, dY, ldy, columns.c, cols);
    if (columns.skip < 8) store_sum(dW + (int64_t)row * cols, columns, cols, alpha, sum);
}

void launch_sums_of_few(int dtype, const TokenIds& ids, float alpha, const void* dY, int64_t ldy, int64_t cols, float* dW, hipStream_t s) {
    const unsigned summing = (unsigned)((ids.n * ((cols + 511) / 512) + 3) / 4), clearing = (unsigned)std::min<int64_t>(2048, (ids.rows + 3) / 4);
    BY_TYPE(dtype, T, hipLaunchKernelGGL((cols < 8 ? &k_sums_of_few<T, true> : &k_sums_of_few<T, false>), dim3(summing + clearing), dim3(256), 0, s, ids, alpha, static_cast<const T*>(dY), ldy,
                                         (int)cols, dW, summing));
}

// Rows whose places lie in several blocks: the block in which such a row ends adds up its parts, in order.
__global__ __launch_bounds__(256) void k_join_sums(const SumArgs a) {
    const int64_t b = blockIdx.x + 1, first = b * a.each, behind = min(first + a.each, a.n);
    const int row = a.order.row_at[first];
    if (row >= a.rows || a.order.row_at[first - 1] != row) return;
    if (behind < a.n && a.order.row_at[behind - 1] == row && a.order.row_at[behind] == row) return;  // it goes on
    const int64_t start = b - blocks_before(a.order, b, a.each, row);
    const int64_t c = (int64_t)blockIdx.y * 256 + threadIdx.x;
    if (c >= a.cols) return;
    float sum = a.partial[(2 * start + 1) * a.ldp + c];
    const float* part = a.partial + c;
    for (int64_t i = start + 1; i <= b; i += 16) {  // the last part again where there are fewer
        float v[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) v[u] = part[2 * min(i + u, b) * a.ldp];
#pragma unroll
        for (int u = 0; u < 16; ++u) sum += i + u <= b ? v[u] : 0.f;
    }
    a.out[(a.index_at ? (int64_t)a.index_at[first] : (int64_t)row) * a.ldo + c] = sum;
}

// Places to a wavefront: some 4096 wavefronts, at most 64 places each.
int sum_places(int64_t n, int64_t cols) {
    const int64_t strips = (cols + 511) / 512, each = n * strips / 4096;
    return each < 4 ? 4 : each > 64 ? 64 : (int)each;
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
    BY_TYPE(dtype, T, hipLaunchKernelGGL((a.cols < 8 ? &k_sums<T, true> : &k_sums<T, false>), dim3((unsigned)((tasks + 3) / 4)), dim3(256), 0, s, a));
    if (blocks > 1) hipLaunchKernelGGL(k_join_sums, dim3((unsigned)(blocks - 1), (unsigned)((a.cols + 255) / 256)), dim3(256), 0, s, a);
}

// ---- gradients of stored tables

// dC[e] = the sum of bins[e][..] in float64, a workgroup to an e; the workgroups behind them: dS of the rows whose sums went to `parts`, in the order
// of their parts and segments.
__global__ __launch_bounds__(256) void k_join_lookup(const LookupGradArgs a, int bins, int kd, float* dC, int of_group) {
    if ((int)blockIdx.x < kd) {
        __shared__ double waves[4];
        const float* mine = a.bins + blockIdx.x * a.pitch;
        double sum = 0.0;
        for (int w = threadIdx.x; w < bins; w += 256) sum += (double)mine[w];
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
        if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = sum;
        __syncthreads();
        if (threadIdx.x == 0) dC[blockIdx.x] = (float)(waves[0] + waves[1] + waves[2] + waves[3]);
        return;
    }
    const int64_t n = a.ids.n;
    // Lanes to a group's segments, a power of two; a wavefront takes as many groups at a time as it has room for, and where that is more than there are, every
    // sixteen parts of a row go to other lanes (5180 tokens of 284 rows of 338 columns, in eleven groups: 20 us with one lane to a group, 500 parts one after another,
    // and 9.5 now).
    const int lane = threadIdx.x & 63;
    int share = 1, at_once = 1;
    while (share < 64 && share < of_group) share <<= 1;
    while (at_once < 64 / share && at_once < a.groups) at_once <<= 1;
    const int part = lane & (share - 1), own = lane / share & (at_once - 1), slice = lane / (share * at_once), slices = 64 / (share * at_once);
    // the sums of a row whose parts end with blocks `start` .. `last` (the last one's at place p) to dS
    auto join = [&](int row, int64_t start, int64_t last, int64_t p) {
        for (int g = own; g - own < a.groups; g += at_once) {  // all lanes take part in the exchanges
            float sum = 0.f;
            const int from = g * of_group, to = g < a.groups ? min(a.per_part, from + of_group) : from;
            auto batch = [&](int64_t q, auto many) {  // the last part again where there are fewer
                constexpr int U = decltype(many)::value;
                for (int j = from + part; j < to; j += share) {
                    float v[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) v[u] = a.parts[(a.few ? p : min((min(q + u, last) + 1) * a.each - 1, p)) * a.per_part + j];
#pragma unroll
                    for (int u = 0; u < U; ++u) sum += q + u <= last ? v[u] : 0.f;
                }
            };
            for (int64_t q = start + slice * 16; q <= last; q += slices * 16) {
                if (q + 8 <= last) batch(q, std::integral_constant<int, 16>());
                else batch(q, std::integral_constant<int, 8>());
            }
            for (int o = 1; o < share; o <<= 1) sum += __shfl_xor(sum, o);
            for (int o = share * at_once; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
            if (part == 0 && slice == 0 && g < a.groups) a.dS[(int64_t)row * a.groups + g] = sum;
        }
    };
    const int64_t wave = (int64_t)(blockIdx.x - kd) * 4 + (threadIdx.x >> 6), waves = (int64_t)(gridDim.x - kd) * 4;
    if (a.few) {  // a wavefront to a token, whose row is in one part if it is the row's first
        for (int64_t t = wave; t < n; t += waves) {
            const int row = a.order.row_at[t];
            if (row < a.ids.rows) join(row, 0, 0, t);
        }
        return;
    }
    // .. to the rows that end in a block
    const int64_t blocks = (n + a.each - 1) / a.each;
    for (int64_t b = wave; b < blocks; b += waves) {
        const Places at(a.order, n, a.ids.rows, b, a.each);
        uint64_t ends = at.row_ends;
        if (!a.segmented) ends = at.began ? ends & (0 - ends) : 0;  // the others are in dS
        for (bool began = at.began; ends; ends &= ends - 1, began = false) {
            const int p = __builtin_ctzll(ends), row = __builtin_amdgcn_readlane(at.row, p);
            join(row, began ? b - blocks_before(a.order, b, a.each, row) : b, b, at.first + p);
        }
    }
}

void launch_join_lookup(const LookupGradPlan& p, const LookupGradArgs& a, int kd, float* dC, int of_group, hipStream_t s) {
    if (!dC) kd = 0;
    const bool parts = a.dS && (a.segmented || (!p.few && a.ids.n > p.each));
    const int64_t joining = ((p.few ? a.ids.n : (a.ids.n + p.each - 1) / p.each) + 3) / 4;
    const unsigned grid = (unsigned)kd + (parts ? (unsigned)std::min<int64_t>(4096, joining) : 0u);
    if (grid > 0) hipLaunchKernelGGL(k_join_lookup, dim3(grid), dim3(256), 0, s, a, p.grid, kd, dC, of_group);
}

// As many workgroups as the compute units hold at once, and blocks of so few places that every wavefront has one: 8192 tokens of 4096 columns, bfloat16,
// k = 16 21.5 us with 24 wavefronts to a compute unit (as the registers allow) and 8 places; when it took 23.5, 30.5 with 16 places and 24.4 with 4.
// A wavefront's bins take 8 KB of LDS at most, 16 for codebooks of more than 256 components: lanes that share bins take turns, and more room for each means
// fewer wavefronts.  The same tokens with 8, 16 and 32 KB: 100 components (d = 1) 52 us, 65 and 80; 128 (d = 8) 34, 35 and 49; in all 400 (d = 4) 82, 72 and 92;
// 512 (d = 2) 95, 79 and 101.
LookupGradPlan lookup_grad_plan(int64_t n, int64_t cols, int esize, int kd) {
    LookupGradPlan p{};
    const int64_t strips = (cols + 511) / 512;
    p.few = n <= FEW_TOKENS;
    p.each = (int)std::max<int64_t>(2, std::min<int64_t>(LOOKUP_PLACES, n * strips / 8192));
    const int64_t tasks = (p.few ? n : (n + p.each - 1) / p.each) * strips;
    p.width_log = 6;
    while (p.width_log > 2 && kd * 4 << p.width_log > (kd > 256 ? 16384 : 8192)) --p.width_log;
    const int wave_bytes = (kd * 4 << p.width_log) + LOOKUP_KEPT * 4;
    p.waves = std::min(4, 144 * 1024 / wave_bytes);
    const int64_t resident = std::max(1, std::min((esize == 4 ? 16 : 24) / p.waves, 156 * 1024 / (wave_bytes * p.waves + kd * 4)));
    p.grid = (int)std::min<int64_t>((tasks + p.waves - 1) / p.waves, 256 * resident);
    return p;
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

// A thread takes 8 columns of a token's row.  Bound by memory: 4096 tokens of 1024 columns to bfloat16, 17 MB read and 8 written, 5.3 us, 4.7 TB/s.
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

// The same for codes of up to 8 bits, D in {1, 2, 4, 8} and rows of at least eight columns: a wavefront takes 512 columns of some tokens' rows, whose codes
// are asked for one token ahead.  The codebook lies in LDS, once: lanes that meet in a bank wait for each other, which the stores cover.
// 8192 tokens of 4096 columns, k = 256, d = 4, float16: 18.5 us (a fill of Y takes 10; 43 with one code read at a time, 64-bit divisions for every eight columns).
template <typename T, int D>
__global__ __launch_bounds__(256) void k_lookup_codes_fast(const LookupArgs a) {
    constexpr int NC = 8 / D;
    extern __shared__ __align__(16) unsigned char lds[];
    struct alignas(D * sizeof(T) > 16 ? 16 : D * sizeof(T)) Entry { T v[D]; };
    T* book = reinterpret_cast<T*>(lds);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int cols = (int)a.cols, strips = (cols + 511) / 512, blocks = (int)((a.ids.n + a.each - 1) / a.each);
    const uint32_t mask = (1u << a.bits) - 1u;
    const int entries = (int)mask + 1;  // codes that are none give NaN
    const float* S = a.S ? a.S : reinterpret_cast<const float*>(a.words);  // without scales some word, which is not used
    const int groups = a.S ? a.groups : 0;
    struct Item {
        uint32_t w[3];
        int sh;
        float s;
    };
    bool built = false;
    for (int task = blockIdx.x * 4 + wave;; task += gridDim.x * 4) {
        const bool there = task < blocks * strips;
        const int b = there ? task / strips : 0, strip = there ? task - b * strips : 0;
        const Columns columns(strip, cols);
        const int c = columns.c, at_bit = c / D * a.bits, g = a.S ? min(c + columns.skip, cols - 1) / a.group : 0;
        const int64_t first = (int64_t)b * a.each;
        const int count = there ? (int)min((int64_t)a.each, a.ids.n - first) : 0;
        const int64_t id = a.ids.raw(first + min(lane, max(count, 1) - 1));
        const int row = id < 0 || id >= a.ids.rows ? 0 : (int)id, kind = id < 0 ? 1 : id >= a.ids.rows ? 2 : 0;
        const int64_t row_bit = row * a.row_bits;
        const uint64_t word = reinterpret_cast<uint64_t>(a.words + (row_bit >> 5)), scale = reinterpret_cast<uint64_t>(S + (int64_t)row * groups);
        // the row's bit, whether its last word but two ends behind the stream, and what its token is
        const int start = (int)(row_bit & 31) | ((row_bit + a.row_bits + 31) / 32 + 3 > a.nwords ? 32 : 0) | kind << 6;
        auto ask = [&](Item& t, int p) {
            const int of = __builtin_amdgcn_readlane(start, p);
            const uint32_t* words = of_lane<uint32_t>(word, p);
            const int bit = (of & 31) + at_bit;
            int from = bit >> 5;
            if (of & 32) from = min(from, (int)(a.words + (a.nwords - 3) - words));
            t.sh = bit - from * 32;
            const u32x3_word w = *reinterpret_cast<const u32x3_word*>(words + from);
#pragma unroll
            for (int i = 0; i < 3; ++i) t.w[i] = w[i];
            t.s = of_lane<float>(scale, p)[g];
        };
        Item now, next;
        ask(now, 0);
        if (!built) {  // the same for the whole workgroup
            for (int i = threadIdx.x; i < entries * D; i += 256) book[i] = i < a.k * D ? static_cast<const T*>(a.C)[i] : Elem<T>::nan();
            __syncthreads();
            built = true;
        }
        if (!there) break;
        for (int p = 0; p < count; ++p) {
            ask(next, min(p + 1, count - 1));
            uint32_t b0 = now.w[0], b1 = now.w[1], b2 = now.w[2];
            if (__any(now.sh >= 32)) {  // only near the stream's end
                const bool two = now.sh >= 64, one = now.sh >= 32;
                b0 = two ? b2 : one ? b1 : b0;
                b1 = two ? 0u : one ? b2 : b1;
                b2 = one ? 0u : b2;
            }
            uint32_t low = __builtin_amdgcn_alignbit(b1, b0, now.sh & 31), high = __builtin_amdgcn_alignbit(b2, b1, now.sh & 31);
            const float by = a.S ? a.alpha * now.s : a.alpha;
            EightOut<T> out;
#pragma unroll
            for (int e = 0; e < NC; ++e) {
                const Entry entry = *reinterpret_cast<const Entry*>(book + (low & mask) * D);
                low = __builtin_amdgcn_alignbit(high, low, a.bits);
                high >>= a.bits;
#pragma unroll
                for (int i = 0; i < D; ++i) out.y.v[e * D + i] = Elem<T>::down(Elem<T>::up(entry.v[i]) * by);
            }
            const int of = __builtin_amdgcn_readlane(start, p) >> 6;
            if (of != 0) {
#pragma unroll
                for (int e = 0; e < 8; ++e) out.y.v[e] = of == 1 ? (T)0.f : Elem<T>::nan();
            }
            T* to = static_cast<T*>(a.Y) + (first + p) * a.ldy + c;
            if (columns.skip == 0) {
                out.store(to, 8);
            } else if (columns.skip < 8) {  // its scale is that of the columns that are its own
#pragma unroll
                for (int e = 1; e < 8; ++e)
                    if (e >= columns.skip) to[e] = out.y.v[e];
            }
            now = next;
        }
    }
}

template <typename T>
static void (*lookup_for(int d))(const LookupArgs) {
    return d == 1 ? &k_lookup_codes_fast<T, 1> : d == 2 ? &k_lookup_codes_fast<T, 2> : d == 4 ? &k_lookup_codes_fast<T, 4> : &k_lookup_codes_fast<T, 8>;
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
    if (a.bits <= 8 && (a.d == 1 || a.d == 2 || a.d == 4 || a.d == 8) && a.nwords >= 3 && a.cols >= 8) {
        const int64_t strips = (a.cols + 511) / 512;
        a.each = (int)std::max<int64_t>(1, std::min<int64_t>(16, a.ids.n * strips / 8192));
        const int64_t tasks = (a.ids.n + a.each - 1) / a.each * strips;
        const unsigned grid = (unsigned)std::min<int64_t>((tasks + 3) / 4, 2048);
        BY_TYPE(dtype, T, hipLaunchKernelGGL(lookup_for<T>(a.d), dim3(grid), dim3(256), ((size_t)a.d << a.bits) * sizeof(T), s, a));
        return;
    }
    const size_t book = (size_t)a.k * a.d * (dtype == 0 ? 4 : 2);
    a.c_in_lds = book <= 32 * 1024;
    BY_TYPE(dtype, T, hipLaunchKernelGGL(k_lookup_codes<T>, dim3(grid_of(a.ids.n * ((a.cols + 7) / 8), 2048)), dim3(256), a.c_in_lds ? book : 0, s, a));
}

}  // namespace idkm

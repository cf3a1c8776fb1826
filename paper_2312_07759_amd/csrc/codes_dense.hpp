// Kernels around the tile product: layers written out as matrices, operands padded and transposed, parts of a sum joined.
#pragma once
#include "codes_product.hpp"

namespace idkm {

// A layer's rows [r0, r0 + nr) or columns [c0, c0 + nc), as the tile product takes them.
struct DenseArgs {
    const uint32_t* words;
    int64_t nwords;
    int64_t rows, cols;  // of the whole layer
    const void* C;       // T [k, d]
    int k, d, bits;
    int c_in_lds;
    const float* S;  // [rows, groups] or null
    int group, groups;
    int64_t first, count;  // rows (or, transposed, columns) to write
    int64_t pad;           // columns (transposed: rows) of the written matrix, zero from the layer's end on
    void* out;             // T [count, pad]
    unsigned group_magic;  // ceil(2^31 / (group / 32)), or 0 for one group
    int group_32;          // group / 32
    int64_t row_bits;
    int d_log;  // of d in {1, 2, 4, 8}
    // rows only: the codewords go out as they are, and S transposed to scales_out [groups, scale_pitch], row `first` its first
    float* scales_out;  // or null
    int64_t scale_pitch;
};

// Group of column c: the product with the rounded-up inverse is off by one at most, and then too large.
__device__ __forceinline__ int group_of(const DenseArgs& a, int c) {
    const unsigned x = (unsigned)c >> 5;
    unsigned g = __umulhi(2u * x, a.group_magic);
    if (__umul24(g, (unsigned)a.group_32) > x) --g;  // both below 2^17
    return (int)g;
}

// A 64 x 64 tile through LDS: every thread of 256 brings columns 8 c .. 8 c + 7 of rows 2 p and 2 p + 1 (p = thread / 8, c = thread
// % 8) and the tile goes out as 64 rows of its transpose, 16 bytes at a time.
template <typename T>
struct TransposeTile {
    static constexpr int PITCH = sizeof(T) == 4 ? 65 : 33;  // words between columns
    static constexpr int WORDS = 64 * PITCH;
    uint32_t* lds;
    __device__ __forceinline__ void put(const T* a, const T* b) const {
        const int p = threadIdx.x >> 3, c = (threadIdx.x & 7) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (sizeof(T) == 4) {
                lds[(c + e) * PITCH + 2 * p] = __builtin_bit_cast(uint32_t, a[e]);
                lds[(c + e) * PITCH + 2 * p + 1] = __builtin_bit_cast(uint32_t, b[e]);
            } else {
                lds[(c + e) * PITCH + p] = __builtin_bit_cast(uint16_t, a[e]) | (uint32_t)__builtin_bit_cast(uint16_t, b[e]) << 16;
            }
        }
    }
    // out: the tile's first element; columns left to write, elements between their rows, elements of a row there is room for
    __device__ __forceinline__ void emit(T* out, int64_t columns, int64_t pitch, int64_t room) const {
        constexpr int PIECES = 64 * (int)sizeof(T) / 16;
#pragma unroll
        for (int i = 0; i < 64 * PIECES / 256; ++i) {
            const int at = i * 256 + threadIdx.x, c = at / PIECES, k = at % PIECES;
            if (c >= columns || k * Elem<T>::PER16 >= room) continue;  // room is a multiple of a piece
            const uint32_t* w = lds + c * PITCH + k * 4;
            *reinterpret_cast<u32x4*>(out + c * pitch + k * Elem<T>::PER16) = u32x4{w[0], w[1], w[2], w[3]};
        }
    }
};

// Eight columns of a row of the layer on their way: asked for, and brought to T.  Where the weights are scaled here (columns, for dX, along
// whose sum every weight has another scale; and float32) each is rounded once: it is an operand of the matrix instruction, and the
// relative error, eps / 2 at most, is that of a weight stored in T.  Zeros behind the last column.
template <typename T, int IB, int W, bool ALIGNED>
struct EightOfLayer {
    static constexpr int NB = 8 / W * IB;
    CodeRun<NB> run;
    float s;
    // row_bit, row_scale: where row r's codes and scales begin, r row_bits and r groups
    __device__ __forceinline__ void ask(const DenseArgs& a, int64_t row_bit, int64_t row_scale, int c) {
        const int64_t bit = row_bit + (unsigned)((c >> a.d_log) * a.bits);
        if (c + 8 <= a.cols) {
            const int64_t base = ALIGNED ? bit >> 5 : min(bit >> 5, a.nwords - CodeRun<NB>::SPAN);
            run.template load_inside<ALIGNED>(a.words + base, 0, (unsigned)(bit - (base << 5)));
        } else {
            run.template load<false, true>(a.words, a.nwords, bit);
        }
        if (a.S) s = a.S[row_scale + group_of(a, c)];
    }
    // in the place of scaling the weights: the thread of a group's first columns writes its scale, of row r
    __device__ __forceinline__ void put_scale(const DenseArgs& a, int r, int c) const {
        const int g = group_of(a, c);
        if (g * a.group == c) a.scales_out[g * a.scale_pitch + r] = s;
    }
    __device__ __forceinline__ void bring(T* out, const DenseArgs& a, int c, const unsigned char* table) const {
        u32x4 raw[8 / Elem<T>::PER16];
        eight_weights<T, IB, W, NB>(raw, run, 0, table);
        __builtin_memcpy(out, raw, sizeof(raw));
        if (a.S && !a.scales_out) {
#pragma unroll
            for (int e = 0; e < 8; ++e) out[e] = Elem<T>::down(Elem<T>::up(out[e]) * s);
        }
        if (c + 8 > a.cols) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + e >= a.cols) out[e] = (T)0.f;
        }
    }
};

// The layer's rows: a thread takes 8 columns at a time, four such pieces asked for together, the first before the table is built and the
// next before these are brought.  4096 x 4096 in 16 bits takes 11.2 us (26 with one code read at a time, 15 with one piece, 12.5 with the pieces asked
// for when they are needed), 12 to 14 with the scales written beside the codewords; bound by issue: some 80 instructions for 8 scaled weights are 5 us, and written at the
// rate of a fill it is 5.
template <typename T, int IB, int W, bool ALIGNED>
__global__ __launch_bounds__(256) void k_dense_rows_fast(const DenseArgs a) {
    constexpr int U = 4;
    extern __shared__ __align__(128) unsigned char lds[];
    const Table<T, IB, W> entries(a.C, a.k, a.bits, a.d);
    const unsigned char* table = Table<T, IB, W>::own(lds);
    const int per_row = (int)(a.pad / 8);
    // a thread's next piece is `step` pieces on: its row, column, codes and scales follow by additions
    const int64_t step = (int64_t)gridDim.x * 256, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int rows_step = (int)(step / per_row), cols_step = (int)(step - (int64_t)rows_step * per_row), count = (int)a.count;
    const int64_t bits_step = rows_step * a.row_bits, scales_step = (int64_t)rows_step * a.groups;
    int r = (int)min(at / per_row, (int64_t)count);
    int c = (int)(at - at / per_row * per_row);
    int64_t row_bit = (a.first + r) * a.row_bits, row_scale = (a.first + r) * a.groups;
    struct Batch {
        EightOfLayer<T, IB, W, ALIGNED> eight[U];
        int rows[U], cols[U];
    };
    auto ask = [&](Batch& b) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            b.rows[u] = r;
            b.cols[u] = c * 8;
            if (r < count && c * 8 < a.cols) b.eight[u].ask(a, row_bit, row_scale, c * 8);
            r += rows_step;
            row_bit += bits_step;
            row_scale += scales_step;
            c += cols_step;
            if (c >= per_row) {
                c -= per_row;
                ++r;
                row_bit += a.row_bits;
                row_scale += a.groups;
            }
        }
    };
    T* out = static_cast<T*>(a.out) + at * 8;
    Batch now, next;
    ask(now);
    entries.build(lds, a.C, a.k, a.bits, a.d);
    __syncthreads();
    for (; now.rows[0] < count; out += U * step * 8) {
        ask(next);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (now.rows[u] >= count) continue;
            struct alignas(16) Eight { T v[8]; } w;
            if (now.cols[u] < a.cols) {
                now.eight[u].bring(w.v, a, now.cols[u], table);
                if (a.scales_out) now.eight[u].put_scale(a, now.rows[u], now.cols[u]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) w.v[e] = (T)0.f;
            }
            *reinterpret_cast<Eight*>(out + u * step * 8) = w;
        }
        now = next;
    }
}

// The layer's columns: out[c, r] = w[r, c], 64 x 64 weights at a time, the next tile's asked for before this one goes through LDS.
// 4096 x 4096 in 16 bits: 17 us (24 with nothing asked for ahead); bound by the lookups and the LDS traffic of the transposition.
template <typename T, int IB, int W, bool ALIGNED>
__global__ __launch_bounds__(256) void k_dense_cols_fast(const DenseArgs a) {
    extern __shared__ __align__(128) unsigned char lds[];
    const Table<T, IB, W> entries(a.C, a.k, a.bits, a.d);
    const unsigned char* table = Table<T, IB, W>::own(lds);
    const TransposeTile<T> tile{reinterpret_cast<uint32_t*>(lds + Table<T, IB, W>::BYTES)};
    const int tiles_c = (int)((a.count + 63) / 64), tiles_r = (int)((a.pad + 63) / 64);
    const int lr = (threadIdx.x >> 3) * 2, lc = (threadIdx.x & 7) * 8;
    EightOfLayer<T, IB, W, ALIGNED> eight[2];
    auto ask = [&](int t) {
        const int tr = t / tiles_c, c0 = (int)a.first + (t - tr * tiles_c) * 64 + lc;
#pragma unroll
        for (int b = 0; b < 2; ++b)
            if (tr * 64 + lr + b < a.rows && c0 < a.cols) eight[b].ask(a, (tr * 64 + lr + b) * a.row_bits, (int64_t)(tr * 64 + lr + b) * a.groups, c0);
    };
    int t = blockIdx.x;
    if (t < tiles_c * tiles_r) ask(t);
    entries.build(lds, a.C, a.k, a.bits, a.d);
    for (; t < tiles_c * tiles_r; t += gridDim.x) {
        const int tr = t / tiles_c, tc = t - tr * tiles_c;
        const int c0 = (int)a.first + tc * 64 + lc;
        T w[2][8];
        __syncthreads();  // the table is there, and the last tile has gone out
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            if (tr * 64 + lr + b < a.rows && c0 < a.cols) {
                eight[b].bring(w[b], a, c0, table);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) w[b][e] = (T)0.f;
            }
        }
        if (t + (int)gridDim.x < tiles_c * tiles_r) ask(t + gridDim.x);
        tile.put(w[0], w[1]);
        __syncthreads();
        tile.emit(static_cast<T*>(a.out) + (int64_t)tc * 64 * a.pad + tr * 64, a.count - tc * 64, a.pad, a.pad - tr * 64);
    }
}

// Codes of more bits and codewords of other lengths, one code at a time.
__device__ __forceinline__ uint32_t code_at(const uint32_t* words, int64_t nwords, int64_t i, int bits) {
    const int64_t off = i * bits, w = off >> 5;
    const int sh = (int)(off & 31);
    unsigned long long win = words[w];
    if (sh + bits > 32) win |= (unsigned long long)words[min(w + 1, nwords - 1)] << 32;
    return (uint32_t)(win >> sh) & ((1u << bits) - 1u);
}

// Weight (r, c) of the layer in T.  A scaled codeword is rounded once, to T: it is an operand of the matrix instruction,
// and its relative error, eps / 2 at most, is that of a weight stored in T.
template <typename T>
__device__ __forceinline__ T weight_of(uint32_t code, int x, const T* C, int k, int d, float s, bool scaled) {
    if (code >= (uint32_t)k) return Elem<T>::nan();
    const T v = C[(int64_t)code * d + x];
    return scaled ? Elem<T>::down(Elem<T>::up(v) * s) : v;
}

// Thread: 8 consecutive columns of a row.
template <typename T>
__global__ __launch_bounds__(256) void k_dense_rows(const DenseArgs a) {
    extern __shared__ __align__(16) unsigned char lds[];
    const T* C = static_cast<const T*>(a.C);
    if (a.c_in_lds) {
        T* s = reinterpret_cast<T*>(lds);
        for (int i = threadIdx.x; i < a.k * a.d; i += 256) s[i] = C[i];
        __syncthreads();
        C = s;
    }
    const int64_t per_row = a.pad / 8, total = a.count * per_row;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < total; at += (int64_t)gridDim.x * 256) {
        const int64_t rr = at / per_row, r = a.first + rr, c0 = (at - rr * per_row) * 8;
        struct alignas(16) Eight { T v[8]; } w;
        int64_t j = c0 / a.d;  // codeword of column c0 in its row
        int x = (int)(c0 - j * a.d);
        const int64_t i0 = r * (a.cols / a.d);
        uint32_t code = 0;
        float s = 1.f;
        if (c0 < a.cols) {
            code = code_at(a.words, a.nwords, i0 + j, a.bits);
            if (a.S) s = a.S[r * a.groups + c0 / a.group];  // groups are multiples of 32: eight columns lie in one
            if (a.scales_out && c0 % a.group == 0) a.scales_out[c0 / a.group * a.scale_pitch + rr] = s;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (c0 + e >= a.cols) {
                w.v[e] = (T)0.f;
                continue;
            }
            w.v[e] = weight_of<T>(code, x, C, a.k, a.d, s, a.S != nullptr && !a.scales_out);
            if (++x == a.d) {
                x = 0;
                ++j;
                if (e < 7 && c0 + e + 1 < a.cols) code = code_at(a.words, a.nwords, i0 + j, a.bits);
            }
        }
        constexpr int NV = sizeof(Eight) / 16;
        u32x4 v[NV];
        __builtin_memcpy(v, &w, sizeof(w));
        u32x4* o = reinterpret_cast<u32x4*>(static_cast<T*>(a.out) + rr * a.pad + c0);
#pragma unroll
        for (int f = 0; f < NV; ++f) o[f] = v[f];
    }
}

// 64 columns x 64 rows through LDS: out[c, r] = w[r, c].
template <typename T>
__global__ __launch_bounds__(256) void k_dense_cols(const DenseArgs a) {
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ T tile[64][64 + 16 / sizeof(T) / 2];
    const T* C = static_cast<const T*>(a.C);
    if (a.c_in_lds) {
        T* s = reinterpret_cast<T*>(lds);
        for (int i = threadIdx.x; i < a.k * a.d; i += 256) s[i] = C[i];
        C = s;
        __syncthreads();
    }
    const int64_t cb = a.first + (int64_t)blockIdx.x * 64, rb = (int64_t)blockIdx.y * 64;
    const int64_t c_end = min(a.cols, a.first + a.count);
    // thread: 16 columns of one row
    {
        const int64_t r = rb + (threadIdx.x >> 2), c0 = cb + (threadIdx.x & 3) * 16;
        int64_t j = c0 / a.d;
        int x = (int)(c0 - j * a.d);
        const int64_t i0 = r * (a.cols / a.d);
        const bool row_there = r < a.rows;
        uint32_t code = 0;
        float s = 1.f;
        if (row_there && c0 < c_end) {
            code = code_at(a.words, a.nwords, i0 + j, a.bits);
            if (a.S) s = a.S[r * a.groups + c0 / a.group];  // c0 is a multiple of 16
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            T v = (T)0.f;
            if (row_there && c0 + e < c_end) {
                v = weight_of<T>(code, x, C, a.k, a.d, s, a.S != nullptr);
                if (++x == a.d) {
                    x = 0;
                    ++j;
                    if (e < 15 && c0 + e + 1 < c_end) code = code_at(a.words, a.nwords, i0 + j, a.bits);
                }
            }
            tile[(threadIdx.x & 3) * 16 + e][threadIdx.x >> 2] = v;
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < 64 * 64; e += 256) {
        const int64_t c = cb + (e >> 6), r = rb + (e & 63);
        if (c < c_end && r < a.pad) static_cast<T*>(a.out)[(c - a.first) * a.pad + r] = tile[e >> 6][e & 63];
    }
}

// Operands brought to the form in which the tile product takes them, several in one launch.
//   rows        out[M, pad] = in[M, N], zero behind column N
//   transposed  out[N, pad] = in[M, N]^T, zero behind column M
struct Operand {
    const void* in;
    int64_t ldi, M, N;
    void* out;
    int64_t pad;
    int transposed;
    int64_t tiles, tiles_n;  // of 64 x 64, and along N (rows: along pad)
};
struct OperandArgs {
    Operand job[3];
    int jobs;
};

template <typename T>
__global__ __launch_bounds__(256) void k_operands(const OperandArgs a) {
    __shared__ __align__(16) uint32_t lds[TransposeTile<T>::WORDS];
    int64_t t = blockIdx.x;
    int j = 0;
    while (j + 1 < a.jobs && t >= a.job[j].tiles) t -= a.job[j++].tiles;
    const Operand& o = a.job[j];
    const int64_t tm = t / o.tiles_n, m0 = tm * 64, n0 = (t - tm * o.tiles_n) * 64;
    const int64_t m = m0 + (threadIdx.x >> 3) * 2, n = n0 + (threadIdx.x & 7) * 8;
    struct alignas(16) Eight { T v[8]; } v[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const T* row = static_cast<const T*>(o.in) + (m + b) * o.ldi;
        if (m + b < o.M && n + 8 <= o.N) {
            u32x4 raw[8 / Elem<T>::PER16];
#pragma unroll
            for (int f = 0; f < 8 / Elem<T>::PER16; ++f) raw[f] = reinterpret_cast<const u32x4_any*>(row + n)[f];
            __builtin_memcpy(v[b].v, raw, sizeof(raw));
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[b].v[e] = m + b < o.M && n + e < o.N ? row[n + e] : (T)0.f;
        }
    }
    if (o.transposed) {  // the same for the whole workgroup
        const TransposeTile<T> tile{lds};
        tile.put(v[0].v, v[1].v);
        __syncthreads();
        tile.emit(static_cast<T*>(o.out) + n0 * o.pad + m0, o.N - n0, o.pad, o.pad - m0);
    } else {
#pragma unroll
        for (int b = 0; b < 2; ++b)
            if (m + b < o.M && n < o.pad) *reinterpret_cast<Eight*>(static_cast<T*>(o.out) + (m + b) * o.pad + n) = v[b];
    }
}

// out[M, N] (rows ldo apart) = the sum over z, in order, of parts[z, M, N].  out may be the first part.
template <typename T>
__global__ __launch_bounds__(256) void k_join_parts(const float* parts, int nz, int64_t M, int64_t N, T* out, int64_t ldo) {
    const int64_t total = M * N;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < total; at += (int64_t)gridDim.x * 256) {
        float sum = parts[at];
        for (int z = 1; z < nz; ++z) sum += parts[z * total + at];
        const int64_t m = at / N;
        out[m * ldo + (at - m * N)] = Elem<T>::down(sum);
    }
}

}  // namespace idkm

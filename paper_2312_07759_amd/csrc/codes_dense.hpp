// Kernels around the tile product: layers written out as matrices, operands padded and transposed, parts of a sum joined.
#pragma once
#include "elem.hpp"

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
};

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
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (c0 + e >= a.cols) {
                w.v[e] = (T)0.f;
                continue;
            }
            w.v[e] = weight_of<T>(code, x, C, a.k, a.d, s, a.S != nullptr);
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

// out[M, pad] = in[M, N] with rows ldi apart, zero behind column N.
template <typename T>
__global__ __launch_bounds__(256) void k_pad_rows(const T* __restrict__ in, int64_t ldi, int64_t M, int64_t N, T* __restrict__ out, int64_t pad) {
    const int64_t total = M * pad;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < total; at += (int64_t)gridDim.x * 256) {
        const int64_t m = at / pad, n = at - m * pad;
        out[at] = n < N ? in[m * ldi + n] : (T)0.f;
    }
}

// out[N, pad] = in[M, N]^T, zero behind column M.
template <typename T>
__global__ __launch_bounds__(256) void k_transpose(const T* __restrict__ in, int64_t ldi, int64_t M, int64_t N, T* __restrict__ out, int64_t pad) {
    __shared__ T tile[64][64 + 16 / sizeof(T) / 2];
    const int64_t nb = (int64_t)blockIdx.x * 64, mb = (int64_t)blockIdx.y * 64;
    for (int e = threadIdx.x; e < 64 * 64; e += 256) {
        const int64_t m = mb + (e >> 6), n = nb + (e & 63);
        tile[e & 63][e >> 6] = m < M && n < N ? in[m * ldi + n] : (T)0.f;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < 64 * 64; e += 256) {
        const int64_t n = nb + (e >> 6), m = mb + (e & 63);
        if (n < N && m < pad) out[n * pad + m] = tile[e >> 6][e & 63];
    }
}

// out[M, N] (rows ldo apart) = the sum over z, in order, of parts[z, M, N].
template <typename T>
__global__ __launch_bounds__(256) void k_join_parts(const float* __restrict__ parts, int nz, int64_t M, int64_t N, T* __restrict__ out, int64_t ldo) {
    const int64_t total = M * N;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < total; at += (int64_t)gridDim.x * 256) {
        float sum = parts[at];
        for (int z = 1; z < nz; ++z) sum += parts[z * total + at];
        const int64_t m = at / N;
        out[m * ldo + (at - m * N)] = Elem<T>::down(sum);
    }
}

}  // namespace idkm

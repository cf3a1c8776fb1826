// Products in 8-bit integers: rows of numbers brought to integers, and few tokens times a layer.  Many tokens: tile_product.hpp.
//
// A row x has the scale s = max(max |x| / 127, 2^-126), a float32 number, and the integers q = x / s to the nearest, ties to even, exactly.  Sums of q
// times the layer's integers are exact in 32 bits; a result is rounded where the sum becomes a float32 number, at the two scales and to its type.
// A row that holds an infinity or NaN has the scale NaN (and integers 0), which makes its results NaN.
#include "layers.h"

namespace idkm {

__device__ __forceinline__ uint32_t size_of(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffff; }

struct RowScale {
    float s, inverse;
    // top: bits of the largest size, infinities and NaN included (which are the largest)
    __device__ __forceinline__ explicit RowScale(uint32_t top) {
        s = top >= 0x7f800000 ? __builtin_nanf("") : fmaxf(__builtin_bit_cast(float, top) / 127.f, 0x1p-126f);
        inverse = 1.f / s;
    }
    // The product with the rounded inverse is at most one off.  What is left, x - q s, is exact where it decides: it is a multiple of half the last
    // place of s and no larger than about s / 2; where it is rounded (x below s / 2, q = 1) it cannot become smaller than s / 2.
    __device__ __forceinline__ int integer(float x) const {
        float q = __builtin_rintf(x * inverse);
        const float left = fmaf(-q, s, x), half = 0.5f * s;
        const bool odd = ((int)q & 1) != 0;
        q += left > half || (left == half && odd) ? 1.f : 0.f;
        q -= left < -half || (left == -half && odd) ? 1.f : 0.f;
        return (int)q;
    }
};

// Eight elements of a row as float32, zero behind its end.
template <typename T>
__device__ __forceinline__ void eight_floats(float* v, const T* row, int64_t c, int64_t cols) {
    struct alignas(16) Eight { T v[8]; } y;
    if (c + 8 <= cols) {
        u32x4 raw[8 / Elem<T>::PER16];
#pragma unroll
        for (int f = 0; f < 8 / Elem<T>::PER16; ++f) raw[f] = reinterpret_cast<const u32x4_any*>(row + c)[f];
        __builtin_memcpy(&y, raw, sizeof(y));
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) y.v[e] = c + e < cols ? row[c + e] : (T)0.f;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = Elem<T>::up(y.v[e]);
}

__device__ __forceinline__ uint32_t larger_of_wave(uint32_t top) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    return top;
}

__device__ __forceinline__ u32x2 eight_integers(const RowScale& s, const float* v) {
    u32x2 q{0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e >> 2] |= ((uint32_t)s.integer(v[e]) & 255u) << (e & 3) * 8;
    return q;
}

// A workgroup to a row; up to 8192 columns stay in registers between the two looks at them.
template <typename T>
__global__ __launch_bounds__(256) void k_int8_rows(const Int8RowsArgs a) {
    constexpr int HELD = 4;
    __shared__ uint32_t tops[4];
    const int64_t t = blockIdx.x;
    const T* row = static_cast<const T*>(a.X) + t * a.ldx;
    float v[HELD][8];
    uint32_t top = 0;
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
        const int64_t c = (h * 256 + threadIdx.x) * 8;
        if (c < a.ldq) eight_floats(v[h], row, c, a.cols);
    }
#pragma unroll
    for (int h = 0; h < HELD; ++h)
        if ((h * 256 + (int)threadIdx.x) * 8 < a.ldq) {
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, size_of(v[h][e]));
        }
    for (int64_t c = (HELD * 256 + threadIdx.x) * 8; c < a.cols; c += 2048) {
        float w[8];
        eight_floats(w, row, c, a.cols);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, size_of(w[e]));
    }
    top = larger_of_wave(top);
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    const RowScale s(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
    if (threadIdx.x == 0) a.scale[t] = s.s;
    int8_t* out = a.Q + t * a.ldq;
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
        const int64_t c = (h * 256 + threadIdx.x) * 8;
        if (c < a.ldq) *reinterpret_cast<u32x2*>(out + c) = eight_integers(s, v[h]);
    }
    for (int64_t c = (HELD * 256 + threadIdx.x) * 8; c < a.ldq; c += 2048) {
        float w[8];
        eight_floats(w, row, c, a.cols);
        *reinterpret_cast<u32x2*>(out + c) = eight_integers(s, w);
    }
}

void launch_int8_rows(int dtype, const Int8RowsArgs& a, hipStream_t s) {
    BY_TYPE(dtype, T, hipLaunchKernelGGL(k_int8_rows<T>, dim3((unsigned)a.n), dim3(256), 0, s, a));
}

// 16 rows of the layer and 16 NT tokens to a workgroup, whose eight wavefronts share the sum in chunks of 256 columns; lane l has row l % 16 and, of
// every 64 columns, the 16 of quarter l / 16.  The layer's first integers are asked for before the tokens are looked at.
// FUSED (up to INT8_FUSED elements of X, NT = 1): every workgroup brings the tokens to integers itself, into LDS, instead of a launch before this one.
template <typename T, int NT, bool FUSED>
__global__ __launch_bounds__(512) void k_int8_few(const Int8FewArgs a) {
    constexpr int U = 4;  // 64 columns each: a chunk
    extern __shared__ __align__(16) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = lane & 15, q = lane >> 4;
    const int64_t r0 = (int64_t)blockIdx.x * 16, t0 = (int64_t)blockIdx.y * 16 * NT;
    const int8_t* W = a.W8 + min(r0 + li, a.rows - 1) * a.ldw + q * 16;  // rows and tokens behind the last: computed from it, not stored
    const int steps = (int)(a.pad / 64), each = ((steps + 7) / 8 + U - 1) / U * U;
    const int first = min(steps, wave * each), last = min(steps, first + each);
    u32x4 w[2][U];
    auto ask = [&](int of, int step) {
#pragma unroll
        for (int u = 0; u < U; ++u) w[of][u] = *reinterpret_cast<const u32x4*>(W + (int64_t)min(step + u, steps - 1) * 64);
    };
    if (first < last) {
        ask(0, first);
        ask(1, first + U);
    }
    float scales[NT][4];
    const int8_t* X[NT];
    if constexpr (FUSED) {
        uint32_t* tops = reinterpret_cast<uint32_t*>(lds);  // [n][8]
        int8_t* held = reinterpret_cast<int8_t*>(lds) + 512;  // [n][pad]
        const int n = (int)a.n;
        for (int t = 0; t < n; ++t) {
            uint32_t top = 0;
            for (int64_t c = threadIdx.x * 8; c < a.cols; c += 4096) {
                float v[8];
                eight_floats(v, static_cast<const T*>(a.X) + t * a.ldx, c, a.cols);
#pragma unroll
                for (int e = 0; e < 8; ++e) top = max(top, size_of(v[e]));
            }
            top = larger_of_wave(top);
            if (lane == 0) tops[t * 8 + wave] = top;
        }
        __syncthreads();
        for (int t = 0; t < n; ++t) {
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, tops[t * 8 + i]);
            const RowScale s(top);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (q * 4 + r == t) scales[0][r] = s.s;
            for (int64_t c = threadIdx.x * 8; c < a.pad; c += 4096) {
                float v[8];
                eight_floats(v, static_cast<const T*>(a.X) + t * a.ldx, c, a.cols);
                *reinterpret_cast<u32x2*>(held + t * a.pad + c) = eight_integers(s, v);
            }
        }
        __syncthreads();
        X[0] = held + min(li, n - 1) * a.pad + q * 16;
    } else {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            X[i] = a.Q + min(t0 + i * 16 + li, a.n - 1) * a.pad + q * 16;
#pragma unroll
            for (int r = 0; r < 4; ++r) scales[i][r] = a.q_scale[min(t0 + i * 16 + q * 4 + r, a.n - 1)];
        }
    }
    intx4 acc[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) acc[i] = intx4{0, 0, 0, 0};
    auto use = [&](int of, int step) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (step + u >= last) break;
#pragma unroll
            for (int i = 0; i < NT; ++i) mma16<int8_t>(acc[i], *reinterpret_cast<const u32x4*>(X[i] + (int64_t)(step + u) * 64), w[of][u]);
        }
    };
    for (int step = first; step < last; step += 2 * U) {
        use(0, step);
        if (step + 2 * U < last) ask(0, step + 2 * U);
        if (step + U < last) {
            use(1, step + U);
            if (step + 3 * U < last) ask(1, step + 3 * U);
        }
    }
    // the wavefronts' sums, exact in any order
    __syncthreads();
    int* sums = reinterpret_cast<int*>(lds);  // [NT][8][256]
#pragma unroll
    for (int i = 0; i < NT; ++i) *reinterpret_cast<intx4*>(sums + ((i * 8 + wave) * 64 + lane) * 4) = acc[i];
    __syncthreads();
    if (wave >= NT) return;
    // wavefront i: tokens i 16 + 4 q + r of row li
    float s[4];
#pragma unroll
    for (int i = 0; i < NT; ++i)
        if (wave == i) {
#pragma unroll
            for (int r = 0; r < 4; ++r) s[r] = scales[i][r];
        }
    intx4 sum{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += *reinterpret_cast<const intx4*>(sums + ((wave * 8 + i) * 64 + lane) * 4);
    if (r0 + li >= a.rows) return;
    const float by = a.scale[r0 + li];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int64_t t = t0 + wave * 16 + q * 4 + r;
        if (t < a.n) static_cast<T*>(a.Y)[t * a.ldy + r0 + li] = Elem<T>::down((float)sum[r] * s[r] * by);
    }
}

template <typename T, int NT, bool FUSED>
static void launch_few(const Int8FewArgs& a, hipStream_t s) {
    const size_t sums = (size_t)NT * 8192, held = FUSED ? 512 + (size_t)(a.n * a.pad) : 0, lds = held > sums ? held : sums;
    void (*const fn)(const Int8FewArgs) = &k_int8_few<T, NT, FUSED>;
    allow_lds(reinterpret_cast<const void*>(fn), lds);
    hipLaunchKernelGGL(fn, dim3((unsigned)((a.rows + 15) / 16), (unsigned)((a.n + 16 * NT - 1) / (16 * NT))), dim3(512), lds, s, a);
}

void launch_int8_few(int dtype, const Int8FewArgs& a, hipStream_t s) {
    if (!a.Q) BY_TYPE(dtype, T, (launch_few<T, 1, true>(a, s)));
    else if (a.n <= 16) BY_TYPE(dtype, T, (launch_few<T, 1, false>(a, s)));
    else if (a.n <= 32) BY_TYPE(dtype, T, (launch_few<T, 2, false>(a, s)));
    else BY_TYPE(dtype, T, (launch_few<T, 4, false>(a, s)));
}

template <typename T>
__global__ __launch_bounds__(256) void k_join_int8(const int32_t* __restrict__ parts, int nz, int64_t M, int64_t N, const float* __restrict__ by_m,
                                                   const float* __restrict__ by_n, T* __restrict__ out, int64_t ldo) {
    const int64_t total = M * N;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < total; at += (int64_t)gridDim.x * 256) {
        int sum = parts[at];
        for (int z = 1; z < nz; ++z) sum += parts[z * total + at];
        const int64_t m = at / N, n = at - m * N;
        out[m * ldo + n] = Elem<T>::down((float)sum * by_m[m] * by_n[n]);
    }
}

void launch_join_int8(int dtype, const int32_t* parts, int nz, int64_t M, int64_t N, const float* by_m, const float* by_n, void* out, int64_t ldo,
                      hipStream_t s) {
    const int64_t g = (M * N + 255) / 256;
    BY_TYPE(dtype, T, hipLaunchKernelGGL(k_join_int8<T>, dim3((unsigned)(g > 8192 ? 8192 : g)), dim3(256), 0, s, parts, nz, M, N, by_m, by_n,
                                         static_cast<T*>(out), ldo));
}

}  // namespace idkm

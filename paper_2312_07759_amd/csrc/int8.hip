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
    // Eight integers, as bytes.  The product with the rounded inverse differs from the quotient by less than 2^-15, so its nearest integer is the quotient's unless it
    // lies beside a tie; then what is left, x - q s, decides, which is exact where it does: it is a multiple of half the last place of s and no larger than
    // about s / 2; where it is rounded (x below s / 2, q = 1) it cannot become smaller than s / 2.
    __device__ __forceinline__ u32x2 integers(const float* x) const {
        float q[8], beside = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float m = x[e] * inverse;
            q[e] = __builtin_rintf(m);
            beside = fmaxf(beside, fabsf(m - q[e]));
        }
        if (__any(beside > 0.5f - 0x1p-14f)) {
            const float half = 0.5f * s;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float left = fmaf(-q[e], s, x[e]);
                const bool odd = ((int)q[e] & 1) != 0;
                q[e] += (left > half || (left == half && odd) ? 1.f : 0.f) - (left < -half || (left == -half && odd) ? 1.f : 0.f);
            }
        }
        uint32_t b[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = (uint32_t)(int)q[e];
        // the low bytes of two registers, then of two pairs
        auto pair = [](uint32_t low, uint32_t high) { return __builtin_amdgcn_perm(high, low, 0x0c0c0400u); };
        return u32x2{pair(b[0], b[1]) | pair(b[2], b[3]) << 16, pair(b[4], b[5]) | pair(b[6], b[7]) << 16};
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

__device__ __forceinline__ uint32_t larger_of_eight(uint32_t top, const float* v) {
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, size_of(v[e]));
    return top;
}

// A workgroup to a row; up to 4096 columns stay in registers between the two looks at them.
// 2048 rows of 4096 columns, bfloat16: 8 to 10 us (a copy's rate: 5; every quotient decided by what is left: 9.6; a wavefront to a row, without a barrier: 10).
template <typename T>
__global__ __launch_bounds__(256) void k_int8_rows(const Int8RowsArgs a) {
    constexpr int HELD = 2;
    __shared__ uint32_t tops[4];
    const int64_t t = blockIdx.x;
    const T* row = static_cast<const T*>(a.X) + t * a.ldx;
    float v[HELD][8];
    uint32_t top = 0;
#pragma unroll
    for (int h = 0; h < HELD; ++h) eight_floats(v[h], row, (int64_t)(h * 256 + threadIdx.x) * 8, a.cols);
#pragma unroll
    for (int h = 0; h < HELD; ++h) top = larger_of_eight(top, v[h]);
    for (int64_t c = (HELD * 256 + threadIdx.x) * 8; c < a.cols; c += 2048) {
        float w[8];
        eight_floats(w, row, c, a.cols);
        top = larger_of_eight(top, w);
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
        const u32x2 q = s.integers(v[h]);
        if (c < a.ldq) *reinterpret_cast<u32x2*>(out + c) = q;
    }
    for (int64_t c = (HELD * 256 + threadIdx.x) * 8; c < a.ldq; c += 2048) {
        float w[8];
        eight_floats(w, row, c, a.cols);
        *reinterpret_cast<u32x2*>(out + c) = s.integers(w);
    }
}

void launch_int8_rows(int dtype, const Int8RowsArgs& a, hipStream_t s) {
    BY_TYPE(dtype, T, hipLaunchKernelGGL(k_int8_rows<T>, dim3((unsigned)a.n), dim3(256), 0, s, a));
}

// 16 rows of the layer and 16 NT tokens to a workgroup, whose WAVES wavefronts share the sum; lane l has row l % 16 and, of every 64 columns, the 16 of quarter
// l / 16.  Integers of four to eight such steps are asked for together, where there are registers the next ones
// before these are used.  The layer is read once for 16 NT tokens: 4096 x 4096 at one token 5.6 us, 3.0 TB/s (a copy's rate: 3.3 us); 41 tokens of 512 x 4608 7 us, the
// latency of four or five batches of loads, one after another, and of the joining of sixteen sums.
// FUSED (up to INT8_FUSED elements of X, NT = 1): every workgroup brings the tokens to integers itself, into LDS, instead of a launch before this one.
template <typename T, int NT, int WAVES, bool FUSED>
__global__ __launch_bounds__(64 * WAVES) void k_int8_few(const Int8FewArgs a) {
    constexpr int U = FUSED ? 8 : NT == 1 ? 6 : 4, XN = FUSED ? 1 : NT;
    constexpr bool AHEAD = FUSED || NT > 1;  // sixteen wavefronts have 128 registers each
    extern __shared__ __align__(16) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = lane & 15, q = lane >> 4;
    const int64_t r0 = (int64_t)blockIdx.x * 16, t0 = (int64_t)blockIdx.y * 16 * NT;
    const int8_t* W = a.W8 + min(r0 + li, a.rows - 1) * a.ldw + q * 16;  // rows and tokens behind the last: computed from it, not stored
    const int steps = (int)(a.pad / 64), each = (steps + WAVES - 1) / WAVES;
    const int first = min(steps, wave * each), last = min(steps, first + each);
    struct Batch {
        u32x4 w[U], x[XN][U];
    };
    const int8_t* X[XN];
    if constexpr (!FUSED) {
#pragma unroll
        for (int i = 0; i < NT; ++i) X[i] = a.Q + min(t0 + i * 16 + li, a.n - 1) * a.pad + q * 16;
    }
    auto ask = [&](Batch& b, int step) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t c = (int64_t)min(step + u, steps - 1) * 64;
            b.w[u] = *reinterpret_cast<const u32x4*>(W + c);
            if constexpr (!FUSED) {
#pragma unroll
                for (int i = 0; i < NT; ++i) b.x[i][u] = *reinterpret_cast<const u32x4*>(X[i] + c);
            }
        }
    };
    Batch now, next;
    if constexpr (!FUSED) ask(now, first);
    float scales[NT][4];
    if constexpr (FUSED) {
        // pieces of eight elements, up to HELD of a thread, which stay in its registers between the two looks at them
        constexpr int HELD = (int)(INT8_FUSED / 8 / (64 * WAVES));
        uint32_t* tops = reinterpret_cast<uint32_t*>(lds);    // [16]
        int8_t* held = reinterpret_cast<int8_t*>(lds) + 64;  // [n][pad]
        const int n = (int)a.n, of_row = (int)(a.pad / 8), pieces = n * of_row, cols = (int)a.cols;
        u32x4 raw[HELD][8 / Elem<T>::PER16];
        auto floats = [&](int h, float* v) {
            struct alignas(16) Eight { T v[8]; } y;
            __builtin_memcpy(&y, raw[h], sizeof(y));
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = Elem<T>::up(y.v[e]);
        };
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            const int piece = h * 64 * WAVES + (int)threadIdx.x;
            if (piece >= pieces) continue;
            const int t = piece / of_row, c = (piece - t * of_row) * 8;
            const T* row = static_cast<const T*>(a.X) + t * a.ldx;
            if (c + 8 <= cols) {
#pragma unroll
                for (int f = 0; f < 8 / Elem<T>::PER16; ++f) raw[h][f] = reinterpret_cast<const u32x4_any*>(row + c)[f];
            } else {
                struct alignas(16) Eight { T v[8]; } y;
#pragma unroll
                for (int e = 0; e < 8; ++e) y.v[e] = c + e < cols ? row[c + e] : (T)0.f;
                __builtin_memcpy(raw[h], &y, sizeof(y));
            }
        }
        ask(now, first);  // behind the tokens, which are waited for first
        if (threadIdx.x < 16) tops[threadIdx.x] = 0;
        __syncthreads();
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            const int piece = h * 64 * WAVES + (int)threadIdx.x;
            uint32_t top = 0;
            if (piece < pieces) {
                float v[8];
                floats(h, v);
                top = larger_of_eight(0, v);
            }
            if (h * 64 * WAVES >= pieces) continue;
            if (of_row % 64 == 0) {  // a wavefront's pieces are of one token
                top = larger_of_wave(top);
                if (lane == 0 && piece < pieces) atomicMax(&tops[piece / of_row], top);
            } else if (piece < pieces) {
                atomicMax(&tops[piece / of_row], top);
            }
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            const int piece = h * 64 * WAVES + (int)threadIdx.x;
            if (piece >= pieces) continue;
            float v[8];
            floats(h, v);
            *reinterpret_cast<u32x2*>(held + piece * 8) = RowScale(tops[piece / of_row]).integers(v);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) scales[0][r] = q * 4 + r < n ? RowScale(tops[q * 4 + r]).s : 0.f;
        __syncthreads();
        X[0] = held + min(li, n - 1) * (int)a.pad + q * 16;
    } else {
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) scales[i][r] = a.q_scale[min(t0 + i * 16 + q * 4 + r, a.n - 1)];
    }
    intx4 acc[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) acc[i] = intx4{0, 0, 0, 0};
    for (int step = first; step < last; step += U) {
        if (AHEAD && step + U < last) ask(next, step + U);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (step + u >= last) break;
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                if constexpr (FUSED) mma16<int8_t>(acc[i], *reinterpret_cast<const u32x4*>(X[i] + (step + u) * 64), now.w[u]);
                else mma16<int8_t>(acc[i], now.x[i][u], now.w[u]);
            }
        }
        if (AHEAD) now = next;
        else if (step + U < last) ask(now, step + U);
    }
    // the wavefronts' sums, exact in any order
    __syncthreads();
    int* sums = reinterpret_cast<int*>(lds);  // [NT][WAVES][256]
#pragma unroll
    for (int i = 0; i < NT; ++i) *reinterpret_cast<intx4*>(sums + ((i * WAVES + wave) * 64 + lane) * 4) = acc[i];
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
    for (int i = 0; i < WAVES; ++i) sum += *reinterpret_cast<const intx4*>(sums + ((wave * WAVES + i) * 64 + lane) * 4);
    if (r0 + li >= a.rows) return;
    const float by = a.scale[r0 + li];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int64_t t = t0 + wave * 16 + q * 4 + r;
        if (t < a.n) static_cast<T*>(a.Y)[t * a.ldy + r0 + li] = Elem<T>::down(TokenScale(s[r]).result(sum[r], by));
    }
}

template <typename T, int NT, int WAVES, bool FUSED>
static void launch_few(const Int8FewArgs& a, hipStream_t s) {
    const size_t sums = (size_t)NT * WAVES * 1024, held = FUSED ? 64 + (size_t)(a.n * a.pad) : 0, lds = held > sums ? held : sums;
    void (*const fn)(const Int8FewArgs) = &k_int8_few<T, NT, WAVES, FUSED>;
    allow_lds(reinterpret_cast<const void*>(fn), lds);
    hipLaunchKernelGGL(fn, dim3((unsigned)((a.rows + 15) / 16), (unsigned)((a.n + 16 * NT - 1) / (16 * NT))), dim3(64 * WAVES), lds, s, a);
}

// Where there are fewer workgroups than compute units, with fewer tokens or more wavefronts to each.
void launch_int8_few(int dtype, const Int8FewArgs& a, hipStream_t s) {
    const int64_t blocks = (a.rows + 15) / 16;
    if (!a.Q) BY_TYPE(dtype, T, (launch_few<T, 1, 8, true>(a, s)));
    else if (a.n > 32 && blocks * ((a.n + 63) / 64) >= 256) BY_TYPE(dtype, T, (launch_few<T, 4, 8, false>(a, s)));
    else if (a.n > 16 && blocks * ((a.n + 31) / 32) >= 256) BY_TYPE(dtype, T, (launch_few<T, 2, 8, false>(a, s)));
    else BY_TYPE(dtype, T, (launch_few<T, 1, 16, false>(a, s)));
}

// The tile_at-th 64 x 64 tile of W8's columns, as numbers of T, which holds integers of eight bits.
template <typename T>
__device__ __forceinline__ void integer_columns(const Int8SplitArgs& a, int64_t tile_at, uint32_t* lds) {
    const int64_t tiles_c = (a.cols + 63) / 64, tr = tile_at / tiles_c, r0 = tr * 64, c0 = (tile_at - tr * tiles_c) * 64;
    const int64_t r = r0 + (threadIdx.x >> 3) * 2, c = c0 + (threadIdx.x & 7) * 8;
    T v[2][8];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const bool there = r + b < a.rows && c < a.cols;
        const u32x2 q = *reinterpret_cast<const u32x2*>(a.W8 + (there ? (r + b) * a.ldw + c : 0));
#pragma unroll
        for (int e = 0; e < 8; ++e) v[b][e] = there ? (T)(float)(int8_t)(q[e >> 2] >> (e & 3) * 8) : (T)0.f;
    }
    const TransposeTile<T> tile{lds};
    tile.put(v[0], v[1]);
    __syncthreads();
    tile.emit(static_cast<T*>(a.B) + c0 * a.pad + r0, a.cols - c0, a.pad, a.pad - r0);
}

// dX of float32: x = dY scale is the sum of three numbers of bfloat16, its upper, middle and lower eight bits (cut off, so that no part becomes infinite;
// below 2^-110 the lowest may be lost), and integers of eight bits are numbers of bfloat16.  The float32 product is thus one of bfloat16 with three times the rows, exact but
// for its float32 sums, three of which make a result.  1001 x 1000 x 512: 22 us; by float32 matrix instructions, a ninth as many a second, 26.7.
__global__ __launch_bounds__(256) void k_int8_split(const Int8SplitArgs a) {
    __shared__ __align__(16) uint32_t lds[TransposeTile<bf16>::WORDS];
    if (blockIdx.x < a.splitting) {
        const int64_t per_row = a.pad / 8, pieces = a.n * per_row;
        for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < pieces; at += (int64_t)a.splitting * 256) {
            const int64_t t = pieces >> 31 ? at / per_row : (unsigned)at / (unsigned)per_row, r = (at - t * per_row) * 8;
            float x[8];
            float by[8];
            eight_floats(x, static_cast<const float*>(a.dY) + t * a.ldy, r, a.rows);
            eight_floats(by, a.scale, r, a.rows);
            u32x4 part[3];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] *= by[e];
                const bool finite = size_of(x[e]) < 0x7f800000;
#pragma unroll
                for (int i = 0; i < 3; ++i) {
                    uint32_t bits = __builtin_bit_cast(uint32_t, x[e]);
                    if (!finite && (bits & 0x7fffff)) bits |= 0x10000;  // a NaN stays one
                    if (!finite && i > 0) bits = 0;                     // .. and is one part
                    const uint32_t high = bits >> 16;
                    part[i][e / 2] = e & 1 ? part[i][e / 2] | high << 16 : high;
                    x[e] -= __builtin_bit_cast(float, bits & 0xffff0000);
                }
            }
#pragma unroll
            for (int i = 0; i < 3; ++i) *reinterpret_cast<u32x4*>(static_cast<bf16*>(a.A) + (i * a.n + t) * a.pad + r) = part[i];
        }
        return;
    }
    integer_columns<bf16>(a, blockIdx.x - a.splitting, lds);
}

void launch_int8_split(const Int8SplitArgs& args, bool dY, hipStream_t s) {
    Int8SplitArgs a = args;
    const int64_t groups = (a.n * (a.pad / 8) + 255) / 256, tiles = ((a.cols + 63) / 64) * ((a.pad + 63) / 64);
    a.splitting = dY ? (unsigned)(groups < 4096 ? groups : 4096) : 0u;
    hipLaunchKernelGGL(k_int8_split, dim3(a.splitting + (unsigned)tiles), dim3(256), 0, s, a);
}

// dX of float16: x = dY scale times a power of two 2^f of its token's, with which the token's largest is 2^14 to 2^15, rounded to float16, and integers as numbers of
// float16; the product's epilogue (or its join) multiplies by 2^-f.  Scale W8 in float16 would be none at all for layers of small weights, and infinite beyond 65504.
// Rounded by half a step, so are x down to 2^-28 of the token's largest; smaller ones by 2^-39 of it.  A workgroup to a token, as in k_int8_rows.
// f <= 126, so that 2^-f is a normal number: of smaller tokens the results are zero.
// 2048 x 4096 x 4096: 81 us in all, 1001 x 1000 x 512 13.7 (with dY as it is and scale W8 78; two parts of bfloat16 instead of one of float16
// 142 and 17.7).
__global__ __launch_bounds__(256) void k_int8_half(const Int8SplitArgs a) {
    constexpr int HELD = 2;
    __shared__ __align__(16) uint32_t lds[TransposeTile<f16>::WORDS];
    if (blockIdx.x >= a.splitting) {
        integer_columns<f16>(a, blockIdx.x - a.splitting, lds);
        return;
    }
    const int64_t t = blockIdx.x;
    const f16* row = static_cast<const f16*>(a.dY) + t * a.ldy;
    uint32_t top = 0;  // bits of the largest finite size
    auto ask = [&](float* x, int64_t r) {
        float by[8];
        eight_floats(x, row, r, a.rows);
        eight_floats(by, a.scale, r, a.rows);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= by[e];
    };
    auto look = [&](const float* x) {
#pragma unroll
        for (int e = 0; e < 8; ++e) top = size_of(x[e]) < 0x7f800000 ? max(top, size_of(x[e])) : top;
    };
    float x[HELD][8];
#pragma unroll
    for (int h = 0; h < HELD; ++h) ask(x[h], (h * 256 + threadIdx.x) * 8);
#pragma unroll
    for (int h = 0; h < HELD; ++h) look(x[h]);
    for (int64_t r = (HELD * 256 + threadIdx.x) * 8; r < a.rows; r += 2048) {
        float y[8];
        ask(y, r);
        look(y);
    }
    top = larger_of_wave(top);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = top;
    __syncthreads();
    top = max(max(lds[0], lds[1]), max(lds[2], lds[3]));
    const int f = min(127 + 14 - (int)(top >> 23), 126);
    if (threadIdx.x == 0) a.by[t] = ldexpf(1.f, -f);
    f16* out = static_cast<f16*>(a.A) + t * a.pad;
    auto put = [&](const float* v, int64_t r) {
        struct alignas(16) Eight { f16 v[8]; } y;
#pragma unroll
        for (int e = 0; e < 8; ++e) y.v[e] = Elem<f16>::down(ldexpf(v[e], f));
        if (r < a.pad) *reinterpret_cast<Eight*>(out + r) = y;
    };
#pragma unroll
    for (int h = 0; h < HELD; ++h) put(x[h], (h * 256 + threadIdx.x) * 8);
    for (int64_t r = (HELD * 256 + threadIdx.x) * 8; r < a.pad; r += 2048) {
        float y[8];
        ask(y, r);
        put(y, r);
    }
}

void launch_int8_half(const Int8SplitArgs& args, bool dY, hipStream_t s) {
    Int8SplitArgs a = args;
    a.splitting = dY ? (unsigned)a.n : 0u;
    hipLaunchKernelGGL(k_int8_half, dim3(a.splitting + (unsigned)(((a.cols + 63) / 64) * ((a.pad + 63) / 64))), dim3(256), 0, s, a);
}

template <typename T>
__global__ __launch_bounds__(256) void k_join_int8(const int32_t* __restrict__ parts, int nz, int64_t M, int64_t N, const float* __restrict__ by_m,
                                                   const float* __restrict__ by_n, T* __restrict__ out, int64_t ldo) {
    const int64_t total = M * N;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < total; at += (int64_t)gridDim.x * 256) {
        int sum = parts[at];
        for (int z = 1; z < nz; ++z) sum += parts[z * total + at];
        const int64_t m = at / N, n = at - m * N;
        out[m * ldo + n] = Elem<T>::down(TokenScale(by_m[m]).result(sum, by_n[n]));
    }
}

void launch_join_int8(int dtype, const int32_t* parts, int nz, int64_t M, int64_t N, const float* by_m, const float* by_n, void* out, int64_t ldo,
                      hipStream_t s) {
    const int64_t g = (M * N + 255) / 256;
    BY_TYPE(dtype, T, hipLaunchKernelGGL(k_join_int8<T>, dim3((unsigned)(g > 8192 ? 8192 : g)), dim3(256), 0, s, parts, nz, M, N, by_m, by_n,
                                         static_cast<T*>(out), ldo));
}

}  // namespace idkm

// Launches of the kernels around the tile product.
#include "layers.h"

namespace idkm {

// dC[e] = the sum of bins[w][e], one wavefront to an e.
__global__ __launch_bounds__(64) void k_join_bins(const float* __restrict__ bins, int nwg, int kd, float* __restrict__ dC) {
    const int e = blockIdx.x;
    double sum = 0.0;
    for (int w = threadIdx.x; w < nwg; w += 64) sum += (double)bins[(size_t)w * kd + e];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if (threadIdx.x == 0) dC[e] = (float)sum;
}

__global__ __launch_bounds__(256) void k_fill_zero(float* out, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) out[i] = 0.f;
}

static unsigned grid_for(int64_t threads) {
    const int64_t g = (threads + 255) / 256;
    return (unsigned)(g < 1 ? 1 : g > 8192 ? 8192 : g);
}

static size_t codebook_lds(DenseArgs& a, int esize) {
    const size_t bytes = (size_t)a.k * a.d * esize;
    a.c_in_lds = bytes <= 32 * 1024;
    return a.c_in_lds ? bytes : 0;
}

#define BY_TYPE(dtype, T, ...)                     \
    do {                                           \
        if ((dtype) == 0) {                        \
            using T = float;                       \
            __VA_ARGS__;                           \
        } else if ((dtype) == 1) {                 \
            using T = f16;                         \
            __VA_ARGS__;                           \
        } else {                                   \
            using T = bf16;                        \
            __VA_ARGS__;                           \
        }                                          \
    } while (0)

void launch_dense_rows(int dtype, const DenseArgs& args, hipStream_t s) {
    DenseArgs a = args;
    BY_TYPE(dtype, T, {
        const size_t lds = codebook_lds(a, sizeof(T));
        hipLaunchKernelGGL(k_dense_rows<T>, dim3(grid_for(a.count * (a.pad / 8))), dim3(256), lds, s, a);
    });
}

void launch_dense_cols(int dtype, const DenseArgs& args, hipStream_t s) {
    DenseArgs a = args;
    const dim3 grid((unsigned)((a.count + 63) / 64), (unsigned)((a.pad + 63) / 64));
    BY_TYPE(dtype, T, {
        const size_t lds = codebook_lds(a, sizeof(T));
        hipLaunchKernelGGL(k_dense_cols<T>, grid, dim3(256), lds, s, a);
    });
}

void launch_pad_rows(int dtype, const void* in, int64_t ldi, int64_t M, int64_t N, void* out, int64_t pad, hipStream_t s) {
    BY_TYPE(dtype, T, hipLaunchKernelGGL(k_pad_rows<T>, dim3(grid_for(M * pad)), dim3(256), 0, s, static_cast<const T*>(in), ldi, M, N,
                                         static_cast<T*>(out), pad));
}

void launch_transpose(int dtype, const void* in, int64_t ldi, int64_t M, int64_t N, void* out, int64_t pad, hipStream_t s) {
    const dim3 grid((unsigned)((N + 63) / 64), (unsigned)((pad + 63) / 64));
    BY_TYPE(dtype, T, hipLaunchKernelGGL(k_transpose<T>, grid, dim3(256), 0, s, static_cast<const T*>(in), ldi, M, N, static_cast<T*>(out), pad));
}

void launch_join_parts(int dtype, const float* parts, int nz, int64_t M, int64_t N, void* out, int64_t ldo, hipStream_t s) {
    BY_TYPE(dtype, T, hipLaunchKernelGGL(k_join_parts<T>, dim3(grid_for(M * N)), dim3(256), 0, s, parts, nz, M, N, static_cast<T*>(out), ldo));
}

void launch_codes_bins(int dtype, const BinArgs& a, int grid, int waves, hipStream_t s) {
    const size_t lds = a.bins ? (size_t)waves * a.codes * 64 * sizeof(float) : 0;
    BY_TYPE(dtype, T, {
        (void)hipFuncSetAttribute(reinterpret_cast<const void*>(&k_codes_bins<T>), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
        hipLaunchKernelGGL(k_codes_bins<T>, dim3((unsigned)grid), dim3((unsigned)waves * 64), lds, s, a);
    });
}

void launch_join_bins(const float* bins, int nwg, int kd, float* dC, hipStream_t s) {
    hipLaunchKernelGGL(k_join_bins, dim3((unsigned)kd), dim3(64), 0, s, bins, nwg, kd, dC);
}

void launch_fill_zero(float* out, int64_t n, hipStream_t s) {
    hipLaunchKernelGGL(k_fill_zero, dim3(grid_for(n)), dim3(256), 0, s, out, n);
}

}  // namespace idkm

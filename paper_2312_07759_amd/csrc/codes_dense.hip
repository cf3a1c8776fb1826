// Launches of the kernels around the tile product.
#include <atomic>

#include "layers.h"

namespace idkm {

// dC[e] = the sum of bins[e][w], w < n, in float64: a workgroup to an e.  The workgroups behind them add up segments:
// dS[r, g] = the sum of the row's segments of the group, in order; listed: the segments' row i belongs to row listed[i], for *listed_count rows.
__global__ __launch_bounds__(256) void k_join_gradients(const float* __restrict__ bins, int64_t n, int kd, float* __restrict__ dC,
                                                        const float* __restrict__ segments, int per_row, int of_group, int groups, int64_t scales,
                                                        float* __restrict__ dS, const int32_t* __restrict__ listed,
                                                        const int32_t* __restrict__ listed_count) {
    if ((int)blockIdx.x >= kd) {
        if (listed) scales = (int64_t)*listed_count * groups;
        for (int64_t i = (int64_t)(blockIdx.x - kd) * 256 + threadIdx.x; i < scales; i += (int64_t)(gridDim.x - kd) * 256) {
            const int64_t r = i / groups;
            const int g = (int)(i - r * groups), last = min(per_row, (g + 1) * of_group);
            float sum = 0.f;
            for (int j = g * of_group; j < last; ++j) sum += segments[r * per_row + j];
            dS[listed ? (int64_t)listed[r] * groups + g : i] = sum;
        }
        return;
    }
    __shared__ double waves[4];
    const float* mine = bins + blockIdx.x * n;
    double sum = 0.0;
    for (int64_t w = threadIdx.x; w < n; w += 256) sum += (double)mine[w];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) dC[blockIdx.x] = (float)(waves[0] + waves[1] + waves[2] + waves[3]);
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

// Kernels with more than 64 KB of dynamic LDS have to be told once on every device; what has been told is kept, without a lock
// (two threads may tell it twice).
void allow_lds(const void* fn, size_t bytes) {
    if (bytes <= 64 * 1024) return;
    static std::atomic<uintptr_t> told[1024];
    int device = 0;
    (void)hipGetDevice(&device);
    const uintptr_t key = reinterpret_cast<uintptr_t>(fn) ^ (uintptr_t)(device + 1) << 56;
    std::atomic<uintptr_t>& slot = told[(key >> 4 ^ key >> 14 ^ key >> 56) & 1023];
    if (slot.load(std::memory_order_relaxed) == key) return;
    if (hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) == hipSuccess) slot.store(key, std::memory_order_relaxed);
}

static int64_t operand_tiles(const OperandArgs& a) {
    int64_t tiles = 0;
    for (int j = 0; j < a.jobs; ++j) tiles += a.job[j].tiles;
    return tiles;
}

// The kernels with lookups take these; a run's words (three at most) have to be there.
static bool fast_codes(const DenseArgs& a) { return a.bits <= 8 && (a.d == 1 || a.d == 2 || a.d == 4 || a.d == 8) && a.nwords >= 4; }

static bool launch_fast(int dtype, const DenseArgs& a, bool columns, hipStream_t s) {
    if (!fast_codes(a)) return false;
    const int at_once = codes_at_once(a.bits, a.d), IB = at_once * a.bits, W = at_once * a.d;
    const DenseFn fn = codes_dense_kernel(dtype, IB, W, columns, a.row_bits % 32 == 0);
    const size_t table = (size_t)128 << IB, tile = columns ? (dtype == 0 ? TransposeTile<float>::WORDS : TransposeTile<bf16>::WORDS) * 4 : 0;
    int64_t grid = columns ? ((a.count + 63) / 64) * ((a.pad + 63) / 64) : (a.count * (a.pad / 8) + 255) / 256;
    // as many workgroups as the compute units hold at once, each with one table
    const int64_t most = columns ? 768 : 1024;
    if (grid > most) grid = most;
    DenseArgs b = a;
    b.dense = (unsigned)grid;
    hipLaunchKernelGGL(fn, dim3((unsigned)(grid + operand_tiles(a.also))), dim3(256), table + tile, s, b);
    return true;
}

void launch_dense_rows(int dtype, const DenseArgs& args, hipStream_t s) {
    DenseArgs a = args;
    if (launch_fast(dtype, a, false, s)) return;
    BY_TYPE(dtype, T, {
        const size_t lds = codebook_lds(a, sizeof(T));
        hipLaunchKernelGGL(k_dense_rows<T>, dim3(grid_for(a.count * (a.pad / 8))), dim3(256), lds, s, a);
    });
}

void launch_dense_cols(int dtype, const DenseArgs& args, hipStream_t s, const OperandArgs& also) {
    DenseArgs a = args;
    // One launch for both: gradients of 512 tokens of 2048 x 2048 in bfloat16 57.5 us in two launches and 55, 500 of 1000 x 1000 in float32 57 and 54, as long where
    // either fills the device by itself (2048 tokens of 4096 x 4096).
    if (fast_codes(a)) {
        a.also = also;
        launch_fast(dtype, a, true, s);
        return;
    }
    launch_operands(dtype, also, s);
    const dim3 grid((unsigned)((a.count + 63) / 64), (unsigned)((a.pad + 63) / 64));
    BY_TYPE(dtype, T, {
        const size_t lds = codebook_lds(a, sizeof(T));
        hipLaunchKernelGGL(k_dense_cols<T>, grid, dim3(256), lds, s, a);
    });
}

void add_operand(OperandArgs* a, const void* in, int64_t ldi, int64_t M, int64_t N, void* out, int64_t pad, bool transposed, const uint8_t* E,
                 const float* scale) {
    Operand& o = a->job[a->jobs++];
    o = Operand{in, ldi, M, N, out, pad, transposed, 0, 0, E, scale};
    o.tiles_n = ((transposed ? N : pad) + 63) / 64;
    o.tiles = o.tiles_n * (((transposed ? pad : M) + 63) / 64);
}

void launch_operands(int dtype, const OperandArgs& a, hipStream_t s) {
    const int64_t tiles = operand_tiles(a);
    if (tiles > 0) BY_TYPE(dtype, T, hipLaunchKernelGGL(k_operands<T>, dim3((unsigned)tiles), dim3(256), 0, s, a));
}

void launch_join_parts(int dtype, const float* parts, int nz, int64_t M, int64_t N, void* out, int64_t ldo, hipStream_t s,
                       const float* by_m) {
    BY_TYPE(dtype, T, hipLaunchKernelGGL(k_join_parts<T>, dim3(grid_for(M * N)), dim3(256), 0, s, parts, nz, M, N, static_cast<T*>(out), ldo, by_m));
}

void launch_codes_bins(int dtype, const BinArgs& args, int grid, int waves, hipStream_t s) {
    BinArgs a = args;
    const size_t book = (size_t)a.k * a.d * (dtype == 0 ? 4 : 2);
    a.c_in_lds = a.dS && book <= 16 * 1024;
    const size_t lds = (a.bins ? (size_t)waves * a.codes * 256 : 0) + (a.c_in_lds ? book : 0);
    BY_TYPE(dtype, T, {
        void (*const fn)(const BinArgs) = a.listed ? &k_codes_bins<T, true> : &k_codes_bins<T, false>;
        allow_lds(reinterpret_cast<const void*>(fn), lds);
        hipLaunchKernelGGL(fn, dim3((unsigned)grid), dim3((unsigned)waves * 64), lds, s, a);
    });
}

// Lanes that have the same bins in k_codes_bins_wide: 16 KB a wavefront.
int bins_shared_by(int k) { return k <= 64 ? 1 : k <= 128 ? 2 : 4; }

template <typename T, int SHARE, bool LISTED>
static void (*wide_for(int d))(const BinArgs) {
    return d == 1 ? &k_codes_bins_wide<T, 1, SHARE, LISTED> : d == 2 ? &k_codes_bins_wide<T, 2, SHARE, LISTED>
           : d == 4 ? &k_codes_bins_wide<T, 4, SHARE, LISTED> : &k_codes_bins_wide<T, 8, SHARE, LISTED>;
}

template <typename T, bool LISTED>
static void launch_bins_runs(const BinArgs& a, bool wide, int grid, int waves, hipStream_t s) {
    void (*const narrow_fn)(const BinArgs) = a.d == 1 ? &k_codes_bins_runs<T, 1, LISTED> : a.d == 2 ? &k_codes_bins_runs<T, 2, LISTED>
                                             : a.d == 4 ? &k_codes_bins_runs<T, 4, LISTED> : &k_codes_bins_runs<T, 8, LISTED>;
    const int share = wide ? bins_shared_by(a.k) : 1;
    void (*const wide_fn)(const BinArgs) = share == 1 ? wide_for<T, 1, LISTED>(a.d) : share == 2 ? wide_for<T, 2, LISTED>(a.d) : wide_for<T, 4, LISTED>(a.d);
    void (*const fn)(const BinArgs) = wide ? wide_fn : narrow_fn;
    const size_t lds = wide ? (a.bins ? (size_t)waves * (64 / share) * a.k * 4 : 0) : ((a.bins ? (size_t)waves * 64 : 0) + 1) * a.k * a.d * 4;
    allow_lds(reinterpret_cast<const void*>(fn), lds);
    hipLaunchKernelGGL(fn, dim3((unsigned)grid), dim3((unsigned)waves * 64), lds, s, a);
}

void launch_codes_bins_runs(int dtype, const BinArgs& a, bool wide, int grid, int waves, hipStream_t s) {
    if (a.listed) BY_TYPE(dtype, T, launch_bins_runs<T, true>(a, wide, grid, waves, s));
    else BY_TYPE(dtype, T, launch_bins_runs<T, false>(a, wide, grid, waves, s));
}

void launch_join_gradients(const float* bins, int64_t n, int kd, float* dC, const float* segments, int64_t rows, int64_t cols, int group,
                           int groups, float* dS, hipStream_t s, const int32_t* listed, const int32_t* listed_count) {
    const int per_row = (int)((cols + 31) / 32), of_group = groups > 1 ? group / 32 : per_row;
    if (!dC) kd = 0;
    const unsigned grid = (unsigned)kd + (segments ? grid_for(rows * groups) : 0u);
    if (grid > 0)
        hipLaunchKernelGGL(k_join_gradients, dim3(grid), dim3(256), 0, s, bins, n, kd, dC, segments, per_row, of_group, groups, rows * groups, dS, listed,
                           listed_count);
}

void launch_fill_zero(float* out, int64_t n, hipStream_t s) {
    hipLaunchKernelGGL(k_fill_zero, dim3(grid_for(n)), dim3(256), 0, s, out, n);
}

}  // namespace idkm

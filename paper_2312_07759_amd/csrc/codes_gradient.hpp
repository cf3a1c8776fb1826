// Gradients of a product with a coded layer in its group scales and its codebook, from P[n, c] = sum_t dY[t, n] X[t, c]:
//   dS[n, g] = sum over the group's columns of P[n, c] C[code, x]        (x = c mod d)
//   dC[j, x] = sum over all (n, c) with that codeword and component of S[n, g] P[n, c]
// P is read once (float32, in `parts` parts that add up).  A lane takes columns with the same component x each time and keeps
// bins of its own for the codewords in LDS ([codeword][lane], a bank to a lane), so no two lanes ever add to the same word and
// the order of every sum is fixed.  A workgroup's bins go to `bins` [workgroup][k d]; k_join_bins adds them up in float64.
#pragma once
#include "codes_dense.hpp"

namespace idkm {

struct BinArgs {
    const uint32_t* words;
    int64_t nwords;
    int64_t rows, cols;
    const void* C;
    int k, d, bits;
    const float* S;
    int group, groups;  // one group a row if there are no scales
    const float* P;     // [parts][count][ldp], rows [first, first + count) of the layer
    int parts;
    int64_t ldp, first, count;
    float* dS;  // [rows, groups] or null
    float* bins;  // [gridDim.x][k d] or null
    int code0, codes;  // codewords binned by this launch
    int lanes;  // of a wavefront that take part: a multiple of d, or 64 if d >= 64
};

template <typename T>
__global__ __launch_bounds__(256) void k_codes_bins(const BinArgs a) {
    extern __shared__ float bin[];  // [wave][codes][64]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nw = blockDim.x >> 6;
    float* mine = bin + (size_t)wave * a.codes * 64;
    if (a.bins)
        for (int j = 0; j < a.codes; ++j) mine[j * 64 + lane] = 0.f;
    const T* C = static_cast<const T*>(a.C);
    const int64_t per_row = a.cols / a.d;
    const int64_t units = a.count * a.groups;  // a wavefront takes a group of a row at a time
    const int64_t plane = a.count * a.ldp;
    for (int64_t u = (int64_t)blockIdx.x * nw + wave; u < units; u += (int64_t)gridDim.x * nw) {
        const int64_t rr = u / a.groups, r = a.first + rr;
        const int g = (int)(u - rr * a.groups);
        const int64_t c0 = (int64_t)g * a.group, c1 = min(a.cols, c0 + a.group);
        const float s = a.S ? a.S[r * a.groups + g] : 1.f;
        float sum = 0.f;
        for (int64_t c = c0 + lane; c < c1; c += a.lanes) {
            if (lane >= a.lanes) break;
            const int64_t j = c / a.d;
            const int x = (int)(c - j * a.d);
            const uint32_t code = code_at(a.words, a.nwords, r * per_row + j, a.bits);
            float p = a.P[rr * a.ldp + c];
            for (int z = 1; z < a.parts; ++z) p += a.P[z * plane + rr * a.ldp + c];
            if (a.dS) sum += p * Elem<T>::up(weight_of<T>(code, x, C, a.k, a.d, 1.f, false));
            const int b = (int)code - a.code0;
            if (a.bins && b >= 0 && b < a.codes) mine[b * 64 + lane] += s * p;
        }
        if (a.dS) {
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
            if (lane == 0) a.dS[r * a.groups + g] = sum;
        }
    }
    if (!a.bins) return;
    __syncthreads();
    // component x of codeword j: the lanes x, x + d, ..
    const int d = a.d;
    for (int e = threadIdx.x; e < a.codes * d; e += blockDim.x) {
        const int j = e / d, x = e - j * d;
        if (a.code0 + j >= a.k) continue;
        double sum = 0.0;
        for (int w = 0; w < nw; ++w)
            for (int l = x; l < a.lanes; l += d) sum += (double)bin[((size_t)w * a.codes + j) * 64 + l];
        a.bins[(size_t)blockIdx.x * (a.k * d) + (a.code0 + j) * d + x] = (float)sum;
    }
}

}  // namespace idkm

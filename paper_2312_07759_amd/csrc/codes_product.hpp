// Y[t, n] = sum_c X[t, c] w[n, c] for few tokens, straight from the packed codes: w[n, c] = S[n, c / group] C[code, c % d].
//
// Bound by reading the codes once.  They go from memory into registers in the layout in which the matrix instruction takes
// them (lane l: layer row l % 16, a run of L consecutive weights for each quarter l / 16), so the codes need no LDS and the
// multiplications no vector instructions; up to 16 NT tokens share one decoding.  A code becomes a weight by reading a table
// in LDS.  Several codes of few bits are looked up at once: the table is indexed by up to 8 bits of the stream and holds their
// 2 .. 8 weights, which costs one LDS read and two vector instructions for all of them.
// The table holds the codewords in X's type, as they are given; a group's scale multiplies the float32 sum over its part
// of the row, so nothing is rounded but the result.
// The wavefronts of a workgroup share 16 rows of the layer and split the sum; their partial sums meet in LDS, in order.
#pragma once
#include <type_traits>

#include "elem.hpp"

namespace idkm {

struct ProductArgs {
    const uint32_t* words;
    int64_t nwords;
    int64_t rows, cols;
    const void* C;  // T [k, d]
    int k;
    const float* S;  // [rows, groups] or null
    int group, groups;
    const void* X;  // T [n, ldx]
    int64_t ldx;
    void* Y;  // T [n, ldy]
    int64_t ldy;
    int64_t n;
};

// Codes looked up at once: c codes of B bits and D weights each, c a power of two, at most 8 bits and 8 weights together.
constexpr int codes_at_once(int B, int D) {
    int c = 1;
    while (2 * c * B <= 8 && 2 * c * D <= 8) c *= 2;
    return c;
}

// The run of code bits that begins `bit` bits into the stream, NB of them, in (NB + 31) / 32 words.  Words behind the
// stream's last are read as that one; what the caller does not use may lie there.  ALIGNED: runs begin with a word.
template <int NB>
struct CodeRun {
    static constexpr int NWORDS = (NB + 31) / 32;
    uint32_t w[NWORDS];
    template <bool ALIGNED>
    __device__ __forceinline__ void load(const uint32_t* words, int64_t nwords, int64_t bit) {
        constexpr int RAW = ALIGNED ? NWORDS : (NB + 31 + 31) / 32;  // words that NB bits may touch
        const int64_t at = bit >> 5;
        uint32_t raw[RAW + 1];
        if (at + RAW <= nwords) {
            __builtin_memcpy(raw, words + at, RAW * 4);
        } else {
#pragma unroll
            for (int i = 0; i < RAW; ++i) raw[i] = words[min(at + i, nwords - 1)];
        }
        raw[RAW] = 0;
        const int sh = (int)(bit & 31);
#pragma unroll
        for (int i = 0; i < NWORDS; ++i) w[i] = ALIGNED ? raw[i] : __builtin_amdgcn_alignbit(raw[i + 1], raw[i], sh);
    }
    // bits [at, at + n), n <= 8, at known to the compiler
    __device__ __forceinline__ uint32_t bits(int at, int n) const {
        const int i = at >> 5, sh = at & 31;
        if (sh + n <= 32) return (w[i] >> sh) & ((1u << n) - 1u);
        return __builtin_amdgcn_alignbit(w[i + 1], w[i], sh) & ((1u << n) - 1u);
    }
};

// B bits a code, D weights a codeword, L consecutive weights of a row to a lane at a time (a chunk: 4 L), 16 NT tokens.
template <typename T, int B, int D, int L, int NT, bool ALIGNED>
__global__ __launch_bounds__(512) void k_codes_product(const ProductArgs a) {
    constexpr int CO = codes_at_once(B, D), IB = CO * B, W = CO * D;  // a table entry: CO codes, IB bits, W weights
    constexpr int NB = L / D * B;
    constexpr int FR = 8 / Elem<T>::PER16;  // 16-byte fragments in 8 weights
    constexpr int SUB = L / 8;
    extern __shared__ __align__(16) unsigned char lds[];
    T* table = reinterpret_cast<T*>(lds);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nw = blockDim.x >> 6;
    const int li = lane & 15, q = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    const int64_t row = min(n0 + li, a.rows - 1);
    const int64_t t0 = (int64_t)blockIdx.y * (16 * NT);

    const int chunks = (int)((a.cols + 4 * L - 1) / (4 * L));
    const int each = (chunks + nw - 1) / nw;
    const int first = min(chunks, wave * each), last = min(chunks, first + each);
    const int64_t row_bit = row * (a.cols / D * B);

    // the table
    {
        const T* C = static_cast<const T*>(a.C);
        for (int e = threadIdx.x; e < (1 << IB) * W; e += blockDim.x) {
            const int entry = e / W, x = e % W;
            const int code = (entry >> (x / D * B)) & ((1 << B) - 1);
            table[e] = code < a.k ? C[code * D + x % D] : Elem<T>::nan();
        }
    }
    __syncthreads();

    floatx4 acc[NT], part[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[j] = part[j] = floatx4{0.f, 0.f, 0.f, 0.f};
    int g_now = first * (4 * L) / max(a.group, 1);
    // the scales of the four rows that this lane holds sums of
    auto close_group = [&](int g) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t n = min(n0 + q * 4 + r, a.rows - 1);
            const float s = a.S[n * a.groups + g];
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                acc[j][r] += s * part[j][r];
                part[j][r] = 0.f;
            }
        }
    };
    // tokens behind the last one are computed from its activations and not stored
    const T* X[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) X[j] = static_cast<const T*>(a.X) + min(t0 + j * 16 + li, a.n - 1) * a.ldx;
    auto chunk = [&](int ch, const CodeRun<NB>& run, auto whole_) {
        constexpr bool whole = decltype(whole_)::value;  // all of the chunk's weights belong to the row
        const int64_t c0 = (int64_t)ch * (4 * L) + q * L;
        if (a.S) {  // a chunk lies in one group
            const int g = (int)((int64_t)ch * (4 * L) / a.group);
            if (g != g_now) {
                close_group(g_now);
                g_now = g;
            }
        }
        u32x4 xf[SUB][NT][FR];
#pragma unroll
        for (int s = 0; s < SUB; ++s)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const T* x = X[j] + c0 + s * 8;
                if constexpr (whole) {
#pragma unroll
                    for (int f = 0; f < FR; ++f) xf[s][j][f] = reinterpret_cast<const u32x4_any*>(x)[f];
                } else {
                    struct alignas(16) Eight { T v[8]; } y;
#pragma unroll
                    for (int i = 0; i < 8; ++i) y.v[i] = c0 + s * 8 + i < a.cols ? x[i] : (T)0.f;
                    __builtin_memcpy(xf[s][j], &y, sizeof(y));
                }
            }
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
            struct alignas(16) Eight { T v[8]; } w;
#pragma unroll
            for (int e = 0; e < 8 / W; ++e) {
                const uint32_t idx = run.bits((s * 8 / W + e) * IB, IB);
                struct alignas(W * sizeof(T) > 16 ? 16 : W * sizeof(T)) Entry { T v[W]; };
                const Entry x = *reinterpret_cast<const Entry*>(table + idx * W);
#pragma unroll
                for (int i = 0; i < W; ++i) w.v[e * W + i] = x.v[i];
            }
            if constexpr (!whole) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c0 + s * 8 + i >= a.cols) w.v[i] = (T)0.f;
            }
            u32x4 wf[FR];
            __builtin_memcpy(wf, &w, sizeof(wf));
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int f = 0; f < FR; ++f) mma16<T>(part[j], wf[f], xf[s][j][f]);
        }
    };
    auto load = [&](int ch, CodeRun<NB>& run) {
        run.template load<ALIGNED>(a.words, a.nwords, row_bit + ((int64_t)ch * (4 * L) + q * L) / D * B);
    };
    const int full = (int)min((int64_t)last, a.cols / (4 * L));  // chunks before this one are whole
    constexpr int U = NT > 1 ? 2 : 4;  // chunks whose codes are asked for together
    int ch = first;
    for (; ch + U <= full; ch += U) {
        CodeRun<NB> run[U];
#pragma unroll
        for (int u = 0; u < U; ++u) load(ch + u, run[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) chunk(ch + u, run[u], std::true_type());
    }
    for (; ch < last; ++ch) {
        CodeRun<NB> run;
        load(ch, run);
        if (ch < full)
            chunk(ch, run, std::true_type());
        else
            chunk(ch, run, std::false_type());
    }
    if (a.S) {
        if (first < last) close_group(g_now);
    } else {
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[j] = part[j];
    }
    // the wavefronts' sums: [wave][token of 16 NT][row of 16]
    __syncthreads();
    float* red = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int j = 0; j < NT; ++j) *reinterpret_cast<floatx4*>(red + ((wave * NT + j) * 16 + li) * 16 + q * 4) = acc[j];
    __syncthreads();
    for (int e = threadIdx.x; e < 256 * NT; e += blockDim.x) {
        float sum = 0.f;
        for (int w = 0; w < nw; ++w) sum += red[w * 256 * NT + e];
        const int64_t t = t0 + (e >> 4), n = n0 + (e & 15);
        if (t < a.n && n < a.rows) static_cast<T*>(a.Y)[t * a.ldy + n] = Elem<T>::down(sum);
    }
}

}  // namespace idkm

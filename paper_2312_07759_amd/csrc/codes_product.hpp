// Y[t, n] = sum_c X[t, c] w[n, c] for few tokens, straight from the packed codes: w[n, c] = S[n, c / group] C[code, c % d].
//
// Codes go from memory into registers in the layout in which the matrix instruction takes them (lane l: layer row l % 16, a
// run of L consecutive weights for each quarter l / 16), so they need no LDS and the multiplications no vector instructions.
// A code becomes a weight by reading a table in LDS.  Several codes of few bits are looked up at once: the table is indexed by
// up to 8 bits of the stream and holds their up to 8 weights, which costs one LDS read and two vector instructions for all.
// The table holds the codewords in X's type, as they are given; a group's scale multiplies the float32 sum over its part
// of the row, so nothing is rounded but the result.
// The wavefronts of a workgroup share 16 rows of the layer and split the sum; their partial sums meet in LDS, in order.
// Bound by the latency of one batch of loads and the issue of few wavefronts, not yet by memory: one token, 4096 x 4096, 4 bits, bfloat16
// 6.2 us (8.9 MB; a large copy moves them in 1.7), 1000 x 512, k = 4, d = 1, float32 4.4 to 4.6 us.
#pragma once
#include <type_traits>

#include "elem.hpp"

namespace idkm {

struct ProductArgs {
    const uint32_t* words;
    int64_t nwords;
    int64_t rows, cols;
    const void* C;  // T [k, d]
    int k, B, D;        // B bits a code, D weights a codeword
    int64_t row_bits;   // of the stream
    const float* S;     // [rows, groups], or groups = 0
    int groups;
    unsigned group_magic;  // ceil(2^31 / chunks of a group): its high product with twice a chunk is the chunk's group
    const void* X;  // T [n, ldx]
    int64_t ldx;
    void* Y;  // T [n, ldy]
    int64_t ldy;
    int64_t n;
    // more than 16 tokens
    float* sums;     // [gridDim.z][n][rows] where several workgroups share a row's sum
};

// Codes looked up at once: c codes of B bits and D weights each, c a power of two, at most 8 bits and 8 weights together.
constexpr int codes_at_once(int B, int D) {
    int c = 1;
    while (2 * c * B <= 8 && 2 * c * D <= 8) c *= 2;
    return c;
}

// The table in LDS: entry e holds the W weights of the codes in the IB bits e, the first code in the low bits.  It has 128 bytes,
// all 32 banks, filled with copies; a lane reads the copy in its own banks, so that no lane waits for another (with one copy, 32
// lanes at random places of 32 banks took 3.5 turns instead of one, and the lookups bounded the product of a single token).
// A thread's first entry is asked for by the constructor, so that the wait for it can come later.
template <typename T, int IB, int W>
struct Table {
    static constexpr int ENTRIES = 1 << IB, BYTES = 128 * ENTRIES;
    static constexpr int WIDTH = W * (int)sizeof(T), STRIDE = WIDTH < 4 ? 4 : WIDTH, COPIES = 128 / STRIDE;
    struct alignas(WIDTH > 16 ? 16 : WIDTH) Entry { T v[W]; };
    T first[W];
    unsigned none;  // bit i: first[i] belongs to a code that is none
    static __device__ __forceinline__ unsigned ask(T* v, unsigned e, const void* codebook, int k, int B, int D) {
        const T* C = static_cast<const T*>(codebook);
        unsigned none = 0;
        int code = 0, part = D;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if (part == D) {
                part = 0;
                code = (int)(e & ((1u << B) - 1u));
                e >>= B;
            }
            v[i] = C[min(code, k - 1) * D + part];
            none |= code < k ? 0u : 1u << i;
            ++part;
        }
        return none;
    }
    // 16-byte pieces h, h + step, .. of entry e, from a place on that depends on the lane: neighbours write to different banks
    static __device__ __forceinline__ void put(unsigned char* lds, unsigned e, const T* v, unsigned none, int h, int step) {
        constexpr int N = WIDTH > 16 ? 2 : 1;  // different pieces
        u32x4 piece[N];
        T x[N * 16 / sizeof(T)];
#pragma unroll
        for (int i = 0; i < N * 16 / (int)sizeof(T); ++i) {
            const int w = i % W;
            x[i] = none >> w & 1 ? Elem<T>::nan() : v[w];
        }
        __builtin_memcpy(piece, x, sizeof(piece));
        for (int j = h; j < 8; j += step) {
            const int at = (j + threadIdx.x) & 7;
            *reinterpret_cast<u32x4*>(lds + e * 128 + at * 16) = N > 1 && (at & 1) ? piece[N - 1] : piece[0];
        }
    }
    __device__ __forceinline__ Table(const void* codebook, int k, int B, int D) {
        none = ask(first, threadIdx.x & (ENTRIES - 1), codebook, k, B, D);
    }
    __device__ __forceinline__ void build(unsigned char* lds, const void* codebook, int k, int B, int D) const {
        const unsigned team = blockDim.x >> IB;  // threads to an entry
        if (team >= 1) {
            const int step = team >= 8 ? 8 : team >= 4 ? 4 : team >= 2 ? 2 : 1;
            if ((int)(threadIdx.x >> IB) < step) put(lds, threadIdx.x & (ENTRIES - 1), first, none, (int)(threadIdx.x >> IB), step);
        } else {
            put(lds, threadIdx.x, first, none, 0, 1);
            for (unsigned e = threadIdx.x + blockDim.x; e < ENTRIES; e += blockDim.x) {
                T v[W];
                const unsigned n = ask(v, e, codebook, k, B, D);
                put(lds, e, v, n, 0, 1);
            }
        }
    }
    // where this lane's copies begin
    static __device__ __forceinline__ const unsigned char* own(const unsigned char* lds) {
        return lds + (threadIdx.x % COPIES) * STRIDE;
    }
};

// The run of code bits that begins `bit` bits into the stream, NB of them, in (NB + 31) / 32 words.  Words behind the
// stream's last are read as that one; what the caller does not use may lie there.  ALIGNED: runs begin with a word.
// NEAR_END false: the caller knows that SPAN words from the run's first one on belong to the stream.
template <int NB>
struct CodeRun {
    static constexpr int NWORDS = (NB + 31) / 32;
    static constexpr int SPAN = (NB + 31 + 31) / 32;  // words that NB bits may touch
    uint32_t w[NWORDS];
    template <bool ALIGNED, bool NEAR_END>
    __device__ __forceinline__ void load(const uint32_t* words, int64_t nwords, int64_t bit) {
        constexpr int RAW = ALIGNED ? NWORDS : SPAN;
        const int64_t at = bit >> 5;
        uint32_t raw[RAW + 1];
        if (!NEAR_END || at + RAW <= nwords) {
            constexpr int Q = RAW / 4 * 4;
#pragma unroll
            for (int i = 0; i < Q; i += 4) {
                const u32x4 v = *reinterpret_cast<const u32x4_word*>(words + at + i);
#pragma unroll
                for (int e = 0; e < 4; ++e) raw[i + e] = v[e];
            }
            if constexpr (RAW - Q >= 2) {
                const u32x2 v = *reinterpret_cast<const u32x2_word*>(words + at + Q);
                raw[Q] = v[0];
                raw[Q + 1] = v[1];
            }
            if constexpr (RAW % 2 == 1) raw[RAW - 1] = words[at + RAW - 1];
        } else {
#pragma unroll
            for (int i = 0; i < RAW; ++i) raw[i] = words[min(at + i, nwords - 1)];
        }
        raw[RAW] = 0;
        const int sh = (int)(bit & 31);
#pragma unroll
        for (int i = 0; i < NWORDS; ++i) w[i] = ALIGNED ? raw[i] : __builtin_amdgcn_alignbit(raw[i + 1], raw[i], sh);
    }
    // The same without a branch, for a run that lies in the stream as a whole (which has at least SPAN words): near its end the
    // words are taken from one further ahead.  `bit` counts from `words` on; no window begins behind word `limit`, which is >= 0.
    template <bool ALIGNED>
    __device__ __forceinline__ void load_inside(const uint32_t* words, int limit, unsigned bit) {
        constexpr int RAW = ALIGNED ? NWORDS : SPAN;
        const int at = (int)(bit >> 5);
        const unsigned from = ALIGNED ? (unsigned)at : (unsigned)min(at, limit);
        uint32_t raw[RAW + 2];
        constexpr int Q = RAW / 4 * 4;
#pragma unroll
        for (int i = 0; i < Q; i += 4) {
            const u32x4 v = *reinterpret_cast<const u32x4_word*>(words + from + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) raw[i + e] = v[e];
        }
        if constexpr (RAW - Q >= 2) {
            const u32x2 v = *reinterpret_cast<const u32x2_word*>(words + from + Q);
            raw[Q] = v[0];
            raw[Q + 1] = v[1];
        }
        if constexpr (RAW % 2 == 1) raw[RAW - 1] = words[from + RAW - 1];
        raw[RAW] = raw[RAW + 1] = 0;
        const int sh = (int)(bit & 31);
        const bool ahead = SPAN > NWORDS && at != (int)from;
#pragma unroll
        for (int i = 0; i < NWORDS; ++i) {
            if constexpr (ALIGNED) {
                w[i] = raw[i];
            } else {
                const uint32_t lo = ahead ? raw[i + 1] : raw[i], hi = ahead ? raw[i + 2] : raw[i + 1];
                w[i] = __builtin_amdgcn_alignbit(hi, lo, sh);
            }
        }
    }
    // bits [at, at + n), n <= 8, at known to the compiler
    __device__ __forceinline__ uint32_t bits(int at, int n) const {
        const int i = at >> 5, sh = at & 31;
        if (sh + n <= 32) return (w[i] >> sh) & ((1u << n) - 1u);
        return __builtin_amdgcn_alignbit(w[i + 1], w[i], sh) & ((1u << n) - 1u);
    }
};

// Eight weights from the run's looked-up codes s * 8 / W ...
template <typename T, int IB, int W, int NB>
__device__ __forceinline__ void eight_weights(u32x4* out, const CodeRun<NB>& run, int s, const unsigned char* own) {
    struct alignas(16) Eight { T v[8]; } w;
#pragma unroll
    for (int e = 0; e < 8 / W; ++e) {
        const uint32_t idx = run.bits((s * 8 / W + e) * IB, IB);
        const auto x = *reinterpret_cast<const typename Table<T, IB, W>::Entry*>(own + idx * 128);
#pragma unroll
        for (int i = 0; i < W; ++i) w.v[e * W + i] = x.v[i];
    }
    __builtin_memcpy(out, &w, sizeof(w));
}

// Eight elements of a row from column c on, zero behind its end.
template <typename T>
__device__ __forceinline__ void eight_of_row(u32x4* out, const T* row, int64_t c, int64_t cols, bool whole) {
    if (whole) {
#pragma unroll
        for (int f = 0; f < 8 / Elem<T>::PER16; ++f) out[f] = reinterpret_cast<const u32x4_any*>(row + c)[f];
    } else {
        struct alignas(16) Eight { T v[8]; } y;
#pragma unroll
        for (int i = 0; i < 8; ++i) y.v[i] = c + i < cols ? row[c + i] : (T)0.f;
        __builtin_memcpy(out, &y, sizeof(y));
    }
}

// Zeros in the place of weights behind column cols: what a row's last run holds there belongs to the next row.
template <typename T>
__device__ __forceinline__ void cut_weights(u32x4* w, int64_t c, int64_t cols) {
    struct alignas(16) Eight { T v[8]; } y;
    __builtin_memcpy(&y, w, sizeof(y));
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c + i >= cols) y.v[i] = (T)0.f;
    __builtin_memcpy(w, &y, sizeof(y));
}

// Up to 16 tokens.  IB bits looked up at once give W weights; L consecutive weights of a row to a lane at a time: four runs make
// a chunk of 4 L columns, which lies in one group.  Everything that a batch of chunks needs (codes, activations, scales) is
// asked for before the first of it is used, the first batch before the table is built.
// APART, for up to 4 tokens: a run lies in one group, a chunk need not.  Of the 16 rows of activations that the matrix instruction
// takes, row 4 p + t is token t's with zeros outside the p-th runs, so each run's sum comes out by itself and gets its own scale (4 bits,
// groups of 64, one token, 4096 x 4096: 9.2 us with runs of 16 instead).
template <typename T, int IB, int W, int L, bool ALIGNED, bool APART>
__global__ __launch_bounds__(512) void k_codes_product(const ProductArgs a) {
    constexpr int NB = L / W * IB;
    constexpr int FR = 8 / Elem<T>::PER16;  // 16-byte fragments in 8 weights
    constexpr int SUB = L / 8;
    constexpr int U = 16 / (SUB * FR);  // chunks of a batch: 64 registers of activations
    extern __shared__ __align__(128) unsigned char lds[];
    const unsigned char* table = Table<T, IB, W>::own(lds);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nw = blockDim.x >> 6;
    const int li = lane & 15, q = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    const int64_t row = min(n0 + li, a.rows - 1);  // rows and tokens behind the last one: computed from it, not stored
    const T* X = static_cast<const T*>(a.X) + min((int64_t)(APART ? li & 3 : li), a.n - 1) * a.ldx;
    const bool mine = !APART || li >> 2 == q;

    const int chunks = (int)((a.cols + 4 * L - 1) / (4 * L));
    const int each = (chunks + nw - 1) / nw;
    const int first = min(chunks, wave * each), last = min(chunks, first + each);
    const int full = min(last, (int)(a.cols / (4 * L)));  // chunks before this one are whole
    const int64_t row_bit = row * a.row_bits + q * NB;
    const int64_t row_bit_last = min(n0 + 15, a.rows - 1) * a.row_bits + 3 * NB;  // of this workgroup's last lane

    const Table<T, IB, W> entries(a.C, a.k, a.B, a.D);
    CodeRun<NB> run[U];
    float scale[U];
    u32x4 xf[U][SUB][FR];
    // without scales some word is read in their place, so that there is no branch between the loads
    const bool scaled = a.groups > 0;
    const float* S = scaled ? a.S + row * a.groups : reinterpret_cast<const float*>(a.words);
    auto ask = [&](int u, int ch, auto whole) {
        run[u].template load<ALIGNED, !decltype(whole)::value>(a.words, a.nwords, row_bit + (int64_t)ch * (4 * NB));
        // APART: the magic is that of runs; the last chunk's runs may lie behind the row
        scale[u] = S[APART ? min((int)__umulhi(2u * (unsigned)(ch * 4 + q), a.group_magic), max(a.groups - 1, 0)) : (int)__umulhi(2u * (unsigned)ch, a.group_magic)];
        if (APART) {
#pragma unroll
            for (int s = 0; s < SUB; ++s)
#pragma unroll
                for (int f = 0; f < FR; ++f) xf[u][s][f] = u32x4{0, 0, 0, 0};
        }
        if (mine) {
#pragma unroll
            for (int s = 0; s < SUB; ++s) eight_of_row(xf[u][s], X, (int64_t)ch * (4 * L) + q * L + s * 8, a.cols, decltype(whole)::value);
        }
    };
    floatx4 acc{0.f, 0.f, 0.f, 0.f};
    auto use = [&](int u, int ch, auto whole) {
        floatx4 part{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
            u32x4 wf[FR];
            eight_weights<T, IB, W, NB>(wf, run[u], s, table);
            if (!decltype(whole)::value) cut_weights<T>(wf, (int64_t)ch * (4 * L) + q * L + s * 8, a.cols);
#pragma unroll
            for (int f = 0; f < FR; ++f) mma16<T>(part, xf[u][s][f], wf[f]);
        }
        const float by = scaled ? scale[u] : 1.f;
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[r] = fmaf(by, part[r], acc[r]);
    };
    const std::true_type whole;
    const std::false_type broken;
    // chunks before this one are whole, and the words that their runs may touch are all there
    const int64_t room = a.nwords * 32 - 32 * (ALIGNED ? CodeRun<NB>::NWORDS : CodeRun<NB>::SPAN) - row_bit_last;
    const int safe = room < 0 ? first : (int)max((int64_t)first, min((int64_t)full, room / (4 * NB) + 1));
    int ch = first;
    bool built = false;
    if (ch + U <= safe) {
#pragma unroll
        for (int u = 0; u < U; ++u) ask(u, ch + u, whole);
        entries.build(lds, a.C, a.k, a.B, a.D);
        __syncthreads();
        built = true;
        for (;;) {
#pragma unroll
            for (int u = 0; u < U; ++u) use(u, ch + u, whole);
            ch += U;
            if (ch + U > safe) break;
#pragma unroll
            for (int u = 0; u < U; ++u) ask(u, ch + u, whole);
        }
    }
    if (!built) {
        entries.build(lds, a.C, a.k, a.B, a.D);
        __syncthreads();
    }
    for (; ch < last; ++ch) {
        if (ch < safe) {
            ask(0, ch, whole);
            use(0, ch, whole);
        } else {
            ask(0, ch, broken);
            use(0, ch, broken);
        }
    }
    // the wavefronts' sums: [wave][token][row]
    __syncthreads();
    float* red = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int r = 0; r < 4; ++r) red[(wave * 16 + q * 4 + r) * 16 + li] = acc[r];
    __syncthreads();
    for (int e = threadIdx.x; e < (APART ? 64 : 256); e += blockDim.x) {
        float sum = 0.f;
        for (int w = 0; w < nw; ++w) {
#pragma unroll
            for (int p = 0; p < (APART ? 4 : 1); ++p) sum += red[w * 256 + p * 64 + e];
        }
        const int64_t t = e >> 4, n = n0 + (e & 15);
        if (t < a.n && n < a.rows) static_cast<T*>(a.Y)[t * a.ldy + n] = Elem<T>::down(sum);
    }
}

// More than 16 tokens: 16 NT of them and 64 rows of the layer to a workgroup.  Its wavefronts are G teams of four, one for each 16 rows;
// the teams take the steps of 128 columns in turn.  The codes go the same way as above.  The activations, which all four wavefronts of a
// team need, come through LDS: up to ST - 1 steps ahead, copied there without passing registers, 16-byte pieces of row r in the
// order c ^ (r mod 8).  gridDim.z workgroups share the columns; every one of them reads all tokens' activations of its columns, so that a
// compute unit reads its share of X instead of all of it (64 tokens of 4096 columns are 512 KB).
// Rows of X begin at multiples of 16 bytes and go on to a multiple of 128 columns, with zeros behind the layer's last.
// 61 tokens, 4096 x 4096, 3 bits, groups of 64, bfloat16: 14.6 us and 3.9 for the joining of four parts; 4 bits in groups of 128, 64 tokens: 13 in
// all.  A workgroup has eight steps here: it is bound by the issue of instructions by G wavefronts a SIMD, so offsets inside a workgroup's rows and tokens are 32 bits
// (16 rows of 4,000,000 codes of 8 bits are 2^29 bits, 64 tokens of as many float columns 2^30 bytes).
template <typename T, int NT>
struct TileOfTokens {
    static constexpr int ROW = 128 * (int)sizeof(T);  // bytes of a token's step
    static constexpr int STAGE = NT * 16 * ROW;
    static constexpr int G = sizeof(T) == 4 ? 2 : 4, THREADS = 256 * G;
    static constexpr int FIT = 128 * 1024 / (G * STAGE);
    static constexpr int ST = FIT < 4 ? FIT : 4;
    static constexpr int TABLE = 32 * 1024;
    static constexpr int LDS = TABLE + G * ST * STAGE;
    static_assert(ST >= 2, "stages");
};

template <typename T, int IB, int W, int L, int NT, bool ALIGNED>
__global__ __launch_bounds__((TileOfTokens<T, NT>::THREADS)) void k_codes_tile(const ProductArgs a) {
    typedef TileOfTokens<T, NT> Tile;
    constexpr int G = Tile::G;
    constexpr int NB = L / W * IB;
    constexpr int PER = Elem<T>::PER16, FR = 8 / PER, SUB = L / 8, CC = 32 / L;
    constexpr int ROW = Tile::ROW, PIECES_ROW = ROW / 16, ST = Tile::ST;
    constexpr int PP = Tile::STAGE / 1024 / 4;  // copies of a wavefront for a step
    static_assert(Table<T, IB, W>::BYTES <= Tile::TABLE, "table");
    extern __shared__ __align__(1024) unsigned char lds[];
    const unsigned char* table = Table<T, IB, W>::own(lds);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = lane & 15, q = lane >> 4, rw = wave & 3, team = wave >> 2;
    unsigned char* stage = lds + Tile::TABLE + team * ST * Tile::STAGE;
    const Table<T, IB, W> entries(a.C, a.k, a.B, a.D);
    // 16 rows from n0 on, clamped; 16 NT tokens from t0 on
    const int64_t n0 = min((int64_t)blockIdx.x * 64 + rw * 16, a.rows - 1), t0 = (int64_t)blockIdx.y * (16 * NT);
    const int row = (int)min((int64_t)li, a.rows - 1 - n0);
    const int whole = (int)(a.cols / 128);  // steps without the broken one
    const int each = (whole + gridDim.z - 1) / gridDim.z;
    const int first = min(whole, (int)blockIdx.z * each), last = min(whole, first + each);
    const int turns = (last - first + G - 1) / G;  // steps first + G i + team; some teams may have no last one
    const int64_t bit0 = n0 * a.row_bits;
    // offsets count from a word from which on there are at least SPAN of them (the stream has 32)
    const int64_t word0 = min(bit0 >> 5, a.nwords - CodeRun<NB>::SPAN);
    const uint32_t* words = a.words + word0;
    const int limit = (int)min(a.nwords - word0 - CodeRun<NB>::SPAN, (int64_t)1 << 30);
    const unsigned row_bit = (unsigned)(bit0 - (word0 << 5)) + (unsigned)row * (unsigned)a.row_bits + q * NB;
    const bool scaled = a.groups > 0;
    const float* S = scaled ? a.S + n0 * a.groups : nullptr;
    const unsigned S_row = (unsigned)(row * a.groups);
    const unsigned char* X = reinterpret_cast<const unsigned char*>(static_cast<const T*>(a.X) + t0 * a.ldx);

    unsigned src[PP];  // of this lane's pieces, from X on
#pragma unroll
    for (int p = 0; p < PP; ++p) {
        const int at = (rw * PP + p) * 64 + lane, r = at / PIECES_ROW, c = (at % PIECES_ROW) ^ (r & 7);
        src[p] = (unsigned)min((int64_t)r, a.n - 1 - t0) * (unsigned)(a.ldx * sizeof(T)) + c * 16;
    }
    auto fetch = [&](int step, int slot) {
        const unsigned char* from = X + (int64_t)step * ROW;
#pragma unroll
        for (int p = 0; p < PP; ++p)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(from + src[p]),
                                             (__attribute__((address_space(3))) void*)(stage + slot * Tile::STAGE + (rw * PP + p) * 1024), 16,
                                             0, 0);
    };
    auto scale_of = [&](int chunk) {
        if (!scaled) return 1.f;
        return S[S_row + min(__umulhi(2u * (unsigned)chunk, a.group_magic), (unsigned)(a.groups - 1))];
    };
    CodeRun<NB> run[ST][CC];
    float scale[ST][CC];
    auto ask = [&](int step, int slot) {
#pragma unroll
        for (int c = 0; c < CC; ++c) {
            run[slot][c].template load_inside<ALIGNED>(words, limit, row_bit + (unsigned)(step * CC + c) * (4 * NB));
            scale[slot][c] = scale_of(step * CC + c);
        }
    };
    floatx4 acc[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[j] = floatx4{0.f, 0.f, 0.f, 0.f};
    auto use = [&](const CodeRun<NB>& codes, float by, int c, int slot, int64_t cut) {
        const unsigned char* x = stage + slot * Tile::STAGE + li * ROW;
        floatx4 part[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) part[j] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < SUB; ++s) {
            u32x4 wf[FR];
            eight_weights<T, IB, W, NB>(wf, codes, s, table);
            const int k = c * 4 * L + q * L + s * 8;
            if (cut >= 0) cut_weights<T>(wf, cut + k, a.cols);
#pragma unroll
            for (int f = 0; f < FR; ++f) {
                const unsigned char* piece = x + (((k / PER + f) ^ (li & 7)) << 4);
#pragma unroll
                for (int j = 0; j < NT; ++j) mma16<T>(part[j], *reinterpret_cast<const u32x4*>(piece + j * 16 * ROW), wf[f]);
            }
        }
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[j][r] = fmaf(by, part[j][r], acc[j][r]);
    };
#pragma unroll
    for (int u = 0; u < ST - 1; ++u)
        if (u < turns) {
            const int step = min(first + G * u + team, last - 1);
            ask(step, u);
            fetch(step, u);
        }
    entries.build(lds, a.C, a.k, a.B, a.D);
    for (int i0 = 0; i0 < turns; i0 += ST) {
#pragma unroll
        for (int u = 0; u < ST; ++u) {
            const int i = i0 + u;
            if (i < turns) {
                // this step's copies are there: of all loads at most as many may be missing as the copies of the ST - 2 steps behind
                // it, and near the end, where there are fewer steps behind it, none
                asm volatile("" ::: "memory");
                if (i + ST - 2 < turns)
                    __builtin_amdgcn_s_waitcnt(0x0070 | ((PP * (ST - 2)) & 15) | (((PP * (ST - 2)) >> 4) << 14));
                else
                    __builtin_amdgcn_s_waitcnt(0x0070);
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                if (i + ST - 1 < turns) {
                    const int step = min(first + G * (i + ST - 1) + team, last - 1);
                    ask(step, (u + ST - 1) % ST);
                    fetch(step, (u + ST - 1) % ST);
                }
                if (first + G * i + team < last) {
#pragma unroll
                    for (int c = 0; c < CC; ++c) use(run[u][c], scale[u][c], c, u, -1);
                }
            }
        }
    }
    __syncthreads();
    if (whole * (int64_t)128 < a.cols && blockIdx.z + 1 == gridDim.z) {  // the row's broken step
        if (team == 0) fetch(whole, 0);
        __builtin_amdgcn_s_waitcnt(0x0070);
        __syncthreads();
        if (team == 0)
            for (int c = 0; c < CC; ++c) {
                CodeRun<NB> codes;
                codes.template load<false, true>(a.words, a.nwords, (n0 + row) * a.row_bits + q * NB + (int64_t)(whole * CC + c) * (4 * NB));
                use(codes, scale_of(whole * CC + c), c, 0, (int64_t)whole * 128);
            }
        __syncthreads();
    }
    // The teams' sums, in order: tile j of the tokens is finished by team j mod G.
    float* red = reinterpret_cast<float*>(lds + Tile::TABLE) + rw * (NT * 256) + lane * 4;
#pragma unroll
    for (int j = 0; j < NT; ++j)
        if (j % G != team) *reinterpret_cast<floatx4*>(red + (team * 4 * NT + j) * 256) = acc[j];
    __syncthreads();
    if ((int64_t)blockIdx.x * 64 + rw * 16 + li >= a.rows) return;
    const bool shared = gridDim.z > 1;
    const int64_t pitch = shared ? a.rows : a.ldy;
    const int64_t out0 = ((shared ? (int64_t)blockIdx.z * a.n : 0) + t0 + q * 4) * pitch + n0 + li;
    float* sums = a.sums + out0;
    T* Y = static_cast<T*>(a.Y) + out0;
    const int tokens = (int)min(a.n - t0, (int64_t)(16 * NT));
#pragma unroll
    for (int j = 0; j < NT; ++j)
        if (j % G == team) {
            floatx4 sum{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int g = 0; g < G; ++g) sum += g == team ? acc[j] : *reinterpret_cast<const floatx4*>(red + (g * 4 * NT + j) * 256);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (j * 16 + q * 4 + r >= tokens) continue;
                if (shared) sums[(j * 16 + r) * pitch] = sum[r];
                else Y[(j * 16 + r) * pitch] = Elem<T>::down(sum[r]);
            }
        }
}

}  // namespace idkm

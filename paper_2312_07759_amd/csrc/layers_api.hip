// C entry points of the operators on coded layers (products and their gradients), group scales and the loss against a
// teacher: checks of arguments, choice of kernels, layout of the caller's workspace.
#include <cfloat>
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <exception>
#include <new>

#include "../../include/idkm.h"
#include "layers.h"

namespace idkm {

int context_device(const idkm_ctx* ctx);
void context_error(idkm_ctx* ctx, const char* msg);

ProductFn codes_product_kernel_1(int, int, int, bool, bool);
ProductFn codes_product_kernel_2(int, int, int, bool, bool);
ProductFn codes_product_kernel_3(int, int, int, bool, bool);
ProductFn codes_product_kernel_4(int, int, int, bool, bool);
ProductFn codes_product_kernel_5(int, int, int, bool, bool);
ProductFn codes_product_kernel_6(int, int, int, bool, bool);
ProductFn codes_product_kernel_7(int, int, int, bool, bool);
ProductFn codes_product_kernel_8(int, int, int, bool, bool);

ProductFn codes_tile_kernel_1(int, int, int, int, bool);
ProductFn codes_tile_kernel_2(int, int, int, int, bool);
ProductFn codes_tile_kernel_3(int, int, int, int, bool);
ProductFn codes_tile_kernel_4(int, int, int, int, bool);
ProductFn codes_tile_kernel_5(int, int, int, int, bool);
ProductFn codes_tile_kernel_6(int, int, int, int, bool);
ProductFn codes_tile_kernel_7(int, int, int, int, bool);
ProductFn codes_tile_kernel_8(int, int, int, int, bool);

DenseFn codes_dense_kernel_1(int, int, bool, bool);
DenseFn codes_dense_kernel_2(int, int, bool, bool);
DenseFn codes_dense_kernel_3(int, int, bool, bool);
DenseFn codes_dense_kernel_4(int, int, bool, bool);
DenseFn codes_dense_kernel_5(int, int, bool, bool);
DenseFn codes_dense_kernel_6(int, int, bool, bool);
DenseFn codes_dense_kernel_7(int, int, bool, bool);
DenseFn codes_dense_kernel_8(int, int, bool, bool);

DenseFn codes_dense_kernel(int dtype, int IB, int W, bool columns, bool aligned) {
    static DenseFn (*const by_bits[8])(int, int, bool, bool) = {
        codes_dense_kernel_1, codes_dense_kernel_2, codes_dense_kernel_3, codes_dense_kernel_4,
        codes_dense_kernel_5, codes_dense_kernel_6, codes_dense_kernel_7, codes_dense_kernel_8};
    return IB >= 1 && IB <= 8 ? by_bits[IB - 1](dtype, W, columns, aligned) : nullptr;
}

ProductFn codes_tile_kernel(int dtype, int IB, int W, int L, int NT, bool aligned) {
    static ProductFn (*const by_bits[8])(int, int, int, int, bool) = {
        codes_tile_kernel_1, codes_tile_kernel_2, codes_tile_kernel_3, codes_tile_kernel_4,
        codes_tile_kernel_5, codes_tile_kernel_6, codes_tile_kernel_7, codes_tile_kernel_8};
    return IB >= 1 && IB <= 8 ? by_bits[IB - 1](dtype, W, L, NT, aligned) : nullptr;
}

ProductFn codes_product_kernel(int dtype, int IB, int W, int L, bool aligned, bool apart) {
    static ProductFn (*const by_bits[8])(int, int, int, bool, bool) = {
        codes_product_kernel_1, codes_product_kernel_2, codes_product_kernel_3, codes_product_kernel_4,
        codes_product_kernel_5, codes_product_kernel_6, codes_product_kernel_7, codes_product_kernel_8};
    return IB >= 1 && IB <= 8 ? by_bits[IB - 1](dtype, W, L, aligned, apart) : nullptr;
}

}  // namespace idkm

using namespace idkm;

namespace {

constexpr int64_t MAX_SIDE = 4000000;      // rows, columns, tokens: 64 of them to a workgroup fit one grid dimension
constexpr int64_t MAX_VOCABULARY = (int64_t)1 << 29;  // offsets in a row are 32 bits of bytes
constexpr int64_t MAX_SCALED_COLS = INT_MAX - 63;  // a lane's 32-bit place in a row goes up to 64 weights beyond its end
constexpr int64_t PANEL = (int64_t)1 << 26;  // weights of a layer that are written out at a time

idkm_status refuse(idkm_ctx* ctx, idkm_status s, const char* msg) {
    if (ctx) context_error(ctx, msg);
    return s;
}

// The context's device is the current one inside; the caller's is again after it.
struct OnDevice {
    int before = -1;
    bool ok = false;
    explicit OnDevice(int device) {
        if (hipGetDevice(&before) != hipSuccess) return;
        ok = before == device || hipSetDevice(device) == hipSuccess;
        if (before == device) before = -1;
    }
    ~OnDevice() {
        if (ok && before >= 0) (void)hipSetDevice(before);
    }
};

// Runs body() on the context's device; no exception leaves a C entry point.
template <class Body>
idkm_status entry(idkm_ctx* ctx, Body body) noexcept {
    if (!ctx) return IDKM_ERR_INVALID_ARG;
    try {
        context_error(ctx, "");
        return body();
    } catch (const std::bad_alloc&) {
        return IDKM_ERR_ALLOC;
    } catch (...) {
        return IDKM_ERR_DEVICE;
    }
}

template <class Launches>
idkm_status launched(idkm_ctx* ctx, Launches launches) {
    OnDevice on(context_device(ctx));
    if (!on.ok) {
        (void)hipGetLastError();
        return refuse(ctx, IDKM_ERR_DEVICE, "the context's device cannot be made current");
    }
    launches();
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? IDKM_OK : refuse(ctx, IDKM_ERR_DEVICE, hipGetErrorString(e));
}

int64_t up_to(int64_t x, int64_t unit) { return (x + unit - 1) / unit * unit; }
int esize_of(int dtype) { return dtype == IDKM_F32 ? 4 : 2; }
bool aligned_to(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

const char* wrong_layer(const idkm_codes_desc* w, idkm_status* st) {
    *st = IDKM_ERR_INVALID_ARG;
    if (!w) return "the layer must be non-NULL";
    if (!w->words || !w->C) return "words and C must be non-NULL";
    if (w->dtype != IDKM_F32 && w->dtype != IDKM_F16 && w->dtype != IDKM_BF16) return "dtype must be an idkm_dtype";
    if (w->rows < 1 || w->cols < 1) return "rows and cols must be >= 1";
    if (w->k < 1 || w->k > 1024 || w->d < 1 || w->d > 64) return "need 1 <= k <= 1024 and 1 <= d <= 64";
    if (w->cols % w->d != 0) return "cols must be a multiple of d";
    if (w->S) {
        if (w->group < 1) return "group must be >= 1 where there are scales";
        if (w->group < w->cols && (w->group % 32 != 0 || w->group % w->d != 0))
            return "a group shorter than a row must be a multiple of 32 and of d";
        if (!aligned_to(w->S, 4)) return "S must be aligned to its type";
    }
    if (!aligned_to(w->words, 4) || !aligned_to(w->C, esize_of(w->dtype))) return "words and C must be aligned to their types";
    *st = IDKM_ERR_UNSUPPORTED;
    if (w->rows > MAX_SIDE || w->cols > MAX_SIDE || w->rows * w->cols > ((int64_t)1 << 36)) return "the layer is too large";
    return nullptr;
}

int groups_of(const idkm_codes_desc& w) { return w.S ? (int)((w.cols + w.group - 1) / w.group) : 0; }

// ---- straight from the codes

struct FewPlan {
    ProductFn fn = nullptr;
    unsigned group_magic = 0;
    int threads;
    int64_t pad = 0;  // columns to which X is brought for the tiles
    int parts = 1;  // workgroups that share a row's sum
    dim3 grid;
    size_t lds;
};

// The matrix-vector form takes up to 16 tokens, tiles of 32 or 64 tokens more, as long as decoding the layer for each of them is
// expected to take less time than writing it out once (see below).
constexpr int64_t VECTOR_TOKENS = 16;

float dense_us(const idkm_codes_desc& w, int64_t n);

FewPlan few_plan(const idkm_codes_desc& w, int64_t n) {
    FewPlan p;
    const int bits = idkm_code_bits(w.k);
    if (bits > 8 || (w.d != 1 && w.d != 2 && w.d != 4 && w.d != 8)) return p;
    // a chunk of four runs has to lie in one group, where their sums are not kept apart
    const bool together = !w.S || w.group >= w.cols || w.group % 128 == 0, apart = !together && n <= 4;
    const int L = together || apart ? 32 : w.group % 64 == 0 ? 16 : 8;
    const int at_once = codes_at_once(bits, w.d), IB = at_once * bits, W = at_once * w.d;
    const int64_t chunks = (w.cols + 4 * L - 1) / (4 * L);
    if (w.S && w.group < w.cols) {  // in chunks, or runs; exact while all (those of a group) < 2^31
        const int64_t of_group = w.group / (apart ? 32 : 4 * L);
        if ((apart ? 4 : 1) * chunks * of_group >= ((int64_t)1 << 31)) return p;
        p.group_magic = (unsigned)((((int64_t)1 << 31) + of_group - 1) / of_group);
    }
    if (n > VECTOR_TOKENS && w.rows * w.cols / w.d * bits < 1024) return p;  // a run's words have to be there
    const bool aligned = (w.cols / w.d * bits) % 32 == 0 && (32 / W * IB) % 32 == 0;
    if (n <= VECTOR_TOKENS) {
        p.fn = codes_product_kernel(w.dtype, IB, W, L, aligned, apart);
        const int waves = chunks < 8 ? (int)chunks : 8;
        p.threads = waves * 64;
        p.grid = dim3((unsigned)((w.rows + 15) / 16));
        const size_t table = (size_t)128 << IB, sums = (size_t)waves * 1024;
        p.lds = table > sums ? table : sums;
        return p;
    }
    const int NT = n <= 32 ? 2 : 4;
    p.fn = codes_tile_kernel(w.dtype, IB, W, L, NT, aligned);
    p.threads = w.dtype == IDKM_F32 ? TileOfTokens<float, 2>::THREADS : TileOfTokens<bf16, 2>::THREADS;
    p.pad = up_to(w.cols, 128);
    const int64_t steps = p.pad / 128;
    // Workgroups, one to a compute unit, in rounds: some 2 us and these for every step of 128 columns, by the runs' length (32, 16, 8) and by the
    // weights that a lookup gives (1, 2, 4 and more): measured, 4096 x 4096, 512 and 1024 tokens, codebooks of 2 to 256 codewords; sums in
    // parts cost as in tile_plan.  Both forms, measured, 256 tokens in bfloat16, scales for 32 weights: 43 us from the codes and 38 written out with 16 codewords,
    // 58 and 38 with 256; for 128 weights 24 and 39, 24 and 35; 512 tokens 43 and 47, 44 and 45.
    static const float measured[2][3][3] = {{{0.65f, 1.05f, 1.7f}, {0.6f, 1.02f, 1.23f}, {0.55f, 0.85f, 1.23f}},
                                            {{2.5f, 2.85f, 3.75f}, {2.45f, 2.85f, 3.25f}, {2.4f, 2.65f, 3.25f}}};
    const float step_us = measured[w.dtype == IDKM_F32][W == 1 ? 0 : W == 2 ? 1 : 2][L == 32 ? 0 : L == 16 ? 1 : 2];
    const int64_t blocks = (w.rows + 63) / 64, tokens = (n + 16 * NT - 1) / (16 * NT);
    float best = 0.f;
    for (int parts = 1; parts <= 16 && (parts == 1 || steps / parts >= 4); ++parts) {
        const int64_t rounds = (blocks * tokens * parts + 255) / 256;
        float us = (float)rounds * (2.f + step_us * (float)((steps + parts - 1) / parts));
        if (parts > 1) us += 3.5f + 2e-6f * (float)n * (float)w.rows * (float)parts;
        if (best == 0.f || us < best) {
            best = us;
            p.parts = parts;
        }
    }
    if (best > dense_us(w, n)) {
        p.fn = nullptr;
        return p;
    }
    p.grid = dim3((unsigned)blocks, (unsigned)tokens, (unsigned)p.parts);
    p.lds = w.dtype == IDKM_F32 ? (NT == 2 ? TileOfTokens<float, 2>::LDS : TileOfTokens<float, 4>::LDS)
                                : (NT == 2 ? TileOfTokens<bf16, 2>::LDS : TileOfTokens<bf16, 4>::LDS);
    return p;
}

// Workspace: the parts' sums, and X with whole steps (which not every call needs).
int64_t few_sums(const FewPlan& p, const idkm_codes_desc& w, int64_t n) { return p.parts > 1 ? up_to(4 * p.parts * n * w.rows, 256) : 0; }
int64_t few_bytes(const FewPlan& p, const idkm_codes_desc& w, int64_t n) {
    return few_sums(p, w, n) + up_to(n * p.pad * esize_of(w.dtype), 256);
}

// ---- tile products

struct TilePlan {
    int which, parts;
    float us;  // expected
    int scaled;  // see tile_shape
};

int64_t tiles_of(const TileShape& t, int64_t M, int64_t N) { return ((M + t.bm - 1) / t.bm) * ((N + t.bn - 1) / t.bn); }

// Float32 parts that go to memory and come back (4 TB/s), and the launch that joins them.
float join_us(int64_t M, int64_t N, int parts) { return parts > 1 ? 3.5f + 2e-6f * (float)M * (float)N * (float)parts : 0.f; }

// A shape with the number of parts of the sum with the least time by its measured step: rounds of workgroups, and the joining of the parts.
TilePlan shape_plan(int which, const TileShape& t, int64_t M, int64_t N, int64_t steps, int scaled) {
    TilePlan best{which, 1, 0.f, scaled};
    const int64_t tiles = tiles_of(t, M, N);
    for (int parts = 1; parts <= 16 && (parts == 1 || steps / parts >= 2); ++parts) {
        // two workgroups share a compute unit's matrix cores, one alone does not use all of them
        float rounds = (float)((tiles * parts + 255) / 256) * 256.f / (float)t.resident;
        if (rounds < 0.7f) rounds = 0.7f;
        const float us = rounds * t.us * (float)((steps + parts - 1) / parts) + join_us(M, N, parts);
        if (best.us == 0.f || us < best.us) best = TilePlan{which, parts, us, scaled};
    }
    return best;
}

// .. and the shape with the least time.
TilePlan tile_plan(int64_t M, int64_t N, int64_t steps, int dtype, int scaled) {
    TilePlan best{0, 1, 0.f, scaled};
    for (int s = 0;; ++s) {
        const TileShape t = tile_shape(dtype, s, scaled);
        if (!t.fn) return best;
        const TilePlan p = shape_plan(s, t, M, N, steps, scaled);
        if (best.us == 0.f || p.us < best.us) best = p;
    }
}

unsigned set_tiles(const TileShape& t, int parts, TileArgs* a) {
    a->tiles_m = (int)((a->M + t.bm - 1) / t.bm);
    a->tiles_n = (int)((a->N + t.bn - 1) / t.bn);
    a->parts = parts;
    return (unsigned)(a->tiles_m * a->tiles_n) * (unsigned)parts;
}

// One product, or (second != nullptr, of the same shape) two in one launch.
void run_tiles(int dtype, const TilePlan& p, const TileArgs& args, hipStream_t s, const TilePlan* p2 = nullptr, const TileArgs* second = nullptr) {
    const TileShape t = tile_shape(dtype, p.which, p.scaled);
    TileJobs jobs{};
    jobs.job[0] = args;
    jobs.first = set_tiles(t, p.parts, &jobs.job[0]);
    unsigned grid = jobs.first;
    if (second) {
        jobs.job[1] = *second;
        grid += set_tiles(t, p2->parts, &jobs.job[1]);
    }
    allow_lds(reinterpret_cast<const void*>(t.fn), t.lds);
    hipLaunchKernelGGL(t.fn, dim3(grid), dim3((unsigned)t.threads), t.lds, s, jobs);
}

// Bytes of a buffer in the workspace.
int64_t buffer(int64_t elements, int esize) { return up_to(elements * esize, 256); }

// out[M, N] in T (rows ldo apart): in one part, or in several that are joined.
void set_out(const TilePlan& p, TileArgs* a, void* out, int64_t ldo, float* parts) {
    a->wide = p.parts > 1;
    a->out = a->wide ? (void*)parts : out;
    a->ldo = a->wide ? a->N : ldo;
}
void run_product(int dtype, const TilePlan& p, TileArgs a, void* out, int64_t ldo, float* parts, hipStream_t s) {
    set_out(p, &a, out, ldo, parts);
    run_tiles(dtype, p, a, s);
    if (p.parts > 1) launch_join_parts(dtype, parts, p.parts, a.M, a.N, out, ldo, s);
}

int64_t panel_of(int64_t lines, int64_t length) {
    int64_t p = PANEL / length / 256 * 256;
    if (p < 256) p = 256;
    return p < lines ? p : lines;
}

DenseArgs dense_of(const idkm_codes_desc& w) {
    DenseArgs a{};
    a.words = w.words;
    a.nwords = idkm_code_words(w.rows * w.cols / w.d, w.k);
    a.rows = w.rows;
    a.cols = w.cols;
    a.C = w.C;
    a.k = w.k;
    a.d = w.d;
    a.bits = idkm_code_bits(w.k);
    a.S = w.S;
    a.group = w.S ? (w.group < w.cols ? w.group : (int)w.cols) : 1;
    a.groups = groups_of(w);
    a.row_bits = w.cols / w.d * a.bits;
    a.d_log = w.d == 8 ? 3 : w.d == 4 ? 2 : w.d == 2 ? 1 : 0;
    a.group_32 = a.group >= 32 ? a.group / 32 : 1;
    a.group_magic = a.groups > 1 ? (unsigned)((((int64_t)1 << 31) + a.group_32 - 1) / a.group_32) : 0;
    return a;
}

// Layout of the workspace of a product: operand rows brought to whole steps, the layer's panel, parts.
struct ProductLayout {
    int64_t pad, panel, operand, matrix, parts, scales, scale_pitch, bytes;
    TilePlan plan;
};

// lines: the layer's rows (product) or columns (dX); sum: the other side.  plan: null for the best one.
// scaled: see scaled_of; the scales of a panel's groups are laid out anew.
ProductLayout product_layout(int dtype, int64_t n, int64_t lines, int64_t sum, const TilePlan* plan = nullptr, int scaled = 0, int groups = 0) {
    const int es = esize_of(dtype);
    ProductLayout l;
    l.pad = up_to(sum, TP_STEP / es);
    l.panel = panel_of(lines, l.pad);
    l.plan = plan ? *plan : tile_plan(n, l.panel, l.pad * es / TP_STEP, dtype, scaled);
    l.operand = 0;
    l.matrix = buffer(n * l.pad, es);
    l.parts = l.matrix + buffer(l.panel * l.pad, es);
    l.scales = l.parts + (l.plan.parts > 1 ? buffer(n * l.panel * l.plan.parts, 4) : 0);
    l.scale_pitch = up_to(l.panel, 128);
    l.bytes = l.scales + (scaled ? buffer(groups * l.scale_pitch, 4) : 0);
    return l;
}

// Which tile product multiplies by the scales of a layer that is written out for Y: with 16-bit types it is one that takes them beside the
// codewords, so that S C is not rounded; groups of odd multiples of 32 take the one that looks for a scale every half step.
int scaled_of(const idkm_codes_desc& w) {
    if (!w.S || w.dtype == IDKM_F32) return 0;
    return w.group >= w.cols || w.group % 64 == 0 ? 1 : 2;
}

ProductLayout written_out(const idkm_codes_desc& w, int64_t n) {
    return product_layout(w.dtype, n, w.rows, w.cols, nullptr, scaled_of(w), groups_of(w));
}

// Expected time of a product whose layer is written out: 0.6 (float: 1) us for a million weights, and launches.
float dense_us(const idkm_codes_desc& w, int64_t n) {
    const ProductLayout l = written_out(w, n);
    return 8.f + (w.dtype == IDKM_F32 ? 1e-6f : 0.6e-6f) * (float)w.rows * (float)l.pad + l.plan.us * (float)((w.rows + l.panel - 1) / l.panel);
}

// The operand as the tile product takes it: itself, or a copy with whole steps, which `copies` is to make.
void operand_of(int dtype, const void* in, int64_t ldi, int64_t n, int64_t sum, const ProductLayout& l, unsigned char* ws, TileArgs* a,
                OperandArgs* copies) {
    const int es = esize_of(dtype);
    if (sum == l.pad && ldi * es % 16 == 0 && aligned_to(in, 16)) {
        a->A = in;
        a->lda = ldi;
    } else {
        add_operand(copies, in, ldi, n, sum, ws + l.operand, l.pad, false);
        a->A = ws + l.operand;
        a->lda = l.pad;
    }
    a->M = n;
    a->ldb = l.pad;
    a->B = ws + l.matrix;
    a->steps = (int)(l.pad * es / TP_STEP);
}

// Gradients of the layer itself.
struct LayerGradLayout {
    int64_t pad, ldp, panel, panels, dy, x, p, bins, segments, bytes;
    TilePlan plan;
    bool runs, wide, segmented;  // which of the kernels for bins
    int group, groups, lanes, run, waves, codes, grid;
};

LayerGradLayout layer_grad_layout(const idkm_codes_desc& w, int64_t n, const TilePlan* plan = nullptr) {
    const int es = esize_of(w.dtype), bits = idkm_code_bits(w.k);
    LayerGradLayout l{};
    l.pad = up_to(n, TP_STEP / es);
    l.ldp = up_to(w.cols, 8);
    l.panel = panel_of(w.rows, l.ldp);
    l.panels = (w.rows + l.panel - 1) / l.panel;
    l.plan = plan ? *plan : tile_plan(l.panel, w.cols, l.pad * es / TP_STEP, w.dtype, 0);
    l.group = w.S ? (int)(w.group < w.cols ? w.group : w.cols) : 0;
    l.runs = bits <= 8 && (w.d == 1 || w.d == 2 || w.d == 4 || w.d == 8) && w.rows * w.cols / w.d * bits > 96;
    l.wide = l.runs && w.k * w.d > 256;  // bins of all components for every lane: 64 KB a wavefront at most
    int64_t tasks;  // of a wavefront, in a panel
    int bin_bytes;  // of a wavefront
    if (l.runs) {
        if (!w.S) l.group = (int)up_to(w.cols, 8);
        l.groups = w.S ? groups_of(w) : 1;
        // lanes of a group of 8 m columns lie together in a wavefront's 512 where m is a power of two
        l.segmented = w.S && (l.wide || l.group > 512 || l.group % 8 != 0 || (l.group & (l.group - 1)) != 0);
        tasks = l.panel * ((w.cols + 511) / 512);
        bin_bytes = l.wide ? w.k * 256 / bins_shared_by(w.k) : w.k * w.d * 256;
        l.codes = w.k;
    } else {
        // a wavefront takes groups of a row at a time; without scales, some hundred columns
        if (!w.S) l.group = (int)(w.cols < 512 ? w.cols : 512 / w.d * w.d);
        l.groups = (int)((w.cols + l.group - 1) / l.group);
        l.lanes = 64 / w.d * w.d;
        if (w.S && l.group % 64 == 32 && l.group < 256 && 32 % w.d == 0) l.lanes = 32;  // no step of which half is behind the group
        const int steps = (l.group + l.lanes - 1) / l.lanes;
        l.run = steps >= 16 ? 1 : 16 / steps;
        if (l.run > l.groups) l.run = l.groups;
        l.codes = w.k < 512 ? w.k : 512;  // bins of 512 codewords fill 128 KB
        tasks = l.panel * ((l.groups + l.run - 1) / l.run);
        bin_bytes = l.codes * 256;
    }
    l.waves = 128 * 1024 / bin_bytes;
    if (l.waves > 4) l.waves = 4;
    // as many workgroups as the compute units hold at once: every one has bins to clear and to write
    int64_t grid = (tasks + l.waves - 1) / l.waves, most = 256 * (150 * 1024 / (bin_bytes * l.waves + 4096));
    if (most > 2048) most = 2048;
    l.grid = (int)(grid < most ? grid : most);
    l.dy = 0;
    l.x = buffer(w.rows * l.pad, es);
    l.p = l.x + buffer(w.cols * l.pad, es);
    l.bins = l.p + buffer(l.panel * l.ldp * l.plan.parts, 4);
    l.segments = l.bins + buffer(l.panels * l.grid * w.k * w.d, 4);
    l.bytes = l.segments + (l.segmented ? buffer(w.rows * ((w.cols + 31) / 32), 4) : 0);
    return l;
}

// Both products of a backward pass: each in launches of its own, or in one launch, where the layer is one panel of either.
struct GradLayout {
    ProductLayout d;
    LayerGradLayout l;
    bool together;
    int64_t bytes;
};

// The same for any of the gradients: their bits do not depend on which others are wanted.
GradLayout grad_layout(const idkm_codes_desc& w, int64_t n) {
    GradLayout g;
    g.d = product_layout(w.dtype, n, w.cols, w.rows);
    g.l = layer_grad_layout(w, n);
    g.together = false;
    g.bytes = g.d.bytes + g.l.bytes;
    if (g.d.panel < w.cols || g.l.panels > 1) return g;
    // In one launch there is one rest of workgroups that do not fill the device instead of two, and one launch less.  Longer sums go
    // first, so that on average half a workgroup of the shorter ones is what the last compute unit is behind.  Whole calls, apart and together:
    // 512 x 4608 float32, 1001 tokens 144 and 122 us; 1024 x 1024, 1001 tokens 73 and 66, in bfloat16 36 and 32; 64 x 576 bfloat16 21 and
    // 17; 4096 x 4096 bfloat16, 64 tokens 73 and 80, which is left apart.
    const int64_t steps_d = g.d.pad * esize_of(w.dtype) / TP_STEP, steps_l = g.l.pad * esize_of(w.dtype) / TP_STEP;
    float least = g.d.plan.us + g.l.plan.us + 3.f;
    TilePlan best_d{}, best_l{};
    for (int s = 0;; ++s) {
        const TileShape t = tile_shape(w.dtype, s, 0);
        if (!t.fn) break;
        const TilePlan d = shape_plan(s, t, n, w.cols, steps_d, 0), l = shape_plan(s, t, w.rows, w.cols, steps_l, 0);
        const float count_d = (float)(tiles_of(t, n, w.cols) * d.parts), count_l = (float)(tiles_of(t, w.rows, w.cols) * l.parts);
        const float each_d = (float)((steps_d + d.parts - 1) / d.parts), each_l = (float)((steps_l + l.parts - 1) / l.parts);
        const float longer = each_d > each_l ? each_d : each_l, shorter = each_d > each_l ? each_l : each_d;
        const float alone = count_d + count_l <= 256.f && t.resident > 256 ? 0.7f : 1.f;
        // A workgroup begins and ends in some 2.4 us, of which two on a compute unit hide a part from each other: that tells where there are few
        // steps.  Nothing is left over where all are resident at once.
        const float ends = (t.resident > 256 ? 0.8f : 2.4f) / t.us;
        float us = (count_d * (each_d + ends) + count_l * (each_l + ends)) / (float)t.resident;
        if (count_d + count_l > (float)t.resident) us += 0.5f * shorter;
        if (us < alone * longer) us = alone * longer;
        us = us * t.us + join_us(n, w.cols, d.parts) + join_us(w.rows, w.cols, l.parts);
        if (us < least) {
            least = us;
            best_d = d;
            best_l = l;
            g.together = true;
        }
    }
    if (g.together) {
        g.d = product_layout(w.dtype, n, w.cols, w.rows, &best_d);
        g.l = layer_grad_layout(w, n, &best_l);
        g.bytes = g.d.bytes + g.l.bytes;
    }
    return g;
}

const char* wrong_workspace(const void* ws, int64_t have, int64_t need) {
    if (need == 0) return nullptr;
    if (!ws || have < need) return "the workspace is smaller than the size asked for";
    if (!aligned_to(ws, 16)) return "the workspace must be 16-byte aligned";
    return nullptr;
}

const char* wrong_scale_shape(int64_t rows, int64_t cols, int64_t group) {
    if (rows < 0 || cols < 1) return "need rows >= 0 and cols >= 1";
    if (group < 1) return "group must be >= 1";
    if (rows > ((int64_t)1 << 36) || cols > MAX_SCALED_COLS || (rows > 0 && cols > ((int64_t)1 << 36) / rows)) return "the matrix is too large";
    return nullptr;
}

ScaleArgs scale_args(int64_t rows, int64_t cols, int64_t group) {
    ScaleArgs a{};
    a.rows = rows;
    a.cols = cols;
    a.group = group < cols ? group : cols;
    a.groups = (cols + a.group - 1) / a.group;
    return a;
}

}  // namespace

extern "C" {

int64_t idkm_codes_linear_workspace(const idkm_codes_desc* w, int64_t n) {
    idkm_status st;
    if (wrong_layer(w, &st) || n < 0 || n > MAX_SIDE) return -1;
    if (n == 0) return 0;
    const FewPlan few = few_plan(*w, n);
    if (few.fn) return few_bytes(few, *w, n);
    return written_out(*w, n).bytes;
}

idkm_status idkm_codes_linear(idkm_ctx* ctx, const idkm_codes_desc* w, const void* X, int64_t n, int64_t ldx, void* Y, int64_t ldy,
                              void* workspace, int64_t workspace_bytes, void* hip_stream) {
    return entry(ctx, [&]() -> idkm_status {
        idkm_status st;
        if (const char* e = wrong_layer(w, &st)) return refuse(ctx, st, e);
        if (n < 0) return refuse(ctx, IDKM_ERR_INVALID_ARG, "n must be >= 0");
        if (n > MAX_SIDE) return refuse(ctx, IDKM_ERR_UNSUPPORTED, "too many tokens");
        if (n == 0) return IDKM_OK;
        const int es = esize_of(w->dtype);
        if (!X || !Y) return refuse(ctx, IDKM_ERR_INVALID_ARG, "X and Y must be non-NULL");
        if (ldx < w->cols || ldy < w->rows) return refuse(ctx, IDKM_ERR_INVALID_ARG, "ldx must be >= cols and ldy >= rows");
        if (!aligned_to(X, es) || !aligned_to(Y, es)) return refuse(ctx, IDKM_ERR_INVALID_ARG, "X and Y must be aligned to their type");
        hipStream_t s = (hipStream_t)hip_stream;
        const FewPlan few = few_plan(*w, n);
        if (few.fn) {
            ProductArgs a{};
            a.words = w->words;
            a.nwords = idkm_code_words(w->rows * w->cols / w->d, w->k);
            a.rows = w->rows;
            a.cols = w->cols;
            a.C = w->C;
            a.k = w->k;
            a.B = idkm_code_bits(w->k);
            a.D = w->d;
            a.row_bits = w->cols / w->d * a.B;
            a.S = w->S;
            a.groups = groups_of(*w);
            a.group_magic = few.group_magic;
            a.X = X;
            a.ldx = ldx;
            a.Y = Y;
            a.ldy = ldy;
            a.n = n;
            if (const char* e = wrong_workspace(workspace, workspace_bytes, few_bytes(few, *w, n)))
                return refuse(ctx, IDKM_ERR_INVALID_ARG, e);
            a.sums = static_cast<float*>(workspace);
            return launched(ctx, [&] {
                if (few.pad > 0 && (few.pad != w->cols || ldx * es % 16 != 0 || !aligned_to(X, 16) || ldx > (1 << 23))) {
                    void* copy = static_cast<unsigned char*>(workspace) + few_sums(few, *w, n);
                    OperandArgs o{};
                    add_operand(&o, X, ldx, n, w->cols, copy, few.pad, false);
                    launch_operands(w->dtype, o, s);
                    a.X = copy;
                    a.ldx = few.pad;
                }
                allow_lds(reinterpret_cast<const void*>(few.fn), few.lds);
                hipLaunchKernelGGL(few.fn, few.grid, dim3((unsigned)few.threads), few.lds, s, a);
                if (few.parts > 1) launch_join_parts(w->dtype, a.sums, few.parts, n, w->rows, Y, ldy, s);
            });
        }
        const ProductLayout l = written_out(*w, n);
        if (const char* e = wrong_workspace(workspace, workspace_bytes, l.bytes)) return refuse(ctx, IDKM_ERR_INVALID_ARG, e);
        unsigned char* ws = static_cast<unsigned char*>(workspace);
        return launched(ctx, [&] {
            TileArgs t{};
            OperandArgs copies{};
            operand_of(w->dtype, X, ldx, n, w->cols, l, ws, &t, &copies);
            launch_operands(w->dtype, copies, s);
            const int unit = l.plan.scaled == 1 ? 64 : 32;
            t.groups = groups_of(*w);
            t.group = w->group < w->cols ? w->group / unit : INT_MAX;
            t.scale_pitch = l.scale_pitch;
            float* scales = l.plan.scaled ? reinterpret_cast<float*>(ws + l.scales) : nullptr;
            t.scales = scales;
            for (int64_t r = 0; r < w->rows; r += l.panel) {
                DenseArgs a = dense_of(*w);
                a.scales_out = scales;
                a.scale_pitch = l.scale_pitch;
                a.first = r;
                a.count = w->rows - r < l.panel ? w->rows - r : l.panel;
                a.pad = l.pad;
                a.out = ws + l.matrix;
                launch_dense_rows(w->dtype, a, s);
                t.N = a.count;
                run_product(w->dtype, l.plan, t, static_cast<unsigned char*>(Y) + r * es, ldy, reinterpret_cast<float*>(ws + l.parts), s);
            }
        });
    });
}

int64_t idkm_codes_linear_backward_workspace(const idkm_codes_desc* w, int64_t n) {
    idkm_status st;
    if (wrong_layer(w, &st) || n < 0 || n > MAX_SIDE) return -1;
    if (n == 0) return 0;
    return grad_layout(*w, n).bytes;
}

idkm_status idkm_codes_linear_backward(idkm_ctx* ctx, const idkm_codes_desc* w, const void* X, int64_t ldx, const void* dY, int64_t lddy,
                                       int64_t n, void* dX, int64_t lddx, float* dC, float* dS, void* workspace, int64_t workspace_bytes,
                                       void* hip_stream) {
    return entry(ctx, [&]() -> idkm_status {
        idkm_status st;
        if (const char* e = wrong_layer(w, &st)) return refuse(ctx, st, e);
        if (n < 0) return refuse(ctx, IDKM_ERR_INVALID_ARG, "n must be >= 0");
        if (n > MAX_SIDE) return refuse(ctx, IDKM_ERR_UNSUPPORTED, "too many tokens");
        if (dS && !w->S) return refuse(ctx, IDKM_ERR_INVALID_ARG, "dS of a layer without scales");
        if (!aligned_to(dC, 4) || !aligned_to(dS, 4)) return refuse(ctx, IDKM_ERR_INVALID_ARG, "dC and dS must be aligned to their type");
        hipStream_t s = (hipStream_t)hip_stream;
        const int es = esize_of(w->dtype), groups = groups_of(*w);
        if (n == 0)
            return launched(ctx, [&] {
                if (dC) launch_fill_zero(dC, (int64_t)w->k * w->d, s);
                if (dS) launch_fill_zero(dS, w->rows * groups, s);
            });
        const bool layer = dC || dS;
        if (!dX && !layer) return IDKM_OK;
        if (!dY || lddy < w->rows) return refuse(ctx, IDKM_ERR_INVALID_ARG, "dY must be non-NULL and lddy >= rows");
        if (layer && (!X || ldx < w->cols)) return refuse(ctx, IDKM_ERR_INVALID_ARG, "X must be non-NULL and ldx >= cols");
        if (dX && lddx < w->cols) return refuse(ctx, IDKM_ERR_INVALID_ARG, "lddx must be >= cols");
        if (!aligned_to(dY, es) || !aligned_to(X, es) || !aligned_to(dX, es))
            return refuse(ctx, IDKM_ERR_INVALID_ARG, "X, dY and dX must be aligned to their type");
        const GradLayout g = grad_layout(*w, n);
        const bool together = g.together && dX && layer;
        if (const char* e = wrong_workspace(workspace, workspace_bytes, g.bytes)) return refuse(ctx, IDKM_ERR_INVALID_ARG, e);
        unsigned char* ws = static_cast<unsigned char*>(workspace);
        return launched(ctx, [&] {
            const ProductLayout& d = g.d;
            const LayerGradLayout& l = g.l;
            TileArgs td{};
            OperandArgs copies{};
            if (dX) operand_of(w->dtype, dY, lddy, n, w->rows, d, ws, &td, &copies);
            unsigned char* of_x = ws;
            ws += d.bytes;
            if (layer) {
                add_operand(&copies, dY, lddy, n, w->rows, ws + l.dy, l.pad, true);
                add_operand(&copies, X, ldx, n, w->cols, ws + l.x, l.pad, true);
            }
            launch_operands(w->dtype, copies, s);
            if (dX) {
                for (int64_t c = 0; c < w->cols; c += d.panel) {
                    DenseArgs a = dense_of(*w);
                    a.first = c;
                    a.count = w->cols - c < d.panel ? w->cols - c : d.panel;
                    a.pad = d.pad;
                    a.out = of_x + d.matrix;
                    launch_dense_cols(w->dtype, a, s);
                    td.N = a.count;
                    float* parts = reinterpret_cast<float*>(of_x + d.parts);
                    if (together) set_out(d.plan, &td, dX, lddx, parts);
                    else run_product(w->dtype, d.plan, td, static_cast<unsigned char*>(dX) + c * es, lddx, parts, s);
                }
            }
            if (!layer) return;
            float* bins = reinterpret_cast<float*>(ws + l.bins);
            int64_t written = 0;
            for (int64_t r = 0; r < w->rows; r += l.panel) {
                const int64_t count = w->rows - r < l.panel ? w->rows - r : l.panel;
                TileArgs t{};
                t.A = ws + l.dy + r * l.pad * es;
                t.lda = l.pad;
                t.M = count;
                t.B = ws + l.x;
                t.ldb = l.pad;
                t.N = w->cols;
                t.steps = (int)(l.pad * es / TP_STEP);
                t.wide = 1;
                t.out = ws + l.p;
                t.ldo = l.ldp;
                if (!together) {
                    run_tiles(w->dtype, l.plan, t, s);
                } else {
                    if ((td.steps + d.plan.parts - 1) / d.plan.parts > (t.steps + l.plan.parts - 1) / l.plan.parts)
                        run_tiles(w->dtype, d.plan, td, s, &l.plan, &t);
                    else
                        run_tiles(w->dtype, l.plan, t, s, &d.plan, &td);
                    if (d.plan.parts > 1)
                        launch_join_parts(w->dtype, reinterpret_cast<const float*>(of_x + d.parts), d.plan.parts, n, w->cols, dX, lddx, s);
                }
                if (l.plan.parts > 1)
                    launch_join_parts(IDKM_F32, reinterpret_cast<const float*>(ws + l.p), l.plan.parts, count, l.ldp, ws + l.p, l.ldp, s);
                BinArgs b{};
                b.words = w->words;
                b.nwords = idkm_code_words(w->rows * w->cols / w->d, w->k);
                b.rows = w->rows;
                b.cols = w->cols;
                b.C = w->C;
                b.k = w->k;
                b.d = w->d;
                b.bits = idkm_code_bits(w->k);
                b.S = w->S;
                b.group = l.group;
                b.groups = l.groups;
                b.P = reinterpret_cast<const float*>(ws + l.p);
                b.ldp = l.ldp;
                b.run = l.run;
                b.pitch = l.panels * l.grid;
                b.at = written;
                b.first = r;
                b.count = count;
                b.lanes = l.lanes;
                b.bins = dC ? bins : nullptr;
                b.segments = l.segmented && dS ? reinterpret_cast<float*>(ws + l.segments) : nullptr;
                if (l.runs) {
                    b.dS = dS;
                    launch_codes_bins_runs(w->dtype, b, l.wide, l.grid, l.waves, s);
                }
                for (int c0 = 0; !l.runs && c0 < (dC ? w->k : 1); c0 += l.codes) {
                    b.dS = c0 == 0 ? dS : nullptr;
                    b.code0 = c0;
                    b.codes = l.codes;
                    launch_codes_bins(w->dtype, b, l.grid, l.waves, s);
                }
                written += l.grid;
            }
            launch_join_gradients(bins, written, w->k * w->d, dC, l.segmented && dS ? reinterpret_cast<const float*>(ws + l.segments) : nullptr, w->rows,
                                  w->cols, l.group, l.groups, dS, s);
        });
    });
}

idkm_status idkm_group_scale(idkm_ctx* ctx, const float* W, int64_t rows, int64_t cols, int64_t group, float* S_out, float* Z_out,
                             void* hip_stream) {
    return entry(ctx, [&]() -> idkm_status {
        if (const char* e = wrong_scale_shape(rows, cols, group)) return refuse(ctx, IDKM_ERR_INVALID_ARG, e);
        if (rows == 0) return IDKM_OK;
        if (!W || !S_out || !Z_out) return refuse(ctx, IDKM_ERR_INVALID_ARG, "W, S_out and Z_out must be non-NULL");
        ScaleArgs a = scale_args(rows, cols, group);
        a.x = W;
        a.out = Z_out;
        a.s_out = S_out;
        return launched(ctx, [&] { launch_group_scale(SCALE_FWD, a, (hipStream_t)hip_stream); });
    });
}

idkm_status idkm_group_unscale(idkm_ctx* ctx, const float* Zq, const float* S, int64_t rows, int64_t cols, int64_t group, float* Wq_out,
                               void* hip_stream) {
    return entry(ctx, [&]() -> idkm_status {
        if (const char* e = wrong_scale_shape(rows, cols, group)) return refuse(ctx, IDKM_ERR_INVALID_ARG, e);
        if (rows == 0) return IDKM_OK;
        if (!Zq || !S || !Wq_out) return refuse(ctx, IDKM_ERR_INVALID_ARG, "Zq, S and Wq_out must be non-NULL");
        ScaleArgs a = scale_args(rows, cols, group);
        a.x = Zq;
        a.S = S;
        a.out = Wq_out;
        return launched(ctx, [&] { launch_group_scale(UNSCALE_FWD, a, (hipStream_t)hip_stream); });
    });
}

idkm_status idkm_group_unscale_backward(idkm_ctx* ctx, const float* dWq, const float* Zq, const float* S, int64_t rows, int64_t cols,
                                        int64_t group, float* dZq_out, float* dS_out, void* hip_stream) {
    return entry(ctx, [&]() -> idkm_status {
        if (const char* e = wrong_scale_shape(rows, cols, group)) return refuse(ctx, IDKM_ERR_INVALID_ARG, e);
        if (rows == 0) return IDKM_OK;
        if (!dWq || !Zq || !S || !dZq_out || !dS_out)
            return refuse(ctx, IDKM_ERR_INVALID_ARG, "dWq, Zq, S, dZq_out and dS_out must be non-NULL");
        ScaleArgs a = scale_args(rows, cols, group);
        a.x = dWq;
        a.y = Zq;
        a.S = S;
        a.out = dZq_out;
        a.s_out = dS_out;
        return launched(ctx, [&] { launch_group_scale(UNSCALE_BWD, a, (hipStream_t)hip_stream); });
    });
}

idkm_status idkm_group_scale_backward(idkm_ctx* ctx, const float* Z, const float* S, const float* dZ, const float* dS, int64_t rows,
                                      int64_t cols, int64_t group, float* dW_out, void* hip_stream) {
    return entry(ctx, [&]() -> idkm_status {
        if (const char* e = wrong_scale_shape(rows, cols, group)) return refuse(ctx, IDKM_ERR_INVALID_ARG, e);
        if (rows == 0) return IDKM_OK;
        if (!Z || !S || !dZ || !dW_out) return refuse(ctx, IDKM_ERR_INVALID_ARG, "Z, S, dZ and dW_out must be non-NULL");
        ScaleArgs a = scale_args(rows, cols, group);
        a.x = dZ;
        a.y = Z;
        a.S = S;
        a.dS = dS;
        a.out = dW_out;
        return launched(ctx, [&] { launch_group_scale(SCALE_BWD, a, (hipStream_t)hip_stream); });
    });
}

int64_t idkm_distill_workspace(int64_t n, int64_t V, int32_t top, int32_t dtype) {
    if (n < 0 || V < 1 || top < 1 || top > 1024 || dtype < 0 || dtype > 2 || n > INT_MAX || V > MAX_VOCABULARY) return -1;
    if (n == 0) return 0;
    int64_t part;
    int parts;
    distill_plan(n, V, esize_of(dtype), &part, &parts);
    return parts == 0 ? 0 : buffer(n * parts * 2, 4) + buffer(n * top, 4);
}

idkm_status idkm_distill(idkm_ctx* ctx, const void* logits, int64_t n, int64_t V, int64_t ldz, idkm_dtype dtype, const int32_t* index,
                         const float* teacher, int32_t top, float tau, const float* weight, float* loss_out, float* lse_out,
                         void* dlogits_out, int64_t ldd, void* workspace, int64_t workspace_bytes, void* hip_stream) {
    return entry(ctx, [&]() -> idkm_status {
        if (dtype != IDKM_F32 && dtype != IDKM_F16 && dtype != IDKM_BF16) return refuse(ctx, IDKM_ERR_INVALID_ARG, "dtype must be an idkm_dtype");
        if (n < 0 || V < 1) return refuse(ctx, IDKM_ERR_INVALID_ARG, "need n >= 0 and V >= 1");
        if (n > INT_MAX || V > MAX_VOCABULARY) return refuse(ctx, IDKM_ERR_UNSUPPORTED, "need n < 2^31 and V <= 2^29");
        if (top < 1 || top > 1024) return refuse(ctx, IDKM_ERR_INVALID_ARG, "need 1 <= top <= 1024");
        if (!(tau >= FLT_MIN) || !std::isfinite(tau))  // of a smaller one the inverse is infinite
            return refuse(ctx, IDKM_ERR_INVALID_ARG, "tau must be finite and > 0, and not subnormal");
        if ((weight != nullptr) != (dlogits_out != nullptr))
            return refuse(ctx, IDKM_ERR_INVALID_ARG, "weight and dlogits_out go together");
        if (n == 0) return IDKM_OK;
        if (!logits || !index || !teacher || !loss_out || !lse_out)
            return refuse(ctx, IDKM_ERR_INVALID_ARG, "logits, index, teacher, loss_out and lse_out must be non-NULL");
        if (ldz < V || (dlogits_out && ldd < V)) return refuse(ctx, IDKM_ERR_INVALID_ARG, "ldz and ldd must be >= V");
        const int es = esize_of(dtype);
        if (!aligned_to(logits, es) || !aligned_to(dlogits_out, es))
            return refuse(ctx, IDKM_ERR_INVALID_ARG, "logits and dlogits_out must be aligned to their type");
        if (dlogits_out == logits && ldd != ldz) return refuse(ctx, IDKM_ERR_INVALID_ARG, "in place, ldd must be ldz");
        DistillArgs a{};
        a.logits = logits;
        a.n = n;
        a.V = V;
        a.ldz = ldz;
        a.index = index;
        a.teacher = teacher;
        a.top = top;
        a.tau = tau;
        a.weight = weight;
        a.loss = loss_out;
        a.lse = lse_out;
        a.dlogits = dlogits_out;
        a.ldd = ldd;
        distill_plan(n, V, es, &a.part, &a.parts);
        if (const char* e = wrong_workspace(workspace, workspace_bytes, idkm_distill_workspace(n, V, top, dtype)))
            return refuse(ctx, IDKM_ERR_INVALID_ARG, e);
        a.stats = static_cast<float*>(workspace);
        if (a.parts > 0) a.listed = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + buffer(n * a.parts * 2, 4));
        return launched(ctx, [&] { launch_distill(dtype, a, (hipStream_t)hip_stream); });
    });
}

}  // extern "C"

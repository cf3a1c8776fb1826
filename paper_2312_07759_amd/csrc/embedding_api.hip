// C entry points of the lookups of tokens' rows in float32 and stored tables and of their gradients.
#include <climits>
#include <cmath>

#include "embedding.h"
#include "entry.hpp"

using namespace idkm;

namespace {

idkm_status wrong_tokens(idkm_ctx* ctx, const void* ids, int32_t id_bytes, int64_t n, float alpha) {
    if (id_bytes != 4 && id_bytes != 8) return refuse(ctx, IDKM_ERR_INVALID_ARG, "id_bytes must be 4 or 8");
    if (n < 0) return refuse(ctx, IDKM_ERR_INVALID_ARG, "n must be >= 0");
    if (n > MAX_SIDE) return refuse(ctx, IDKM_ERR_UNSUPPORTED, "too many tokens");
    if (!std::isfinite(alpha)) return refuse(ctx, IDKM_ERR_INVALID_ARG, "alpha must be finite");
    if (n > 0 && (!ids || !aligned_to(ids, (size_t)id_bytes))) return refuse(ctx, IDKM_ERR_INVALID_ARG, "ids must be non-NULL and aligned to their type");
    return IDKM_OK;
}

idkm_status wrong_table(idkm_ctx* ctx, int64_t rows, int64_t cols, int dtype) {
    if (dtype != IDKM_F32 && dtype != IDKM_F16 && dtype != IDKM_BF16) return refuse(ctx, IDKM_ERR_INVALID_ARG, "dtype must be an idkm_dtype");
    if (rows < 1 || cols < 1) return refuse(ctx, IDKM_ERR_INVALID_ARG, "rows and cols must be >= 1");
    if (rows > MAX_SIDE || cols > MAX_SIDE || rows * cols > ((int64_t)1 << 36)) return refuse(ctx, IDKM_ERR_UNSUPPORTED, "the table is too large");
    return IDKM_OK;
}

idkm_status wrong_side(idkm_ctx* ctx, const void* y, int64_t ld, int64_t cols, int dtype) {
    if (!y || ld < cols) return refuse(ctx, IDKM_ERR_INVALID_ARG, "Y and dY must be non-NULL and their rows at least cols apart");
    if (!aligned_to(y, (size_t)esize_of(dtype))) return refuse(ctx, IDKM_ERR_INVALID_ARG, "Y and dY must be aligned to their type");
    return IDKM_OK;
}

TokenIds tokens_of(const void* ids, int32_t id_bytes, int64_t n, int64_t rows) { return TokenIds{ids, id_bytes == 8, n, (int)rows}; }

SumArgs sums_of(const TokenOrder& order, int64_t n, int64_t rows, float alpha, const void* dY, int64_t ldy, int64_t cols) {
    SumArgs a{};
    a.order = order;
    a.n = n;
    a.rows = (int)rows;
    a.alpha = alpha;
    a.dY = dY;
    a.ldy = ldy;
    a.cols = cols;
    return a;
}

// Workspace of a stored table's gradient.  direct: see lookup_gradient.hpp; the others sum the rows first.
struct CodesGradLayout : BinPlan {
    bool direct;
    LookupGradPlan plan;
    int per_part;
    int64_t lines, ldp, order, index, partial, p, bins, segments, bytes;
};

CodesGradLayout codes_grad_layout(const idkm_codes_desc& w, int64_t n) {
    CodesGradLayout l{};
    l.lines = n < w.rows ? n : w.rows;  // different rows, at most
    static_cast<BinPlan&>(l) = bin_plan(w, l.lines);
    l.order = 0;
    // Many strips of 512 columns and a large codebook: the turns of lanes with the same bins take longer than sums written out and read again.  k = 256, d = 8,
    // bfloat16, scales of groups of 128: 2000 tokens of 2048 columns 50.5 us in one pass and 53, 8192 of 4096 146 and 125; d = 4, half the components: 38.5
    // and 51.5, 120 and 123.
    l.direct = l.runs && w.cols >= 8 && (w.k * w.d <= 1024 || n * ((w.cols + 511) / 512) <= 16384);
    if (l.direct) {
        l.plan = lookup_grad_plan(n, w.cols, esize_of(w.dtype), w.k * w.d);
        l.segmented = w.S && (l.group > 512 || l.group % 8 != 0 || (l.group & (l.group - 1)) != 0);
        l.per_part = w.S ? l.segmented ? (int)((w.cols + 31) / 32) : l.groups : 0;
        l.bins = buffer(sort_words(n), 4);
        l.segments = l.bins + buffer((int64_t)l.plan.grid * w.k * w.d, 4);
        l.bytes = l.segments + buffer(n * l.per_part, 4);
        return l;
    }
    l.ldp = up_to(w.cols, 8);
    l.index = buffer(sort_words(n), 4);
    l.partial = l.index + buffer(2 * n + 1, 4);
    l.p = l.partial + buffer(sum_partials(n, w.cols), 4);
    l.bins = l.p + buffer(l.lines * l.ldp, 4);
    l.segments = l.bins + buffer((int64_t)l.grid * w.k * w.d, 4);
    l.bytes = l.segments + (l.segmented ? buffer(l.lines * ((w.cols + 31) / 32), 4) : 0);
    return l;
}

}  // namespace

extern "C" {

idkm_status idkm_embedding(idkm_ctx* ctx, const float* W, int64_t rows, int64_t cols, const void* ids, int32_t id_bytes, int64_t n, float alpha,
                           void* Y, int64_t ldy, idkm_dtype dtype, void* hip_stream) {
    return entry(ctx, [&]() -> idkm_status {
        if (idkm_status st = wrong_table(ctx, rows, cols, dtype)) return st;
        if (idkm_status st = wrong_tokens(ctx, ids, id_bytes, n, alpha)) return st;
        if (n == 0) return IDKM_OK;
        if (!W || !aligned_to(W, 4)) return refuse(ctx, IDKM_ERR_INVALID_ARG, "W must be non-NULL and aligned to its type");
        if (idkm_status st = wrong_side(ctx, Y, ldy, cols, dtype)) return st;
        LookupArgs a{};
        a.ids = tokens_of(ids, id_bytes, n, rows);
        a.alpha = alpha;
        a.cols = cols;
        a.Y = Y;
        a.ldy = ldy;
        a.W = W;
        return launched(ctx, [&] { launch_lookup_table(dtype, a, (hipStream_t)hip_stream); });
    });
}

int64_t idkm_embedding_backward_workspace(int64_t rows, int64_t cols, int64_t n) {
    if (rows < 1 || cols < 1 || n < 0 || rows > MAX_SIDE || cols > MAX_SIDE || n > MAX_SIDE || rows * cols > ((int64_t)1 << 36)) return -1;
    if (n <= FEW_TOKENS) return 0;
    return buffer(sort_words(n), 4) + buffer(sum_partials(n, cols), 4);
}

idkm_status idkm_embedding_backward(idkm_ctx* ctx, int64_t rows, int64_t cols, const void* ids, int32_t id_bytes, int64_t n, float alpha,
                                    const void* dY, int64_t lddy, idkm_dtype dtype, float* dW, void* workspace, int64_t workspace_bytes,
                                    void* hip_stream) {
    return entry(ctx, [&]() -> idkm_status {
        if (idkm_status st = wrong_table(ctx, rows, cols, dtype)) return st;
        if (idkm_status st = wrong_tokens(ctx, ids, id_bytes, n, alpha)) return st;
        if (!dW || !aligned_to(dW, 4)) return refuse(ctx, IDKM_ERR_INVALID_ARG, "dW must be non-NULL and aligned to its type");
        if (n > 0)
            if (idkm_status st = wrong_side(ctx, dY, lddy, cols, dtype)) return st;
        if (const char* e = wrong_workspace(workspace, workspace_bytes, idkm_embedding_backward_workspace(rows, cols, n)))
            return refuse(ctx, IDKM_ERR_INVALID_ARG, e);
        hipStream_t s = (hipStream_t)hip_stream;
        unsigned char* ws = static_cast<unsigned char*>(workspace);
        return launched(ctx, [&] {
            const TokenIds tokens = tokens_of(ids, id_bytes, n, rows);
            if (n <= FEW_TOKENS) {
                if (n == 0) launch_fill_zero(dW, rows * cols, s);
                else launch_sums_of_few(dtype, tokens, alpha, dY, lddy, cols, dW, s);
                return;
            }
            const TokenOrder order = launch_sort(tokens, reinterpret_cast<int32_t*>(ws), dW, rows * cols, s);
            SumArgs a = sums_of(order, n, rows, alpha, dY, lddy, cols);
            a.out = dW;
            a.ldo = cols;
            a.partial = reinterpret_cast<float*>(ws + buffer(sort_words(n), 4));
            launch_sums(dtype, a, s);
        });
    });
}

idkm_status idkm_codes_embedding(idkm_ctx* ctx, const idkm_codes_desc* w, const void* ids, int32_t id_bytes, int64_t n, float alpha, void* Y,
                                 int64_t ldy, void* hip_stream) {
    return entry(ctx, [&]() -> idkm_status {
        idkm_status st;
        if (const char* e = wrong_layer(w, &st)) return refuse(ctx, st, e);
        if ((st = wrong_tokens(ctx, ids, id_bytes, n, alpha))) return st;
        if (n == 0) return IDKM_OK;
        if ((st = wrong_side(ctx, Y, ldy, w->cols, w->dtype))) return st;
        LookupArgs a{};
        a.ids = tokens_of(ids, id_bytes, n, w->rows);
        a.alpha = alpha;
        a.cols = w->cols;
        a.Y = Y;
        a.ldy = ldy;
        a.words = w->words;
        a.nwords = idkm_code_words(w->rows * w->cols / w->d, w->k);
        a.C = w->C;
        a.k = w->k;
        a.d = w->d;
        a.bits = idkm_code_bits(w->k);
        a.row_bits = w->cols / w->d * a.bits;
        a.S = w->S;
        a.groups = groups_of(*w);
        a.group = w->S ? (w->group < w->cols ? w->group : (int)w->cols) : 1;
        return launched(ctx, [&] { launch_lookup_codes(w->dtype, a, (hipStream_t)hip_stream); });
    });
}

int64_t idkm_codes_embedding_backward_workspace(const idkm_codes_desc* w, int64_t n) {
    idkm_status st;
    if (wrong_layer(w, &st) || n < 0 || n > MAX_SIDE) return -1;
    if (n == 0) return 0;
    return codes_grad_layout(*w, n).bytes;
}

idkm_status idkm_codes_embedding_backward(idkm_ctx* ctx, const idkm_codes_desc* w, const void* ids, int32_t id_bytes, int64_t n, float alpha,
                                          const void* dY, int64_t lddy, float* dC, float* dS, void* workspace, int64_t workspace_bytes,
                                          void* hip_stream) {
    return entry(ctx, [&]() -> idkm_status {
        idkm_status st;
        if (const char* e = wrong_layer(w, &st)) return refuse(ctx, st, e);
        if ((st = wrong_tokens(ctx, ids, id_bytes, n, alpha))) return st;
        if (dS && !w->S) return refuse(ctx, IDKM_ERR_INVALID_ARG, "dS of a table without scales");
        if (!aligned_to(dC, 4) || !aligned_to(dS, 4)) return refuse(ctx, IDKM_ERR_INVALID_ARG, "dC and dS must be aligned to their type");
        if (!dC && !dS) return IDKM_OK;
        if (n > 0 && (st = wrong_side(ctx, dY, lddy, w->cols, w->dtype))) return st;
        const CodesGradLayout l = codes_grad_layout(*w, n > 0 ? n : 1);
        if (const char* e = wrong_workspace(workspace, workspace_bytes, n > 0 ? l.bytes : 0)) return refuse(ctx, IDKM_ERR_INVALID_ARG, e);
        hipStream_t s = (hipStream_t)hip_stream;
        unsigned char* ws = static_cast<unsigned char*>(workspace);
        return launched(ctx, [&] {
            const int64_t scales = dS ? w->rows * groups_of(*w) : 0;
            if (n == 0) {
                if (dS) launch_fill_zero(dS, scales, s);
                if (dC) launch_fill_zero(dC, (int64_t)w->k * w->d, s);
                return;
            }
            const TokenIds tokens = tokens_of(ids, id_bytes, n, w->rows);
            int32_t* sorted = reinterpret_cast<int32_t*>(ws);
            const BinArgs bins = bins_of(*w, l);
            if (l.direct) {
                LookupGradArgs a{};
                a.ids = tokens;
                a.order = l.plan.few ? TokenOrder{sorted, nullptr} : launch_sort(tokens, sorted, dS, scales, s);
                a.alpha = alpha;
                a.dY = dY;
                a.ldy = lddy;
                a.cols = (int)w->cols;
                a.words = w->words;
                a.nwords = bins.nwords;
                a.row_bits = w->cols / w->d * bins.bits;
                a.C = w->C;
                a.k = w->k;
                a.bits = bins.bits;
                a.S = w->S;
                a.group = l.group;
                a.groups = l.groups;
                a.dS = dS;
                a.parts = reinterpret_cast<float*>(ws + l.segments);
                a.per_part = l.per_part;
                a.segmented = l.segmented;
                a.bins = reinterpret_cast<float*>(ws + l.bins);
                a.pitch = l.plan.grid;
                a.few = l.plan.few;
                a.each = l.plan.each;
                launch_lookup_gradient(w->dtype, w->d, l.plan, a, s);
                // segments of a group; one where a part has a sum for each
                launch_join_lookup(l.plan, a, w->k * w->d, dC, !l.segmented ? 1 : l.groups > 1 ? l.group / 32 : l.per_part, s);
                return;
            }
            const TokenOrder order = launch_sort(tokens, sorted, dS, scales, s);
            int32_t* index = reinterpret_cast<int32_t*>(ws + l.index);
            const RowsOfTokens rows{index, index + n, index + 2 * n};
            launch_rows(order, n, (int)w->rows, rows, s);
            float* P = reinterpret_cast<float*>(ws + l.p);
            SumArgs a = sums_of(order, n, w->rows, alpha, dY, lddy, w->cols);
            a.index_at = rows.index_at;
            a.out = P;
            a.ldo = l.ldp;
            a.partial = reinterpret_cast<float*>(ws + l.partial);
            launch_sums(w->dtype, a, s);
            BinArgs b = bins;
            b.P = P;
            b.ldp = l.ldp;
            b.pitch = l.grid;
            b.listed = rows.row_of;
            b.listed_count = rows.count;
            b.bins = dC ? reinterpret_cast<float*>(ws + l.bins) : nullptr;
            b.segments = l.segmented && dS ? reinterpret_cast<float*>(ws + l.segments) : nullptr;
            run_bins(w->dtype, l, b, dS, s);
            launch_join_gradients(b.bins, l.grid, w->k * w->d, dC, b.segments, l.lines, w->cols, l.group, l.groups, dS, s, rows.row_of, rows.count);
        });
    });
}

}  // extern "C"

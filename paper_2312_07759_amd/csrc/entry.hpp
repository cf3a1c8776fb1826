// What the C entry points of the operators on layers share: checks of arguments, errors, the context's device.
#pragma once
#include <cstdint>
#include <exception>
#include <new>

#include "../../include/idkm.h"
#include "layers.h"

namespace idkm {

int context_device(const idkm_ctx* ctx);
void context_error(idkm_ctx* ctx, const char* msg);

constexpr int64_t MAX_SIDE = 4000000;  // rows, columns, tokens: 64 of them to a workgroup fit one grid dimension

inline idkm_status refuse(idkm_ctx* ctx, idkm_status s, const char* msg) {
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

inline int esize_of(int dtype) { return dtype == IDKM_F32 ? 4 : dtype == TP_INT8 ? 1 : 2; }
inline bool aligned_to(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

inline const char* wrong_layer(const idkm_codes_desc* w, idkm_status* st) {
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

inline int groups_of(const idkm_codes_desc& w) { return w.S ? (int)((w.cols + w.group - 1) / w.group) : 0; }

inline const char* wrong_workspace(const void* ws, int64_t have, int64_t need) {
    if (need == 0) return nullptr;
    if (!ws || have < need) return "the workspace is smaller than the size asked for";
    if (!aligned_to(ws, 16)) return "the workspace must be 16-byte aligned";
    return nullptr;
}

// Which of the kernels for bins, and its launch, for `lines` rows of a layer.
struct BinPlan {
    bool runs, wide, segmented;
    int group, groups, lanes, run, waves, codes, grid;
};
BinPlan bin_plan(const idkm_codes_desc& w, int64_t lines);
BinArgs bins_of(const idkm_codes_desc& w, const BinPlan& l);
void run_bins(int dtype, const BinPlan& l, BinArgs b, float* dS, hipStream_t s);

// Bytes of a buffer in the workspace.
inline int64_t buffer(int64_t elements, int esize) { return up_to(elements * esize, 256); }

}  // namespace idkm

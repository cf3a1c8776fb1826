// Host-side lookup of the kernels for coded layers, group scales and the loss against a teacher, and their arguments.
#pragma once
#include "codes_gradient.hpp"
#include "codes_product.hpp"
#include "tile_product.hpp"

// T is the type that dtype names.
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

namespace idkm {

inline int64_t up_to(int64_t x, int64_t unit) { return (x + unit - 1) / unit * unit; }

// Up to 16 tokens, straight from the codes.  IB bits looked up at once give W weights (see codes_at_once), L weights of a row to a
// lane at a time (8, 16, 32); aligned: every run of codes begins with a word; apart: up to 4 tokens, L = 32, a scale for every run.
// nullptr if not instantiated.
typedef void (*ProductFn)(const ProductArgs);
ProductFn codes_product_kernel(int dtype, int IB, int W, int L, bool aligned, bool apart);
// 17 tokens and more, 16 NT of them at a time (NT in {2, 4}).
ProductFn codes_tile_kernel(int dtype, int IB, int W, int L, int NT, bool aligned);

// A layer written out, codes looked up as above; columns: its transpose; aligned: eight columns' codes begin with a word.
typedef void (*DenseFn)(const DenseArgs);
DenseFn codes_dense_kernel(int dtype, int IB, int W, bool columns, bool aligned);

struct TileShape {
    int bm, bn, threads;
    size_t lds;
    void (*fn)(const TileJobs);
    int resident;  // workgroups that the device holds at once
    float us;      // of a step of all of them
};
constexpr int TP_INT8 = 3;  // beside idkm_dtype's
// The shapes of a type's tile product, from 0 on; fn = nullptr behind the last.  scaled: SC of k_tile_product, 16-bit types only.
TileShape tile_shape(int dtype, int which, int scaled);

void launch_dense_rows(int dtype, const DenseArgs& a, hipStream_t s);
// also: operands to bring, in the same launch or in one before it
void launch_dense_cols(int dtype, const DenseArgs& a, hipStream_t s, const OperandArgs& also);
void allow_lds(const void* fn, size_t bytes);  // before a launch of fn with so much dynamic LDS
// Up to three operands to a launch.
void add_operand(OperandArgs* a, const void* in, int64_t ldi, int64_t M, int64_t N, void* out, int64_t pad, bool transposed,
                 const uint8_t* E = nullptr, const float* scale = nullptr);
void launch_operands(int dtype, const OperandArgs& a, hipStream_t s);
// by_m: factors [M] of the rows, or null.
void launch_join_parts(int dtype, const float* parts, int nz, int64_t M, int64_t N, void* out, int64_t ldo, hipStream_t s, const float* by_m = nullptr);
void launch_codes_bins(int dtype, const BinArgs& a, int grid, int waves, hipStream_t s);
int bins_shared_by(int k);
void launch_codes_bins_runs(int dtype, const BinArgs& a, bool wide, int grid, int waves, hipStream_t s);
void launch_fill_zero(float* out, int64_t n, hipStream_t s);
// dC from bins [kd][n] (null: not), dS from segments (null: not); listed, listed_count: see BinArgs, `rows` at most then.
void launch_join_gradients(const float* bins, int64_t n, int kd, float* dC, const float* segments, int64_t rows, int64_t cols, int group,
                           int groups, float* dS, hipStream_t s, const int32_t* listed = nullptr, const int32_t* listed_count = nullptr);

void launch_keep8(int dtype, const KeepArgs& a, hipStream_t s);
void launch_restore8(int dtype, const KeepArgs& a, hipStream_t s);

// Rows in 8-bit integers: Q [n, ldq], zero behind column cols, and their scales.
struct Int8RowsArgs {
    const void* X;  // T [n, ldx]
    int64_t n, cols, ldx;
    int8_t* Q;
    int64_t ldq;  // a multiple of 16
    float* scale;
};
void launch_int8_rows(int dtype, const Int8RowsArgs& a, hipStream_t s);

// Up to a few dozen tokens times a layer of 8-bit integers.
struct Int8FewArgs {
    const int8_t* W8;  // [rows, ldw]
    int64_t rows, ldw;
    const float* scale;  // [rows]
    const int8_t* Q;     // [n, pad], or null: X itself is brought to integers by every workgroup
    const float* q_scale;
    const void* X;  // T [n, ldx]
    int64_t cols, pad, ldx, n;  // pad: cols in whole steps of 128, Q's rows
    void* Y;  // T [n, ldy]
    int64_t ldy;
};
constexpr int64_t INT8_FUSED = 4 * 8192;  // elements of X, in whole steps of 128 columns, that a workgroup brings to integers itself, at most
void launch_int8_few(int dtype, const Int8FewArgs& a, hipStream_t s);
// Operands of the gradient of a product, float32: dY times the scales in three parts of 16 bits, and columns of W8 in 16 bits; float16: the same in one part,
// every token divided by a power of two.
struct Int8SplitArgs {
    const void* dY;  // T [n, ldy]
    int64_t n, ldy, rows;
    const float* scale;  // [rows]
    const int8_t* W8;    // [rows, ldw], from the first column that is wanted on
    int64_t ldw, cols;
    void* A;      // bf16 [3, n, pad] or f16 [n, pad], zero behind column `rows`
    void* B;      // [cols, pad], A's type
    int64_t pad;  // a multiple of 64
    float* by;    // float16: [n], the powers of two
    unsigned splitting;  // workgroups, set by the launch
};
void launch_int8_split(const Int8SplitArgs& a, bool dY, hipStream_t s);  // dY: A too, or B alone
void launch_int8_half(const Int8SplitArgs& a, bool dY, hipStream_t s);   // .. of float16
// out[M, N] in the type of dtype = by_m by_n times the sum of the parts [nz][M, N].
void launch_join_int8(int dtype, const int32_t* parts, int nz, int64_t M, int64_t N, const float* by_m, const float* by_n, void* out, int64_t ldo,
                      hipStream_t s);

constexpr int SCALE_FWD = 0, UNSCALE_FWD = 1, UNSCALE_BWD = 2, SCALE_BWD = 3;
struct ScaleArgs {
    int64_t rows, cols, group, groups;
    const float* x;   // W, Zq, dWq, dZ
    const float* y;   // UNSCALE_BWD: Zq, SCALE_BWD: Z
    const float* S;   // all but SCALE_FWD
    const float* dS;  // SCALE_BWD, or null
    float* out;       // Z, Wq, dZq, dW
    float* s_out;     // SCALE_FWD: S, UNSCALE_BWD: dS
};
void launch_group_scale(int op, const ScaleArgs& a, hipStream_t s);

struct DistillArgs {
    const void* logits;  // T [n, ldz]
    int64_t n, V, ldz;
    const int32_t* index;  // [n, top]
    const float* teacher;  // [n, top]
    int top;
    float tau;
    const float* weight;  // [n] or null
    float* loss;          // [n]
    float* lse;           // [n]
    void* dlogits;        // T [n, ldd] or null
    int64_t ldd;
    int64_t part;   // columns of a part
    int parts;      // workgroups that share a row; 0: a row stays in one
    float* stats;   // [n, parts, 2]
    float* listed;  // [n, top]
};
void distill_plan(int64_t n, int64_t V, int esize, int64_t* part, int* parts);
void launch_distill(int dtype, const DistillArgs& a, hipStream_t s);

}  // namespace idkm

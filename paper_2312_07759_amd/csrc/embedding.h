// Host-side launches of the lookups in tables, stored and float32, and of their gradients.
#pragma once
#include "codes_gradient.hpp"
#include "lookup_gradient.hpp"

namespace idkm {

struct LookupArgs {
    TokenIds ids;
    float alpha;
    int64_t cols;
    void* Y;  // T [n, ldy]
    int64_t ldy;
    const float* W;  // [rows, cols] of a float32 table; a stored one's:
    const uint32_t* words;
    int64_t nwords, row_bits;
    const void* C;  // T [k, d]
    int k, d, bits;
    const float* S;  // [rows, groups] or null
    int group, groups;
    int c_in_lds;
    int each;  // tokens of a wavefront at a time
};
void launch_lookup_table(int dtype, const LookupArgs& a, hipStream_t s);
void launch_lookup_codes(int dtype, const LookupArgs& a, hipStream_t s);

// Workspace of a sort, in int32: the order, a second one and counts where there are more than GROUP_TOKENS tokens.
int64_t sort_words(int64_t n);
// clear: `count` floats that are set to zero on the way.
TokenOrder launch_sort(const TokenIds& ids, int32_t* workspace, float* clear, int64_t count, hipStream_t s);

// The different rows among sorted tokens: index_at[p] of the row at place p, row_of[index], and their number.
struct RowsOfTokens {
    int32_t* index_at;  // [n]
    int32_t* row_of;    // [n]
    int32_t* count;     // [1]
};
void launch_rows(const TokenOrder& order, int64_t n, int rows, const RowsOfTokens& out, hipStream_t s);

// Sums of dY over the tokens of each row: out[row or its index, c] = alpha sum dY[t, c].
struct SumArgs {
    TokenOrder order;
    const int32_t* index_at;  // null: rows of `out` are the table's
    int64_t n;
    int rows;
    float alpha;
    const void* dY;  // T [n, ldy]
    int64_t ldy, cols;
    float* out;  // [.., ldo]
    int64_t ldo;
    int each;          // places to a wavefront
    float* partial;    // [2 blocks][ldp]: of runs that go on beyond their wavefront's places
    int64_t ldp;
};
// dW of a table, up to FEW_TOKENS tokens.
void launch_sums_of_few(int dtype, const TokenIds& ids, float alpha, const void* dY, int64_t ldy, int64_t cols, float* dW, hipStream_t s);

// A stored table's gradient in one pass; grid: workgroups that sum, each with a column of `bins`.
struct LookupGradPlan {
    bool few;
    int each, grid, waves, width_log;  // width_log: see LookupGradArgs
};
LookupGradPlan lookup_grad_plan(int64_t n, int64_t cols, int esize, int kd);
void launch_lookup_gradient(int dtype, int d, const LookupGradPlan& p, const LookupGradArgs& a, hipStream_t s);
// dC from bins, dS of the rows that went to `parts`; of_group: segments of a group, or 1.
void launch_join_lookup(const LookupGradPlan& p, const LookupGradArgs& a, int kd, float* dC, int of_group, hipStream_t s);
int sum_places(int64_t n, int64_t cols);
int64_t sum_partials(int64_t n, int64_t cols);  // floats
void launch_sums(int dtype, const SumArgs& a, hipStream_t s);

}  // namespace idkm

// Instantiations of the product of few tokens with codes of which CODE_BITS bits are looked up at once; included by one source
// file for each.
#include "layers.h"

namespace idkm {

template <typename T, int W, bool APART>
static ProductFn for_run(int L, bool aligned) {
    constexpr int IB = CODE_BITS;
    if constexpr (!APART) {
        if (L == 8) return &k_codes_product<T, IB, W, 8, false, false>;
        if (L == 16) return &k_codes_product<T, IB, W, 16, false, false>;
    }
    if constexpr (32 / W * IB % 32 == 0) {
        if (aligned) return &k_codes_product<T, IB, W, 32, true, APART>;
    }
    return &k_codes_product<T, IB, W, 32, false, APART>;
}

template <typename T>
static ProductFn for_type(int W, int L, bool aligned, bool apart) {
    // codes of one to four bits are looked up together until they are eight weights or five bits and more
    switch (W) {
        case 1: if constexpr (CODE_BITS >= 5) return apart ? for_run<T, 1, true>(L, aligned) : for_run<T, 1, false>(L, aligned); break;
        case 2: if constexpr (CODE_BITS >= 5) return apart ? for_run<T, 2, true>(L, aligned) : for_run<T, 2, false>(L, aligned); break;
        case 4: if constexpr (CODE_BITS >= 5) return apart ? for_run<T, 4, true>(L, aligned) : for_run<T, 4, false>(L, aligned); break;
        case 8: return apart ? for_run<T, 8, true>(L, aligned) : for_run<T, 8, false>(L, aligned);
    }
    return nullptr;
}

template <typename T, int W, int NT>
static ProductFn tile_for_run(int L, bool aligned) {
    constexpr int IB = CODE_BITS;
    if (L == 8) return &k_codes_tile<T, IB, W, 8, NT, false>;
    if (L == 16) return &k_codes_tile<T, IB, W, 16, NT, false>;
    if constexpr (32 / W * IB % 32 == 0) {
        if (aligned) return &k_codes_tile<T, IB, W, 32, NT, true>;
    }
    return &k_codes_tile<T, IB, W, 32, NT, false>;
}

template <typename T>
static ProductFn tile_for_type(int W, int L, int NT, bool aligned) {
    switch (W) {
        case 1: if constexpr (CODE_BITS >= 5) return NT == 2 ? tile_for_run<T, 1, 2>(L, aligned) : tile_for_run<T, 1, 4>(L, aligned); break;
        case 2: if constexpr (CODE_BITS >= 5) return NT == 2 ? tile_for_run<T, 2, 2>(L, aligned) : tile_for_run<T, 2, 4>(L, aligned); break;
        case 4: if constexpr (CODE_BITS >= 5) return NT == 2 ? tile_for_run<T, 4, 2>(L, aligned) : tile_for_run<T, 4, 4>(L, aligned); break;
        case 8: return NT == 2 ? tile_for_run<T, 8, 2>(L, aligned) : tile_for_run<T, 8, 4>(L, aligned);
    }
    return nullptr;
}

#define CODES_PRODUCT_NAME2(b) codes_product_kernel_##b
#define CODES_PRODUCT_NAME(b) CODES_PRODUCT_NAME2(b)
ProductFn CODES_PRODUCT_NAME(CODE_BITS)(int dtype, int W, int L, bool aligned, bool apart) {
    if (dtype == 0) return for_type<float>(W, L, aligned, apart);
    if (dtype == 1) return for_type<f16>(W, L, aligned, apart);
    return for_type<bf16>(W, L, aligned, apart);
}

#define CODES_TILE_NAME2(b) codes_tile_kernel_##b
#define CODES_TILE_NAME(b) CODES_TILE_NAME2(b)
ProductFn CODES_TILE_NAME(CODE_BITS)(int dtype, int W, int L, int NT, bool aligned) {
    if (dtype == 0) return tile_for_type<float>(W, L, NT, aligned);
    if (dtype == 1) return tile_for_type<f16>(W, L, NT, aligned);
    return tile_for_type<bf16>(W, L, NT, aligned);
}

template <typename T, int W>
static DenseFn dense_for_width(bool columns, bool aligned) {
    if constexpr (8 / W * CODE_BITS % 32 == 0) {
        if (aligned) return columns ? &k_dense_cols_fast<T, CODE_BITS, W, true> : &k_dense_rows_fast<T, CODE_BITS, W, true>;
    }
    return columns ? &k_dense_cols_fast<T, CODE_BITS, W, false> : &k_dense_rows_fast<T, CODE_BITS, W, false>;
}

template <typename T>
static DenseFn dense_for_type(int W, bool columns, bool aligned) {
    switch (W) {
        case 1: if constexpr (CODE_BITS >= 5) return dense_for_width<T, 1>(columns, aligned); break;
        case 2: if constexpr (CODE_BITS >= 5) return dense_for_width<T, 2>(columns, aligned); break;
        case 4: if constexpr (CODE_BITS >= 5) return dense_for_width<T, 4>(columns, aligned); break;
        case 8: return dense_for_width<T, 8>(columns, aligned);
    }
    return nullptr;
}

#define CODES_DENSE_NAME2(b) codes_dense_kernel_##b
#define CODES_DENSE_NAME(b) CODES_DENSE_NAME2(b)
DenseFn CODES_DENSE_NAME(CODE_BITS)(int dtype, int W, bool columns, bool aligned) {
    if (dtype == 0) return dense_for_type<float>(W, columns, aligned);
    if (dtype == 1) return dense_for_type<f16>(W, columns, aligned);
    return dense_for_type<bf16>(W, columns, aligned);
}

}  // namespace idkm

// Instantiations of the product of few tokens with codes of CODE_BITS bits; included by one source file for each.
#include "layers.h"

namespace idkm {

template <typename T, int D, int NT>
static ProductFn for_run(int L, bool aligned) {
    constexpr int B = CODE_BITS;
    if (L == 8) return &k_codes_product<T, B, D, 8, NT, false>;
    if constexpr (32 / D * B % 32 == 0) {
        if (aligned) return &k_codes_product<T, B, D, 32, NT, true>;
    }
    return &k_codes_product<T, B, D, 32, NT, false>;
}

template <typename T>
static ProductFn for_type(int d, int L, int NT, bool aligned) {
    switch (d) {
        case 1: return NT == 1 ? for_run<T, 1, 1>(L, aligned) : for_run<T, 1, 4>(L, aligned);
        case 2: return NT == 1 ? for_run<T, 2, 1>(L, aligned) : for_run<T, 2, 4>(L, aligned);
        case 4: return NT == 1 ? for_run<T, 4, 1>(L, aligned) : for_run<T, 4, 4>(L, aligned);
        case 8: return NT == 1 ? for_run<T, 8, 1>(L, aligned) : for_run<T, 8, 4>(L, aligned);
    }
    return nullptr;
}

#define CODES_PRODUCT_NAME2(b) codes_product_kernel_##b
#define CODES_PRODUCT_NAME(b) CODES_PRODUCT_NAME2(b)
ProductFn CODES_PRODUCT_NAME(CODE_BITS)(int dtype, int d, int L, int NT, bool aligned) {
    if (dtype == 0) return for_type<float>(d, L, NT, aligned);
    if (dtype == 1) return for_type<f16>(d, L, NT, aligned);
    return for_type<bf16>(d, L, NT, aligned);
}

}  // namespace idkm

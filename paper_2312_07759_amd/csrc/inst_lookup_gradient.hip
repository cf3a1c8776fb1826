// Gradients of lookups in stored tables: types and lengths of codewords.
#include <algorithm>

#include "embedding.h"
#include "layers.h"

namespace idkm {

template <typename T, bool FEW, bool SHARED>
static void (*gradient_for(int d))(const LookupGradArgs) {
    return d == 1 ? &k_lookup_gradient<T, 1, FEW, SHARED> : d == 2 ? &k_lookup_gradient<T, 2, FEW, SHARED>
           : d == 4 ? &k_lookup_gradient<T, 4, FEW, SHARED> : &k_lookup_gradient<T, 8, FEW, SHARED>;
}

void launch_lookup_gradient(int dtype, int d, const LookupGradPlan& p, const LookupGradArgs& args, hipStream_t s) {
    LookupGradArgs a = args;
    a.few = p.few;
    a.each = p.each;
    a.summing = (unsigned)p.grid;
    a.width_log = p.width_log;
    const unsigned clearing = p.few && a.dS ? (unsigned)std::min<int64_t>(512, ((int64_t)a.ids.rows + 63) / 64) : 0u;
    const int kd = a.k * d;
    // a stored group shorter than a row is a multiple of 32
    const int sums = a.segmented ? 16 : a.groups > 1 ? 512 / a.group : 1;
    for (a.sums_log = 0; 1 << a.sums_log < sums;) ++a.sums_log;
    const size_t lds = 4 * ((size_t)p.waves * ((kd << p.width_log) + LOOKUP_KEPT) + kd);
    BY_TYPE(dtype, T, {
        void (*fn)(const LookupGradArgs) = nullptr;
        if (p.width_log < 6) fn = p.few ? gradient_for<T, true, true>(d) : gradient_for<T, false, true>(d);
        else fn = p.few ? gradient_for<T, true, false>(d) : gradient_for<T, false, false>(d);
        allow_lds(reinterpret_cast<const void*>(fn), lds);
        hipLaunchKernelGGL(fn, dim3(a.summing + clearing), dim3((unsigned)p.waves * 64), lds, s, a);
    });
}

}  // namespace idkm

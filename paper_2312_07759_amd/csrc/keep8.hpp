// Activations kept in 8 bits: blocks of 32 columns of a row share a power of two 2^e, x = q 2^e with q in [-127, 127].
// A power of two so that every kept value is a number of x's own type (at most seven bits, none below the type's smallest): what is made of
// kept activations needs no further rounding, and the matrix instructions take them as they take x.
// e: the smallest with which the block's largest size, rounded, is at most 127, so errors are at most half of 2^e; in the type's last binade,
// where the next power would round to infinity, the largest values are cut to 127 2^e instead.  The byte E is e + 133, the exponent field of the block's
// largest size (1 for subnormal blocks) or one more.  q = -128 is no number: an infinity or NaN comes back as NaN, and has no part in e.
#pragma once
#include "elem.hpp"

namespace idkm {

constexpr int KEEP_BLOCK = 32;

template <typename T>
struct Keep8 {
    // the last exponent field of T's finite numbers, as float32's
    static constexpr int LAST = sizeof(T) == 4 ? 254 : __is_same(T, f16) ? 127 + 15 : 254;
    // top: bits of the block's largest finite size
    static __device__ __forceinline__ int field(uint32_t top) {
        const int f = max((int)(top >> 23), 1);
        // rounds beyond 127: a significand of 127.5 / 64 and more
        return f + ((top >> 23) >= 1 && f < LAST && (top & 0x7fffff) >= 0x7f0000 ? 1 : 0);
    }
    // x 2^-e to the nearest integer, ties to even, in two exact steps: 2^-e may lie beyond float32's range
    static __device__ __forceinline__ int quotient(float x, int field) {
        const float q = __builtin_rintf(ldexpf(x, 133 - field));
        return (__builtin_bit_cast(uint32_t, x) & 0x7fffffff) >= 0x7f800000 ? -128 : (int)fminf(fmaxf(q, -127.f), 127.f);
    }
    static __device__ __forceinline__ T value(int q, int field) { return q == -128 ? Elem<T>::nan() : Elem<T>::down(ldexpf((float)q, field - 133)); }
};

struct KeepArgs {
    void* X;  // T [n, ldx]
    int64_t n, cols, ldx;
    int8_t* Q;   // [n, 32 blocks]
    uint8_t* E;  // [n, blocks]
    int64_t blocks;
};

}  // namespace idkm

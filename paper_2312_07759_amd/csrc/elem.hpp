// Element types of the operators on quantised layers: float, IEEE half and bfloat16, with the 16-byte fragments that one
// lane hands to the matrix instructions.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace idkm {

typedef _Float16 f16;
typedef __bf16 bf16;
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x2 u32x2_word __attribute__((aligned(4)));
typedef u32x4 u32x4_word __attribute__((aligned(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));  // 16 bytes from any even address: global memory allows it
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <typename T>
struct Elem;
template <>
struct Elem<float> {
    static constexpr int PER16 = 4;  // elements in 16 bytes
    static __device__ float up(float x) { return x; }
    static __device__ float down(float x) { return x; }
    static __device__ float nan() { return __builtin_nanf(""); }
};
template <>
struct Elem<f16> {
    static constexpr int PER16 = 8;
    static __device__ float up(f16 x) { return (float)x; }
    static __device__ f16 down(float x) { return (f16)x; }  // to the nearest, ties to even
    static __device__ f16 nan() { return (f16)__builtin_nanf(""); }
};
template <>
struct Elem<bf16> {
    static constexpr int PER16 = 8;
    static __device__ float up(bf16 x) { return (float)x; }
    static __device__ bf16 down(float x) { return (bf16)x; }
    static __device__ bf16 nan() { return (bf16)__builtin_nanf(""); }
};

// acc[r] += sum over the fragments' elements of a[4 q + r] b[i]: the 16 x 16 block a b^T with the rows of a along acc's
// registers (lane l: i = l % 16 is its row of a and of b on input and its row of b on output, q = l / 16).  A lane holds 16
// bytes of its row: for 16-bit types elements 8 q .. 8 q + 7 of 32 in one instruction, for float elements 4 q .. 4 q + 3
// of 16, of which instruction e takes element e of every lane.  Sums are float32 in the matrix core.
template <typename T>
__device__ __forceinline__ void mma16(floatx4& acc, u32x4 a, u32x4 b) {
    if constexpr (sizeof(T) == 4) {
        const floatx4 fa = __builtin_bit_cast(floatx4, a), fb = __builtin_bit_cast(floatx4, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[e], fb[e], acc, 0, 0, 0);
    } else if constexpr (__is_same(T, f16)) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), acc, 0, 0, 0);
    } else {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
    }
}

}  // namespace idkm

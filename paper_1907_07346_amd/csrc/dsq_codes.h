// What the kernels that multiply with 4-bit messages share: codes as matrix operands, and where they lie in a message.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dsq {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x4 u32x4_at4 __attribute__((aligned(4)));             // a message is aligned to its words only
typedef u32x2 u32x2_at4 __attribute__((aligned(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// The 16-bit type that operands are multiplied in, and how many of them an input of type T is the sum of.  bf16 has fp32's range,
// and three pieces of 8 bits hold all of an fp32 number.
template <typename T>
struct Operand {
    using type = T;
    static constexpr int pieces = 1;
};
template <>
struct Operand<float> {
    using type = __bf16;
    static constexpr int pieces = 3;
};
template <typename O>
using Eight = O __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x4 matrix_fma(Eight<__bf16> a, Eight<__bf16> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 matrix_fma(Eight<_Float16> a, Eight<_Float16> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// A code q as an operand: 0.5 + q / 32, whose upper mantissa bits are q: one shift and one and-or for two codes, where (2 q - 15) itself
// takes five times that.  kCentre = 0.5 + 7.5 / 32 is taken off again as a product of its own, sum (0.5 + q/32) x - sum kCentre x =
// sum (2 q - 15) x / 64: at most twice what the sum's terms are, so one or two bits of fp32's 24.  Not so for infinite x, whose sign
// the difference loses: results that are not finite are computed once more (see the callers).
constexpr float kCentre = 0.734375f, kPerCode = 64.f / 15.f;     // scale * kPerCode takes such a sum to the decoded one
template <typename O>
struct CodeBits;
template <>
struct CodeBits<__bf16> {
    static constexpr int shift = 3;
    static constexpr uint32_t mask = 0x00780078u, one = 0x3F003F00u, centre = 0x3F3C3F3Cu;
};
template <>
struct CodeBits<_Float16> {
    static constexpr int shift = 6;
    static constexpr uint32_t mask = 0x03C003C0u, one = 0x38003800u, centre = 0x39E039E0u;
};
// Two codes: nibble N of either half of w.
template <typename O, int N>
__device__ __forceinline__ uint32_t code_pair(uint32_t w) {
    using B = CodeBits<O>;
    constexpr int by = 4 * N - B::shift;
    const uint32_t v = by > 0 ? w >> (by > 0 ? by : 0) : w << (by > 0 ? 0 : -by);
    return (v & B::mask) | B::one;
}
// The eight codes of a word, in the order 0 4 1 5 2 6 3 7.
template <typename O>
__device__ __forceinline__ Eight<O> code_operand(uint32_t w) {
    const u32x4 v = {code_pair<O, 0>(w), code_pair<O, 1>(w), code_pair<O, 2>(w), code_pair<O, 3>(w)};
    return __builtin_bit_cast(Eight<O>, v);
}
template <typename O>
__device__ __forceinline__ Eight<O> centre_operand() {
    constexpr uint32_t c = CodeBits<O>::centre;
    const u32x4 v = {c, c, c, c};
    return __builtin_bit_cast(Eight<O>, v);
}
// Eight numbers as operands: `pieces` of them, largest first, whose sum they are.
template <typename O, int P>
__device__ __forceinline__ void split_operand(const float (&x)[8], Eight<O> (&out)[P]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float rest = x[e];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const O piece = (O)rest;
            out[p][e] = piece;
            rest -= (float)piece;
        }
    }
}

}  // namespace
}  // namespace dsq

// What the kernels that multiply with 4-bit messages share: codes as matrix operands, and where they lie in a message.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace dsq {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x4 u32x4_at4 __attribute__((aligned(4)));             // a message is aligned to its words only
typedef u32x2 u32x2_at4 __attribute__((aligned(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <typename O>
using Eight = O __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x4 matrix_fma(Eight<__bf16> a, Eight<__bf16> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 matrix_fma(Eight<_Float16> a, Eight<_Float16> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
// Sixteen products of blocks of 4 x 4 with sums of four: lane l has row l % 4 of one operand and column l % 4 of the other, both of block l / 4, and gets that
// column of the result, whose register l % 4 is the product of what it gave itself.
template <typename O>
__device__ __forceinline__ f32x4 own_products(u32x2 a, u32x2 b, f32x4 c) {
    typedef short Bits __attribute__((ext_vector_type(4)));
    typedef _Float16 Halves __attribute__((ext_vector_type(4)));
    if constexpr (std::is_same_v<O, _Float16>) return __builtin_amdgcn_mfma_f32_4x4x4f16(__builtin_bit_cast(Halves, a), __builtin_bit_cast(Halves, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(__builtin_bit_cast(Bits, a), __builtin_bit_cast(Bits, b), c, 0, 0, 0);
}

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
    static constexpr uint32_t mask = 0x03C003C0u, one = 0x38003800u;
};
// Two codes: nibble N of either half of w.  (mask in a vector register and one in a scalar register are what the instruction that does both takes.)
struct CodeMasks {
    uint32_t mask, one;
};
template <typename O>
__device__ __forceinline__ CodeMasks code_masks() {
    CodeMasks m{CodeBits<O>::mask, CodeBits<O>::one};
    asm("" : "+v"(m.mask));
    asm("" : "+s"(m.one));
    return m;
}
template <typename O, int N>
__device__ __forceinline__ uint32_t code_pair(uint32_t w, CodeMasks m) {
    constexpr int by = 4 * N - CodeBits<O>::shift;
    const uint32_t v = by > 0 ? w >> (by > 0 ? by : 0) : w << (by > 0 ? 0 : -by);
    return (v & m.mask) | m.one;
}
// The eight codes of a word, in the order 0, 4, 1, 5, 2, 6, 3, 7.
template <typename O>
__device__ __forceinline__ Eight<O> code_operand(uint32_t w, CodeMasks m) {
    const u32x4 v = {code_pair<O, 0>(w, m), code_pair<O, 1>(w, m), code_pair<O, 2>(w, m), code_pair<O, 3>(w, m)};
    return __builtin_bit_cast(Eight<O>, v);
}
// Eight columns of a 16-bit type in that order.
__device__ __forceinline__ u32x4 in_code_order(u32x4 v) {
    return {__builtin_amdgcn_perm(v.z, v.x, 0x05040100u), __builtin_amdgcn_perm(v.z, v.x, 0x07060302u), __builtin_amdgcn_perm(v.w, v.y, 0x05040100u),
            __builtin_amdgcn_perm(v.w, v.y, 0x07060302u)};
}
template <typename O>
__device__ __forceinline__ Eight<O> centre_operand() {
    constexpr uint32_t c = CodeBits<O>::centre;
    const u32x4 v = {c, c, c, c};
    return __builtin_bit_cast(Eight<O>, v);
}
// Eight numbers as operands: P of them, largest first, whose sum they are (but for what is below the last one's last bit).
template <int P>
__device__ __forceinline__ void split_operand(const float (&x)[8], Eight<__bf16> (&out)[P]) {
    typedef float Two __attribute__((ext_vector_type(2)));
    typedef __bf16 Pair __attribute__((ext_vector_type(2)));
    u32x4 bits[P];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        Two rest = {x[2 * e], x[2 * e + 1]};
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const uint32_t v = __builtin_bit_cast(uint32_t, __builtin_convertvector(rest, Pair));
            bits[p][e] = v;
            if (p + 1 < P) {
                rest.x -= __uint_as_float(v << 16);
                rest.y -= __uint_as_float(v & 0xFFFF0000u);
            }
        }
    }
#pragma unroll
    for (int p = 0; p < P; ++p) out[p] = __builtin_bit_cast(Eight<__bf16>, bits[p]);
}

}  // namespace
}  // namespace dsq

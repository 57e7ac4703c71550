// What the kernels over rows of logits share: the order of logits, and sums of exponentials around a running maximum.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dsq {
namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// A logit's place in the row's order as one number: larger values first, +0 and -0 alike, NaN above all, and among equal values the lower
// index above the higher.  0 is below every rank and ~0 above.
__device__ __forceinline__ uint32_t logit_key(float z) {
    if (z != z) return 0xFFFFFFFEu;
    const uint32_t bits = __float_as_uint(z + 0.f);            // -0 + 0 = +0
    return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}
__device__ __forceinline__ uint64_t logit_rank(float z, uint32_t index) { return (uint64_t)logit_key(z) << 32 | (uint32_t)~index; }
__device__ __forceinline__ uint32_t rank_index(uint64_t rank) { return ~(uint32_t)rank; }

// 2^x as the hardware has it: results below 2^-126 are 0.
__device__ __forceinline__ float power2(float x) { return __builtin_amdgcn_exp2f(x); }

// sum over some logits of 2^(scale (z - max)), with scale = log2(e) / temperature.  The maximum that is subtracted is taken as 0 where it
// is infinite: a row of minus infinities has sum 0, one with plus infinity has an infinite sum.
struct Spread {
    float max, sum;
};
constexpr Spread kNoSpread{-__builtin_huge_valf(), 0.f};
__device__ __forceinline__ float reference(float max) { return fabsf(max) == __builtin_huge_valf() ? 0.f : max; }
__device__ __forceinline__ Spread spread_of(float z) { return {z, z == -__builtin_huge_valf() ? 0.f : z == __builtin_huge_valf() ? z : 1.f}; }
__device__ __forceinline__ Spread join(Spread a, Spread b, float scale) {
    const float m = fmaxf(a.max, b.max), r = reference(m);
    // (An empty or all-masked side has sum 0 and a reference of 0, which may lie far above the other's maximum.)
    const float sa = a.sum == 0.f ? 0.f : a.sum * exp2f((reference(a.max) - r) * scale);
    const float sb = b.sum == 0.f ? 0.f : b.sum * exp2f((reference(b.max) - r) * scale);
    return {m, sa + sb};
}
// Joins the spreads of a workgroup's WAVES * 64 threads, in an order that is always the same; every thread gets the result.  sums: 2 * WAVES floats of LDS.
template <int WAVES>
__device__ Spread workgroup_spread(Spread s, float scale, float* sums) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) s = join(s, Spread{__shfl_xor(s.max, o), __shfl_xor(s.sum, o)}, scale);
    if (WAVES == 1) return s;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
        sums[2 * (threadIdx.x / 64)] = s.max;
        sums[2 * (threadIdx.x / 64) + 1] = s.sum;
    }
    __syncthreads();
    s = kNoSpread;
    for (int w = 0; w < WAVES; ++w) s = join(s, Spread{sums[2 * w], sums[2 * w + 1]}, scale);
    return s;
}
// ln of the sum of exp(z / temperature).
__device__ __forceinline__ float spread_lse(Spread s, float temperature) { return reference(s.max) / temperature + kLn2 * log2f(s.sum); }

}  // namespace
}  // namespace dsq

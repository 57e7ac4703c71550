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
// The larger one; NaN if there is one.
__device__ __forceinline__ float max_or_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// sum over some logits z of 2^(scale z - at), with scale = log2(e) / temperature, and the largest of them.  `at` is the largest times scale, as rounded: terms
// and sum share it, whatever it is, and one multiply-add makes an exponent of a logit.  NaN anywhere makes all of it NaN.
constexpr float kInf = __builtin_huge_valf();
struct Spread {
    float max, sum;
};
constexpr Spread kNoSpread{-kInf, 0.f};
// What exponents are made with.  Where the largest is infinite they count from 0: a row of minus infinities has sum 0, one with plus infinity an infinite
// sum.  Where the largest is finite but not with the factor, numbers lie so far apart that only those equal to it count, with any factor.
struct Exponents {
    float scale, at;
    __device__ float operator()(float z) const { return power2(fmaf(z, scale, -at)); }
};
__device__ __forceinline__ Exponents exponents(float max, float scale) {
    const float at = max * scale;
    if (fabsf(at) != kInf) return {scale, at};
    if (fabsf(max) == kInf) return {scale, 0.f};
    return {1.f, max};
}
__device__ __forceinline__ Spread spread_of(float z) { return {z, z == -kInf ? 0.f : z == kInf ? z : z == z ? 1.f : z}; }
__device__ __forceinline__ Spread join(Spread a, Spread b, float scale) {
    const float m = max_or_nan(a.max, b.max), at = exponents(m, scale).at;
    // (An empty or all-masked side has sum 0 and counts from 0, which may lie far above the other's largest.)
    const float sa = a.sum == 0.f ? 0.f : a.sum * power2(exponents(a.max, scale).at - at);
    const float sb = b.sum == 0.f ? 0.f : b.sum * power2(exponents(b.max, scale).at - at);
    return {m, sa + sb};
}
// Adds M times N logits whose largest is `most` (-inf counts for nothing).
template <int M, int N>
__device__ __forceinline__ void add_logits(Spread& s, const float (&z)[M][N], float most, float scale) {
    const float m = max_or_nan(s.max, most);
    const Exponents e = exponents(m, scale);
    float total = s.sum == 0.f ? 0.f : s.sum * power2(exponents(s.max, scale).at - e.at);
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
        for (int k = 0; k < N; ++k) total += e(z[i][k]);
    s = {m, total};
}
template <int N>
__device__ __forceinline__ float largest_of(const float (&z)[N]) {
    float m = z[0];
#pragma unroll
    for (int e = 1; e < N; ++e) m = max_or_nan(m, z[e]);
    return m;
}
// op over 2, 4, 8 or 16 adjacent lanes, or all 64, in all of them and in an order that is always the same: a lane with its neighbour, with the other two of
// its four, with its mirror image in eight and in sixteen, and the four sixteens one after the other.
template <int CTRL, typename V>
__device__ __forceinline__ V other_lane(V v) {
    return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
template <int LANES, typename V, typename F>
__device__ __forceinline__ V over_lanes(V v, F op) {
    if (LANES >= 2) v = op(v, other_lane<0xB1>(v));               // quad_perm 1 0 3 2
    if (LANES >= 4) v = op(v, other_lane<0x4E>(v));               // quad_perm 2 3 0 1
    if (LANES >= 8) v = op(v, other_lane<0x141>(v));              // row_half_mirror
    if (LANES >= 16) v = op(v, other_lane<0x140>(v));             // row_mirror
    if (LANES == 64) {
        auto sixteen = [&](int of) { return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), of)); };
        v = op(op(sixteen(0), sixteen(16)), op(sixteen(32), sixteen(48)));
    }
    return v;
}
template <int LANES>
__device__ __forceinline__ float total_over_lanes(float v) {
    return over_lanes<LANES>(v, [](float a, float b) { return a + b; });
}
// Joins the lanes' spreads as join does, but the largest first, so that each sum is scaled once (8 x 32003, fp32, k = 16, a row's whole gradient: 11.3 us with
// joins two by two over lane shuffles).
template <int LANES>
__device__ __forceinline__ Spread spread_over_lanes(Spread s, float scale) {
    const float m = over_lanes<LANES>(s.max, [](float a, float b) { return max_or_nan(a, b); });
    return {m, total_over_lanes<LANES>(s.sum == 0.f ? 0.f : s.sum * power2(exponents(s.max, scale).at - exponents(m, scale).at))};
}
// Joins the spreads of a workgroup's WAVES * 64 threads; every thread gets the result.  sums: 2 * WAVES floats of LDS.
template <int WAVES>
__device__ Spread workgroup_spread(Spread s, float scale, float* sums) {
    static_assert(WAVES <= 16 && (WAVES & (WAVES - 1)) == 0);
    s = spread_over_lanes<64>(s, scale);
    if (WAVES == 1) return s;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
        sums[2 * (threadIdx.x / 64)] = s.max;
        sums[2 * (threadIdx.x / 64) + 1] = s.sum;
    }
    __syncthreads();
    const int w = threadIdx.x & (WAVES - 1);
    return spread_over_lanes<WAVES>(Spread{sums[2 * w], sums[2 * w + 1]}, scale);
}
// ln of the sum of exp(z / temperature) is base + rest: the largest (0 where that is infinite) and, for what `at` was rounded to, the sum.
struct LogSum {
    float from, rest;                                             // base = from / temperature
};
__device__ __forceinline__ LogSum log_sum(Spread s, float scale) {
    const Exponents e = exponents(s.max, scale);
    const float from = fabsf(s.max) == kInf ? 0.f : s.max;
    return {from, kLn2 * (log2f(s.sum) - fmaf(from, e.scale, -e.at))};
}

// 16 bytes of logits, at any element's address.
template <typename T>
struct Pieces {
    static constexpr uint32_t E = 16 / sizeof(T);
    typedef T Piece __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
};

}  // namespace
}  // namespace dsq

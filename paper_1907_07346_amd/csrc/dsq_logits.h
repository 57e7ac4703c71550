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
// What exponents are made with.  The rounding of `at` makes the largest's own term 2^-64 to 2^64 as long as |at| < 2^31.  From there on neighbours in fp32 are
// 64 or more apart in the exponent, so that only what equals the largest counts (2^31 others add 2^-33 of it): any factor that tells them apart will do, and
// a power of two makes its term 1.  Where the largest is infinite exponents count from 0: a row of minus infinities has sum 0, one with plus infinity an
// infinite sum.
struct Exponents {
    float scale, at;
    bool alone;                                                   // only what equals the largest counts
    __device__ float operator()(float z) const { return power2(fmaf(z, scale, -at)); }
};
__device__ __forceinline__ Exponents exponents(float max, float scale) {
    const float at = max * scale;
    if (!(fabsf(at) >= 2147483648.f)) return {scale, at, false};  // (and NaN)
    if (fabsf(max) == kInf) return {scale, 0.f, false};
    const uint32_t up = 380u - (__float_as_uint(max) >> 23 & 255u);                        // |max| times it lies between 2^126 and 2^127
    const float apart = __uint_as_float((up < 254u ? up : 254u) << 23);
    return {apart, max * apart, true};
}
__device__ __forceinline__ Spread spread_of(float z, float scale) { return {z, exponents(z, scale)(z)}; }
// The sum of s when it counts from e, the exponents of `max`, which is at least s.max.  (Exponents of another kind than e's are never subtracted from its.)
__device__ __forceinline__ float sum_from(Spread s, float max, Exponents e, float scale) {
    if (s.sum == 0.f || s.max == max) return s.sum;               // (an empty or all-masked side counts from 0, which may lie far above)
    const Exponents own = exponents(s.max, scale);
    return own.alone || e.alone ? 0.f : s.sum * power2(own.at - e.at);
}
__device__ __forceinline__ Spread join(Spread a, Spread b, float scale) {
    const float m = max_or_nan(a.max, b.max);
    const Exponents e = exponents(m, scale);
    return {m, sum_from(a, m, e, scale) + sum_from(b, m, e, scale)};
}
// Adds M times N logits whose largest is `most` (-inf counts for nothing).
template <int M, int N>
__device__ __forceinline__ void add_logits(Spread& s, const float (&z)[M][N], float most, float scale) {
    const float m = max_or_nan(s.max, most);
    const Exponents e = exponents(m, scale);
    float total = sum_from(s, m, e, scale);
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
    return {m, total_over_lanes<LANES>(sum_from(s, m, exponents(m, scale), scale))};
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

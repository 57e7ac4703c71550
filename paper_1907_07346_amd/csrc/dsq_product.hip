// Products with a matrix that is held as messages (ds_product).
#include "dsq_answers.h"

namespace dsq {
namespace {

__device__ __forceinline__ float wave_total(float v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// A wave per row and four tokens: each lane takes every 64th word (eight codes).  A code counts as (2 code - 15) / 16, below 1, so that a
// block's sum is not infinite before y is.
template <typename T>
__global__ void __launch_bounds__(256) product_kernel(ProductArgs a) {
    const uint64_t r = (uint64_t)blockIdx.x * 4 + threadIdx.x / 64;
    const uint64_t t0 = (uint64_t)blockIdx.y * 4;
    if (r >= a.rows) return;
    const uint32_t lane = threadIdx.x & 63, per = a.block / 8;
    const uint8_t* row = a.msg + r * a.row_bytes;
    const T* x = static_cast<const T*>(a.in);
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    for (uint64_t w = lane; w < (a.cols + 7) / 8; w += 64) {
        const uint8_t* block = row + w / per * (4 + a.block / 2);
        const float unit = *reinterpret_cast<const float*>(block) * (16.f / 15.f);
        const uint32_t word = *reinterpret_cast<const uint32_t*>(block + 4 + 4 * (w % per));
        for (int t = 0; t < 4; ++t) {
            if (t0 + t >= a.tokens) break;
            float part = 0.f;
            for (int e = 0; e < 8; ++e)
                if (8 * w + e < a.cols) part = fmaf((float)(2 * (int)(word >> (4 * e) & 15u) - 15) * 0.0625f, (float)x[(t0 + t) * a.in_ld + 8 * w + e], part);
            sum[t] = fmaf(unit, part, sum[t]);
        }
    }
    for (int t = 0; t < 4; ++t) {
        const float total = wave_total(sum[t]);
        if (lane == 0 && t0 + t < a.tokens) static_cast<T*>(a.out)[(t0 + t) * a.out_ld + r] = (T)total;
    }
}

}  // namespace

uint64_t product_work_bytes(const ds_matrix&) { return 0; }

hipError_t launch_product(const ProductArgs& a, hipStream_t stream) {
    const uint64_t tiles = (a.tokens + 3) / 4, most = 65535;
    for (uint64_t lo = 0; lo < tiles; lo += most) {
        ProductArgs b = a;
        const uint64_t n = tiles - lo < most ? tiles - lo : most;
        by_dtype(a.dtype, [&](auto kind) {
            using T = decltype(kind);
            b.in = static_cast<const T*>(a.in) + 4 * lo * a.in_ld;
            b.out = static_cast<T*>(a.out) + 4 * lo * a.out_ld;
            b.tokens = a.tokens - 4 * lo;
            hipLaunchKernelGGL(product_kernel<T>, dim3((unsigned)((a.rows + 3) / 4), (unsigned)n), dim3(256), 0, stream, b);
        });
    }
    return hipGetLastError();
}

}  // namespace dsq

// The gradient of ds_product with respect to its vectors (ds_product_gradient): products with the matrix's transpose.
#include "dsq_answers.h"

namespace dsq {
namespace {

// A thread per word (eight columns) and token.
template <typename T>
__global__ void __launch_bounds__(64) product_gradient_kernel(ProductArgs a) {
    const uint64_t w = (uint64_t)blockIdx.x * 64 + threadIdx.x, t = blockIdx.y;
    if (w >= (a.cols + 7) / 8) return;
    const uint32_t per = a.block / 8;
    const uint8_t* block = a.msg + w / per * (4 + a.block / 2);
    const T* dy = static_cast<const T*>(a.in) + t * a.in_ld;
    float sum[8] = {};
    for (uint64_t r = 0; r < a.rows; ++r, block += a.row_bytes) {
        const float d = (float)dy[r] * (*reinterpret_cast<const float*>(block) / 15.f);
        const uint32_t word = *reinterpret_cast<const uint32_t*>(block + 4 + 4 * (w % per));
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = fmaf((float)(2 * (int)(word >> (4 * e) & 15u) - 15), d, sum[e]);
    }
    for (int e = 0; e < 8; ++e)
        if (8 * w + e < a.cols) static_cast<T*>(a.out)[t * a.out_ld + 8 * w + e] = (T)sum[e];
}

}  // namespace

uint64_t product_gradient_work_bytes(const ds_matrix&) { return 0; }

hipError_t launch_product_gradient(const ProductArgs& a, hipStream_t stream) {
    const uint64_t most = 65535;
    for (uint64_t lo = 0; lo < a.tokens; lo += most) {
        ProductArgs b = a;
        const uint64_t n = a.tokens - lo < most ? a.tokens - lo : most;
        by_dtype(a.dtype, [&](auto kind) {
            using T = decltype(kind);
            b.in = static_cast<const T*>(a.in) + lo * a.in_ld;
            b.out = static_cast<T*>(a.out) + lo * a.out_ld;
            hipLaunchKernelGGL(product_gradient_kernel<T>, dim3((unsigned)(((a.cols + 7) / 8 + 63) / 64), (unsigned)n), dim3(64), 0, stream, b);
        });
    }
    return hipGetLastError();
}

}  // namespace dsq

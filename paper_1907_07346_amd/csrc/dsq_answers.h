// Internal declarations of the operators on messages and logits: what their host side (dsq_answers_host.cpp) hands to the
// kernels' launchers once a call has been checked.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dsq.h"

namespace dsq {

constexpr int kMaxTop = 256;              // pairs per row of logits

struct ProductArgs {
    const uint8_t* msg;
    const void* in;                       // x (product) or dy (gradient): tokens rows of pitch in_ld
    void* out;                            // y or dx: tokens rows of pitch out_ld
    void* work;
    uint64_t rows, cols, tokens, in_ld, out_ld;
    uint64_t row_bytes;                   // of the message
    uint32_t block;
    int32_t dtype;
};
uint64_t product_work_bytes(const ds_matrix& m);
hipError_t launch_product(const ProductArgs& a, hipStream_t stream);
uint64_t product_gradient_work_bytes(const ds_matrix& m);
hipError_t launch_product_gradient(const ProductArgs& a, hipStream_t stream);

struct LogitsArgs {
    const void* z;
    uint64_t rows, vocab, z_ld, dz_ld;
    uint32_t k;
    int32_t dtype;
    float temperature;
    uint2* pairs;                         // top logits: written
    float* lse;
    const uint2* given;                   // distillation: the teacher's pairs
    const float* teacher_lse;
    const float* weight;
    float* loss;
    void* dz;
    void* work;
};
uint64_t top_logits_work_bytes(const ds_logits& l);
hipError_t launch_top_logits(const LogitsArgs& a, hipStream_t stream);
uint64_t distill_work_bytes(const ds_logits& l);
hipError_t launch_distill(const LogitsArgs& a, hipStream_t stream);

// f(T()) with the C++ type of a ds_dtype.
template <typename F>
auto by_dtype(int32_t dtype, F f) {
    if (dtype == DS_BF16) return f(__bf16());
    if (dtype == DS_F16) return f(_Float16());
    return f(float());
}

}  // namespace dsq

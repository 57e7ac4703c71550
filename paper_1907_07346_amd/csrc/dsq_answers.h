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

struct SampleArgs {
    const void* z;
    uint64_t rows, vocab, z_ld;
    int32_t dtype, top_k;
    float temperature, top_p, min_p;
    ds_sampling_rows each;                                        // rows' own parameters in place of these
    const float* u;
    int32_t* token;
    float* logp;
    void* work;
};
uint64_t sample_work_bytes(const ds_sampling& s);
hipError_t launch_sample(const SampleArgs& a, hipStream_t stream);

// A tensor of a worker's gradient, as the table holds it: records[tensors + 1], the last one of no elements; behind them first_tile[workers + 1], the tiles before
// a worker's; behind those tensor_of[tiles].
constexpr uint32_t kGradientTile = 16384;                         // elements; the last tile of a tensor has fewer
struct TensorRecord {
    void* data;
    uint64_t count;
    uint64_t column;                                              // elements of the worker's tensors before it
    uint64_t first_tile;
    uint32_t dtype, worker;
    uint64_t worker_from;                                         // the tensor is the first one of this worker to `worker`, or this is worker + 1
};
inline uint64_t gradients_table_bytes(uint64_t workers, uint64_t tensors, uint64_t tiles) {
    return (tensors + 1) * sizeof(TensorRecord) + (workers + 1) * sizeof(uint64_t) + tiles * sizeof(uint32_t);
}
struct RecordBatch {                                              // of a launch, by value
    static constexpr uint32_t kMost = 64;
    TensorRecord record[kMost];
    uint64_t first, here;                                         // records before them, and how many
};
hipError_t launch_lay(const ds_gradients& g, const RecordBatch& batch, hipStream_t stream);
struct ClipArgs {
    ds_gradients g;
    double max_norm;
    float* out;                                                   // or NULL: in place
    uint64_t out_ld;
    float* norm;
    void* work;
};
uint64_t gradient_norm_work_bytes(const ds_gradients& g);
hipError_t launch_gradient_norm(const ClipArgs& a, hipStream_t stream);
uint64_t clip_work_bytes(const ds_gradients& g);
hipError_t launch_clip(const ClipArgs& a, hipStream_t stream);

// f(T()) with the C++ type of a ds_dtype.
template <typename F>
auto by_dtype(int32_t dtype, F f) {
    if (dtype == DS_BF16) return f(__bf16());
    if (dtype == DS_F16) return f(_Float16());
    return f(float());
}

}  // namespace dsq

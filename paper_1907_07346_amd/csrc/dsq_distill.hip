// The loss of a row of logits against a teacher's (index, logit) pairs, and its gradient (ds_distill).
#include "dsq_answers.h"
#include "dsq_logits.h"

namespace dsq {
namespace {

// A workgroup per row: the row's sum, the teacher's probabilities, the dense part of the gradient, then the listed columns.
template <typename T>
__global__ void __launch_bounds__(256) distill_kernel(LogitsArgs a) {
    __shared__ float sums[8];
    __shared__ uint32_t index[kMaxTop];
    __shared__ float prob[kMaxTop];
    const uint64_t row = blockIdx.x;
    const T* z = static_cast<const T*>(a.z) + row * a.z_ld;
    T* dz = a.dz ? static_cast<T*>(a.dz) + row * a.dz_ld : nullptr;
    const float scale = kLog2e / a.temperature, weight = a.weight ? a.weight[row] : 1.f;
    const uint32_t j = threadIdx.x;

    // teacher: ln p and p of entry j
    const uint2 pair = j < a.k ? a.given[row * a.k + j] : make_uint2(~0u, 0u);
    const bool listed = pair.x < a.vocab;
    const float teacher = __uint_as_float(pair.y);
    const float zj = listed ? (float)z[pair.x] : 0.f;
    const Spread ts = workgroup_spread<4>(listed ? spread_of(teacher) : kNoSpread, scale, sums);
    const Spread own = [&] {
        Spread s = kNoSpread;
        for (uint64_t v = j; v < a.vocab; v += 256) s = join(s, spread_of((float)z[v]), scale);
        return workgroup_spread<4>(s, scale, sums);
    }();
    // ln of p and of the student's probability: around the maxima, where what is subtracted is small
    const float lp = a.teacher_lse ? teacher / a.temperature - a.teacher_lse[row] : (teacher - reference(ts.max)) / a.temperature - kLn2 * log2f(ts.sum);
    const bool some = listed && teacher != -__builtin_huge_valf();
    const float p = some ? expf(lp) : 0.f;
    const float top = reference(own.max), lq = (zj - top) / a.temperature - kLn2 * log2f(own.sum);
    const float term = p != 0.f ? p * (lp - lq) : 0.f;
    index[j] = pair.x;
    prob[j] = p;
    __syncthreads();
    float mass = 0.f, loss = 0.f;
    for (uint32_t i = 0; i < a.k; ++i) mass += prob[i];
    __syncthreads();
    __shared__ float terms[kMaxTop];
    terms[j] = term;
    __syncthreads();
    for (uint32_t i = 0; i < a.k; ++i) loss += terms[i];
    const bool skip = weight == 0.f || mass == 0.f;
    if (a.loss && j == 0) a.loss[row] = skip ? 0.f : weight * loss;
    if (!dz) return;
    const float c = weight / a.temperature, each = c * mass / own.sum;
    for (uint64_t v = j; v < a.vocab; v += 256) dz[v] = (T)(skip ? 0.f : each * exp2f(((float)z[v] - top) * scale));
    __syncthreads();
    if (skip || !listed) return;
    float all = 0.f;
    for (uint32_t i = 0; i < a.k; ++i)
        if (index[i] == pair.x) {
            if (i < j) return;                                  // the first entry of an index writes it
            all += prob[i];
        }
    dz[pair.x] = (T)(each * exp2f((zj - top) * scale) - c * all);
}

}  // namespace

uint64_t distill_work_bytes(const ds_logits&) { return 0; }

hipError_t launch_distill(const LogitsArgs& a, hipStream_t stream) {
    by_dtype(a.dtype, [&](auto kind) {
        hipLaunchKernelGGL(distill_kernel<decltype(kind)>, dim3((unsigned)a.rows), dim3(256), 0, stream, a);
    });
    return hipGetLastError();
}

}  // namespace dsq

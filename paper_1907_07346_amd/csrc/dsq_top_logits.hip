// The largest logits of every row as (index, value) pairs, and the row's log-sum-exp (ds_top_logits).
#include "dsq_answers.h"
#include "dsq_logits.h"

namespace dsq {
namespace {

// A workgroup per row.  The next largest logit is the largest rank below the last one, k times over.
template <typename T>
__global__ void __launch_bounds__(256) top_logits_kernel(LogitsArgs a) {
    __shared__ uint64_t scratch[4];
    __shared__ float sums[8];
    __shared__ uint64_t found[kMaxTop];
    const T* z = static_cast<const T*>(a.z) + (uint64_t)blockIdx.x * a.z_ld;
    uint64_t last = ~0ull;
    for (uint32_t j = 0; j < a.k; ++j) {
        uint64_t best = 0;
        for (uint64_t v = threadIdx.x; v < a.vocab; v += 256) {
            const uint64_t rank = logit_rank((float)z[v], (uint32_t)v);
            if (rank < last && rank > best) best = rank;
        }
        for (int o = 32; o; o >>= 1) {
            const uint64_t other = __shfl_xor((unsigned long long)best, o);
            best = other > best ? other : best;
        }
        __syncthreads();
        if ((threadIdx.x & 63) == 0) scratch[threadIdx.x / 64] = best;
        __syncthreads();
        for (int w = 0; w < 4; ++w) best = scratch[w] > best ? scratch[w] : best;
        last = best;
        if (threadIdx.x == 0) found[j] = best;
    }
    __syncthreads();
    for (uint32_t j = threadIdx.x; j < a.k; j += 256) {
        const uint32_t at = rank_index(found[j]);
        uint32_t place = 0;
        for (uint32_t i = 0; i < a.k; ++i) place += rank_index(found[i]) < at ? 1u : 0u;
        a.pairs[(uint64_t)blockIdx.x * a.k + place] = make_uint2(at, __float_as_uint((float)z[at]));
    }
    if (!a.lse) return;
    const float scale = kLog2e / a.temperature;
    Spread s = kNoSpread;
    for (uint64_t v = threadIdx.x; v < a.vocab; v += 256) s = join(s, spread_of((float)z[v]), scale);
    s = workgroup_spread<4>(s, scale, sums);
    if (threadIdx.x == 0) a.lse[blockIdx.x] = spread_lse(s, a.temperature);
}

}  // namespace

uint64_t top_logits_work_bytes(const ds_logits&) { return 0; }

hipError_t launch_top_logits(const LogitsArgs& a, hipStream_t stream) {
    by_dtype(a.dtype, [&](auto kind) {
        hipLaunchKernelGGL(top_logits_kernel<decltype(kind)>, dim3((unsigned)a.rows), dim3(256), 0, stream, a);
    });
    return hipGetLastError();
}

}  // namespace dsq
